"""Rotary positions, the microscaled 4-bit cache and the attention over it without a GPU: the oracle against plain library routines, frequencies, plans and their
refusals, and every plan's accesses walked on the host against the buffers."""
import ctypes
import math

import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx
from oracle import serve_oracle as so

torch = pytest.importorskip("torch")


def _refused(status, make):
    with pytest.raises(lc.LayoutCopyError) as e:
        make()
    assert e.value.status_name == status, e.value


# ---- the oracle ----
def test_oracle_rotation_is_a_product_of_complex_numbers():
    rng = np.random.default_rng(0)
    x, p, f = rng.standard_normal((5, 3, 12)), rng.integers(-1000, 100000, 5), rng.random(4).astype(np.float32)
    for pairs in ("half", "neighbours"):
        a, b = (slice(0, 4), slice(4, 8)) if pairs == "half" else (slice(0, 8, 2), slice(1, 8, 2))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * p[:, None, None] * f.astype(np.float64)) * 1.5
        y, _ = so.rotate(x, p, f, 8, pairs, factor=1.5)
        assert np.allclose(y[..., a], z.real) and np.allclose(y[..., b], z.imag) and (y[..., 8:] == x[..., 8:]).all()
        back, _ = so.rotate(y, p, f, 8, pairs, transposed=True, factor=1 / 1.5)   # the other way undoes it
        assert np.allclose(back, x)


def test_oracle_attention_is_torchs():
    rng = np.random.default_rng(1)
    T, heads, kv, D, length, page = 6, 4, 2, 64, 40, 8
    codes = rng.integers(0, 256, 10 * page * kv * D // 2, dtype=np.uint8)
    scales = rng.integers(124, 128, 10 * page * kv * D // 32, dtype=np.uint8)
    ct, st = "(80,2,64):(128,64,1)", "(80,2,2):(4,2,1)"
    pool = so.Pool(codes, ct, scales, st, D)
    q = rng.standard_normal((T, heads, D))
    table = rng.permutation(10)[:5][None]
    o, lse = np.zeros((T, heads, D)), np.zeros((T, heads))
    so.attention(q, pool, pool, heads // kv, 1, page, 5, T, [length], None, table, 0.3, True, 0, o, lse)
    slots = table[0][np.arange(length) // page] * page + np.arange(length) % page
    k = torch.from_numpy(np.repeat(pool(slots), heads // kv, 1)).transpose(0, 1)
    mask = torch.arange(length)[None] <= torch.arange(length - T, length)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), k, k, attn_mask=mask, scale=0.3)
    assert np.allclose(o, want.transpose(0, 1).numpy())


def test_oracle_writes_what_it_reads():
    rng = np.random.default_rng(2)
    ct, st = "((4,3),2,64):((64,512),256,1)", "((4,3),2,2):((2,16),8,1)"
    codes, scales = rng.integers(0, 256, 768, dtype=np.uint8), rng.integers(0, 256, 48, dtype=np.uint8)
    x = rng.choice([0.0, 1.0, -6.0, 3.0, 0.5], (3, 2, 50))
    x[:, :, ::32] = 6.0   # the block's scale is 1
    before = codes.copy()
    so.write_slots(codes, ct, scales, st, [7, -1, 0], x, "cover")
    got = so.read_slots(codes, ct, scales, st, np.array([7, 0]))
    assert (got[:, :, :50] == x[[0, 2]]).all() and (got[:, :, 50:] == 0).all()
    assert (codes != before).sum() <= 2 * 2 * 32


# ---- frequencies ----
def test_frequencies():
    plain = np.array(lc.lc_rope_frequencies(128, 10000.0))
    want = 10000.0 ** (-np.arange(64) / 64)
    assert (plain == want.astype(np.float32)).all()
    assert (np.array(lc.lc_rope_frequencies(128, 10000.0, "linear", 8.0)) == (want / 8).astype(np.float32)).all()
    base = np.array(lc.lc_rope_frequencies(128, 10000.0, "base", 8.0))
    assert base[0] == 1.0 and abs(base[-1] / (want[-1] / 8) - 1) < 2 ** -22   # (fp32's rounding, and that of the powers)
    # ramps: as it is above `fast` turns, stretched below `slow`, between them in between
    turns = 4096 * want / (2 * math.pi)
    for rule in ("parts", "bands"):
        f = np.array(lc.lc_rope_frequencies(128, 10000.0, rule, 16.0, 4096, 1.0, 32.0))
        ratio = f / want
        assert (abs(ratio[turns > 40] - 1) < 2 ** -23).all() and (abs(ratio[turns < 0.8] * 16 - 1) < 2 ** -22).all()
        inside = (turns < 28) & (turns > 1.2)
        assert inside.sum() > 10 and (ratio[inside] < 1).all() and (ratio[inside] > 1 / 16).all() and (np.diff(ratio) <= 2 ** -22).all()
    first, last = math.floor(64 * math.log(4096 / (32 * 2 * math.pi)) / math.log(10000)), math.ceil(64 * math.log(4096 / (2 * math.pi)) / math.log(10000))
    parts = np.array(lc.lc_rope_frequencies(128, 10000.0, "parts", 16.0, 4096, 1.0, 32.0))
    keep = np.clip(1 - (np.arange(64) - first) / (last - first), 0, 1)
    assert np.allclose(parts, want * keep + want / 16 * (1 - keep), rtol=2 ** -22, atol=0)
    bands = np.array(lc.lc_rope_frequencies(128, 10000.0, "bands", 8.0, 8192, 1.0, 4.0))
    keep = np.clip((8192 * want / (2 * math.pi) - 1) / 3, 0, 1)
    assert np.allclose(bands, want * keep + want / 8 * (1 - keep), rtol=2 ** -22, atol=0)


@pytest.mark.parametrize("args", [(127,), (0,), (64, 1.0), (64, 0.5), (64, 10000.0, "linear", 0.5), (64, float("nan")), (64, 10000.0, "linear", float("inf")), (2, 10000.0, "base", 2.0),
                                  (64, 10000.0, "parts", 2.0, 0), (64, 10000.0, "parts", 2.0, 100, 2.0, 1.0), (64, 10000.0, "bands", 2.0, 100, 0.0, 1.0)])
def test_frequencies_refused(args):
    _refused("INVALID_ARG", lambda: lc.lc_rope_frequencies(*args))


# ---- plans of rotary positions ----
def _dense(T, H, D, order="thd"):
    return {"thd": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, H * D, D), "htd": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, D, T * D), "gaps": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, H * D + 24, D + 3 if T == 1 else D),
            "dht": "(%d,%d,%d):(1,%d,%d)" % (T, H, D, T, T * H), "back": "(%d,%d,%d):(-%d,%d,1)" % (T, H, D, H * D, D)}[order]


@pytest.mark.parametrize("T,H,D,rotary", [(1, 1, 2, 2), (1, 1, 1 + 2, 2), (5, 3, 64, 64), (7, 40, 128, 64), (64, 40, 128, 128), (33, 9, 80, 40), (130, 1, 96, 96), (3, 2, 4096, 4096), (2, 70, 256, 256), (2000, 12, 80, 80)])
@pytest.mark.parametrize("pairs", ["half", "neighbours"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rope_walk(T, H, D, rotary, pairs, dtype):
    es = lc.DTYPE_BYTES[dtype]
    for order in ("thd", "htd", "dht", "back"):
        x, y = _dense(T, H, D, order), _dense(T, H, D)
        plan = lc.RopePlan(x, y, dtype, rotary, pairs)
        L, M = lc.Layout(x), lc.Layout(y)
        assert plan.debug_walk_on_host(-L.min_offset * es, L.cosize * es, 0, M.cosize * es) == T * H * D * es, plan.describe()
        with pytest.raises(lc.LayoutCopyError):
            plan.debug_walk_on_host(-L.min_offset * es, L.cosize * es, 0, M.cosize * es - 1)


@pytest.mark.parametrize("x,y,dtype,rotary,status", [
    ("(4,2,64):(128,64,1)", "(4,2,64):(128,64,1)", "f32", 63, "INVALID_ARG"),
    ("(4,2,64):(128,64,1)", "(4,2,64):(128,64,1)", "f32", 66, "INVALID_ARG"),
    ("(4,2,64):(128,64,1)", "(4,2,64):(128,64,1)", "f32", 0, "INVALID_ARG"),
    ("(4,128):(128,1)", "(4,2,64):(128,64,1)", "f32", 64, "INVALID_ARG"),
    ("(4,2,64):(128,64,1)", "(4,2,62):(128,64,1)", "f32", 62, "SIZE_MISMATCH"),
    ("(4,2,64):(128,64,1)", "(4,2,64):(128,32,1)", "f32", 64, "DST_ALIASES"),
    ("(4,2,64):(128,64,1)", "(4,2,64):(128,64,1)", "b16", 64, "UNSUPPORTED_DTYPE"),
    ("(4,2,64):(128,64,1)", "(4,2,64):(128,64,1)", "mxfp4", 64, "UNSUPPORTED_DTYPE"),
    ("(1,1,8192):(1,1,1)", "(1,1,8192):(1,1,1)", "f32", 64, "TOO_LARGE"),
    ("(2147483648,1,2):(2,1,1)", "(2147483648,1,2):(2,1,1)", "f32", 2, "TOO_LARGE"),
    ("((2,2,2,2,2),1,2):((2,100,1000,5000,20000),1,1)", "(32,1,2):(2,1,1)", "f32", 2, "TOO_LARGE"),
])
def test_rope_refused(x, y, dtype, rotary, status):
    _refused(status, lambda: lc.RopePlan(x, y, dtype, rotary))


def test_rope_of_more_workgroups_than_a_grid_holds():
    """One unit a lane would need a grid of more than 2^32 lanes: four are taken."""
    assert "T=20000000" in lc.RopePlan(_dense(20000000, 32, 64), _dense(20000000, 32, 64), "f16", 64).describe()
    _refused("TOO_LARGE", lambda: lc.RopePlan(_dense(200000000, 32, 64), _dense(200000000, 32, 64), "f16", 64))


# ---- plans of the cache ----
def _pool(slots, heads, width, page=None, order="heads"):
    """Layouts of codes and scales."""
    def text(w):
        if page is None:
            return "(%d,%d,%d):(%d,%d,1)" % (slots, heads, w, heads * w, w)
        pages = slots // page
        if order == "heads":
            return "((%d,%d),%d,%d):((%d,%d),%d,1)" % (page, pages, heads, w, w, heads * page * w, page * w)
        return "((%d,%d),%d,%d):((%d,%d),%d,1)" % (page, pages, heads, w, heads * w, page * heads * w, w)
    return text(width), text(width // 32)


@pytest.mark.parametrize("T,H,D,width,page,order", [(1, 1, 1, 32, None, "heads"), (5, 3, 64, 64, 8, "heads"), (40, 8, 128, 128, 16, "heads"), (33, 5, 80, 96, 16, "tokens"), (7, 1, 256, 320, 4, "tokens"),
                                                    (300, 8, 128, 128, 64, "heads"), (1200, 8, 64, 64, 16, "tokens")])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_cache_walk(T, H, D, width, page, order, dtype):
    rng = np.random.default_rng(T)
    slots_n = 2 * T // (page or 1) * (page or 1) + 2 * (page or 1)
    codes, scales = _pool(slots_n, H, width, page, order)
    slots = rng.permutation(slots_n - 1)[:T].astype(np.int32)
    slots[0] = slots_n - 1   # the last one, too
    if T > 2:
        slots[1:-1:5] = [-1, slots_n, -2 ** 31, 2 ** 31 - 1][T % 4]   # nobody's
    there = int(((slots >= 0) & (slots < slots_n)).sum())
    es, q, s = lc.DTYPE_BYTES[dtype], lc.Layout(codes).cosize // 2, lc.Layout(scales).cosize
    for x_order in ("thd", "htd", "dht", "back"):
        x = lc.Layout(_dense(T, H, D, x_order))
        write, read = lc.MxCacheWritePlan(x, codes, scales, dtype), lc.MxCacheReadPlan(codes, scales, x, dtype)
        before, size = -x.min_offset * es, x.cosize * es
        assert write.debug_walk_on_host(slots, before, size, q, s) == there * H * (width // 2 + width // 32), write.describe()
        assert read.debug_walk_on_host(slots, before, size, q, s) == there * H * D * es, read.describe()
        for short in ((before, size, q - 1, s), (before, size, q, s - 1)):
            with pytest.raises(lc.LayoutCopyError):
                write.debug_walk_on_host(slots, *short)
        with pytest.raises(lc.LayoutCopyError):
            read.debug_walk_on_host(slots, before, size - 1, q, s)
        twice = np.full(T, slots_n - 1, np.int32)   # reads may name a slot more than once
        assert read.debug_walk_on_host(twice, before, size, q, s) == T * H * D * es


@pytest.mark.parametrize("x,codes,scales,dtype,status", [
    ("(4,2,64):(128,64,1)", "(8,2,80):(160,80,1)", "(8,2,2):(4,2,1)", "f32", "SIZE_MISMATCH"),
    ("(4,2,65):(130,65,1)", "(8,2,64):(128,64,1)", "(8,2,2):(4,2,1)", "f32", "SIZE_MISMATCH"),
    ("(4,3,64):(192,64,1)", "(8,2,64):(128,64,1)", "(8,2,2):(4,2,1)", "f32", "SIZE_MISMATCH"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(128,64,1)", "(8,2,3):(6,3,1)", "f32", "SIZE_MISMATCH"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(128,64,1)", "(9,2,2):(4,2,1)", "f32", "SIZE_MISMATCH"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(128,64,2)", "(8,2,2):(4,2,1)", "f32", "BLOCK_LAYOUT"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(144,72,1)", "(8,2,2):(4,2,1)", "f32", "BLOCK_LAYOUT"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(-128,64,1)", "(8,2,2):(4,2,1)", "f32", "NEGATIVE_STRIDE"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(128,64,1)", "(8,2,2):(4,-2,1)", "f32", "NEGATIVE_STRIDE"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(64,64,1)", "(8,2,2):(4,2,1)", "f32", "DST_ALIASES"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(128,64,1)", "(8,2,2):(3,2,1)", "f32", "DST_ALIASES"),
    ("(4,2,64):(128,64,1)", "(8,2,64):(128,64,1)", "(8,2,2):(4,2,1)", "b16", "UNSUPPORTED_DTYPE"),
    ("(4,128):(128,1)", "(8,2,64):(128,64,1)", "(8,2,2):(4,2,1)", "f32", "INVALID_ARG"),
    ("(4,2,64):(128,64,1)", "(8,128):(128,1)", "(8,4):(4,1)", "f32", "INVALID_ARG"),
])
def test_cache_refused(x, codes, scales, dtype, status):
    _refused(status, lambda: lc.MxCacheWritePlan(x, codes, scales, dtype))
    if status not in ("DST_ALIASES",):
        _refused(status, lambda: lc.MxCacheReadPlan(codes, scales, x, dtype))


def test_read_refuses_rows_that_alias():
    _refused("DST_ALIASES", lambda: lc.MxCacheReadPlan("(8,2,64):(128,64,1)", "(8,2,2):(4,2,1)", "(4,2,64):(64,64,1)", "f32"))


# ---- plans of the attention ----
def _attention(T=8, heads=8, kv=2, D=64, slots=64, page=16, order="heads", q=None, o=None, dtype="bf16", **more):
    codes, scales = _pool(slots, kv, (D + 31) // 32 * 32, max(page, 1), order)
    args = dict(sequences=2, page=page, pages_per_sequence=3, max_queries=4, scale=0.125)
    args.update(more)
    o_dtype = args.pop("o_dtype", None)
    codes, scales = args.pop("codes", codes), args.pop("scales", scales)
    return lc.MxAttentionPlan(q or _dense(T, heads, D), codes, scales, o or _dense(T, heads, D), dtype, o_dtype, **args)


@pytest.mark.parametrize("change,status", [
    (dict(dtype="f32"), "UNSUPPORTED_DTYPE"), (dict(dtype="f16", o_dtype="bf16"), "UNSUPPORTED_DTYPE"), (dict(heads=7), "INVALID_ARG"), (dict(sequences=0), "INVALID_ARG"), (dict(page=0, order="heads", codes="(64,2,64):(128,64,1)", scales="(64,2,2):(4,2,1)"), "INVALID_ARG"),
    (dict(pages_per_sequence=0), "INVALID_ARG"), (dict(max_queries=0), "INVALID_ARG"), (dict(window=-1), "INVALID_ARG"), (dict(window=5, causal=False), "INVALID_ARG"),
    (dict(scale=float("nan")), "INVALID_ARG"), (dict(scale=float("inf")), "INVALID_ARG"), (dict(D=288), "INVALID_ARG"), (dict(page=12, codes="(64,2,64):(128,64,1)", scales="(64,2,2):(4,2,1)"), "INVALID_ARG"),
    (dict(codes="(64,2,32):(64,32,1)", scales="(64,2,1):(2,1,1)"), "SIZE_MISMATCH"), (dict(o=_dense(8, 8, 32)), "SIZE_MISMATCH"), (dict(o="(8,8,64):(64,64,1)"), "DST_ALIASES"),
    (dict(q="(8,512):(512,1)"), "INVALID_ARG"), (dict(codes="(64,2,64):(128,64,2)"), "BLOCK_LAYOUT"), (dict(codes="(64,2,64):(-128,64,1)"), "NEGATIVE_STRIDE"),
    (dict(sequences=65536), "TOO_LARGE"), (dict(pages_per_sequence=1 << 30), "TOO_LARGE"), (dict(page=16, pages_per_sequence=1 << 27), "TOO_LARGE"),
])
def test_attention_refused(change, status):
    _refused(status, lambda: _attention(**change))


def test_attention_calls_refused():
    """What a call is given is looked at before anything is launched (none of these addresses is touched)."""
    plan = _attention(sequences=2, pages_per_sequence=64, page=16, slots=4096)
    assert plan.workspace_bytes > 0
    at = 1 << 20
    good = dict(q_ptr=at, k_codes_ptr=at, k_scales_ptr=at, v_codes_ptr=at, v_scales_ptr=at, pages_ptr=at, lengths_ptr=at, starts_ptr=at, o_ptr=at, workspace_ptr=at,
                workspace_bytes=plan.workspace_bytes)
    for key in ("q_ptr", "k_codes_ptr", "k_scales_ptr", "v_codes_ptr", "v_scales_ptr", "lengths_ptr", "o_ptr"):
        _refused("INVALID_ARG", lambda: plan.execute(**dict(good, **{key: None})))
    for key, off in (("q_ptr", 1), ("o_ptr", 1), ("k_codes_ptr", 8), ("v_codes_ptr", 8), ("pages_ptr", 2), ("lengths_ptr", 2), ("starts_ptr", 1)):
        _refused("MISALIGNED", lambda: plan.execute(**dict(good, **{key: at + off})))
    _refused("MISALIGNED", lambda: plan.execute(**dict(good, lse_ptr=at + 2)))
    for change in (dict(workspace_ptr=None), dict(workspace_ptr=at + 8), dict(workspace_bytes=plan.workspace_bytes - 1)):
        _refused("WORKSPACE_TOO_SMALL", lambda: plan.execute(**dict(good, **change)))
    few = _attention(sequences=2, pages_per_sequence=3, page=16, slots=80)   # 96 slots without a table
    _refused("INVALID_ARG", lambda: few.execute(**dict(good, pages_ptr=None, workspace_bytes=1 << 30)))
    odd = _attention(T=9, sequences=2)
    _refused("INVALID_ARG", lambda: odd.execute(**dict(good, starts_ptr=None, workspace_bytes=1 << 30)))


def test_rope_and_cache_calls_refused():
    at = 1 << 20
    rope = lc.RopePlan(_dense(4, 2, 64), _dense(4, 2, 64), "f32", 64)
    for bad in ((None, at, at, at), (at, None, at, at), (at, at, None, at), (at, at, at, None)):
        _refused("INVALID_ARG", lambda: rope.execute(*bad))
    for bad in ((at + 2, at, at, at), (at, at + 2, at, at), (at, at, at + 2, at), (at, at, at, at + 2)):
        _refused("MISALIGNED", lambda: rope.execute(*bad))
    codes, scales = _pool(64, 2, 64, 16)
    write, read = lc.MxCacheWritePlan(_dense(4, 2, 64), codes, scales, "bf16"), lc.MxCacheReadPlan(codes, scales, _dense(4, 2, 64), "bf16")
    for call in (write.execute, read.execute):
        rows, first = (0, 1) if call == write.execute else (2, 0)
        for i in (0, 1, 2, 6):
            args = [at] * 7
            args[i] = None
            _refused("INVALID_ARG", lambda: call(*args))
        for some in ((3,), (4, 5), (3, 4), (5,)):   # half of the second tensor
            args = [at] * 7
            for i in some:
                args[i] = None
            _refused("INVALID_ARG", lambda: call(*args))
        for i, off in ((rows, 1), (rows + 3, 1), (first, 8), (first + 3, 8), (6, 2)):
            args = [at] * 7
            args[i] += off
            _refused("MISALIGNED", lambda: call(*args))
    # a plan of the other direction
    L = lc.lib()
    assert L.lc_mx_cache_read_plan_execute(write._h, at, at, at, None, None, None, at, None) == 1
    assert L.lc_mx_cache_write_plan_execute(read._h, at, at, at, None, None, None, at, None) == 1
    h = ctypes.c_void_p()
    assert L.lc_rope_plan_create(None, None, 0, 2, 0, 0, ctypes.byref(h)) == 1 and L.lc_rope_plan_execute(None, at, at, at, at, 1.0, None) == 1
    assert L.lc_mx_attention_plan_execute(None, *([at] * 11), 0, None) == 1 and L.lc_mx_attention_plan_workspace_bytes(None) == -1 and not h


def _pairs(T, B, page, each, most, lengths, starts, group, heads, causal, window, pages=None, pool_pages=1 << 30):
    n = 0
    for b, (first, queries, position, length) in enumerate(so.sequences(T, B, lengths, starts, page, each, most)):
        j = np.arange(length)
        there = np.ones(length, bool) if pages is None else (pages[b][j // page] >= 0) & (pages[b][j // page] < pool_pages)
        for i in range(queries):
            seen = there & (j <= position + i) if causal else there
            n += int((seen & (j > position + i - window)).sum() if window else seen.sum())
    return n * heads


WALKS = [  # B, queries, lengths, heads, kv, page, each, window, causal
    (1, [1], [1], 1, 1, 1, 1, 0, True), (1, [1], [997], 8, 2, 16, 64, 0, True), (3, [1, 1, 1], [0, 17, 640], 6, 2, 16, 40, 0, True), (2, [5, 3], [300, 2], 4, 1, 24, 13, 0, True),
    (2, [40, 7], [200, 100], 4, 2, 16, 13, 0, True), (2, [40, 7], [200, 100], 4, 2, 3, 67, 50, True), (1, [300], [300], 2, 1, 32, 10, 0, True), (1, [300], [1000], 2, 2, 64, 16, 100, True),
    (2, [9, 9], [500, 0], 8, 8, 16, 32, 0, False), (9, [1] * 9, [2000] * 9, 4, 4, 16, 125, 700, True), (1, [200], [90], 1, 1, 16, 6, 0, True), (5, [3, 0, 9, 1, 0], [10, 50, 3, 65, 9], 8, 2, 8, 9, 4, True),
    (4, [130, 1, 2, 64], [1000, 64, 65, 128], 8, 8, 128, 8, 0, True)]


@pytest.mark.parametrize("B,queries,lengths,heads,kv,page,each,window,causal", WALKS)
@pytest.mark.parametrize("order", ["heads", "tokens", None])
@pytest.mark.parametrize("table", [True, False])
def test_attention_walk(B, queries, lengths, heads, kv, page, each, window, causal, order, table):
    rng = np.random.default_rng(3)
    T, D = sum(queries) + 2, 64
    slots = (B * each + 2) * page
    codes, scales = _pool(slots, kv, 64, page if order else None, order or "heads")
    plan = lc.MxAttentionPlan(_dense(T, heads, D), codes, scales, _dense(T, heads, D), "bf16", sequences=B, page=page, pages_per_sequence=each, max_queries=max(queries), scale=1.0,
                              causal=causal, window=window)
    starts = np.cumsum([0] + queries).astype(np.int32)
    lengths = np.array(lengths, np.int32)
    pages = rng.permutation(B * each + 2)[:B * each].astype(np.int32).reshape(B, each) if table else None
    sizes = (T * heads * D * 2, lc.Layout(codes).cosize // 2, lc.Layout(scales).cosize, T * heads * D * 2)
    want = _pairs(T, B, page, each, max(queries), lengths, starts, heads // kv, heads, causal, window)
    assert plan.debug_walk_on_host(pages, lengths, starts, *sizes) == want, plan.describe()
    if table and order:   # a pool that ends with the last page that is named
        pages[pages == B * each + 1] = B * each
        assert plan.debug_walk_on_host(pages, lengths, starts, sizes[0], (B * each + 1) * page * kv * 32, sizes[2], sizes[3]) == want
    # numbers that do not fit are cut to what does
    most = max(queries)
    for some_lengths, some_starts in ((np.full(B, 2 ** 31 - 1, np.int32), starts), (np.full(B, -5, np.int32), starts), (lengths, starts - 1), (lengths, np.full(B + 1, 2 ** 31 - 1, np.int32)),
                                      (lengths, starts[::-1].copy()), (lengths, np.arange(B + 1, dtype=np.int32) * (T + 3)), (lengths, np.full(B + 1, -2 ** 31, np.int32))):
        want = _pairs(T, B, page, each, most, some_lengths, some_starts, heads // kv, heads, causal, window)
        assert plan.debug_walk_on_host(pages, some_lengths, some_starts, *sizes) == want
    if table:   # pages outside the pool
        pages[rng.random(pages.shape) < 0.3] = -1
        pages[rng.random(pages.shape) < 0.2] = B * each + 2
        want = _pairs(T, B, page, each, most, lengths, starts, heads // kv, heads, causal, window, pages, B * each + 2)
        assert plan.debug_walk_on_host(pages, lengths, starts, *sizes) == want


@pytest.mark.parametrize("codes,scales", [("(4194304,2,(32,8)):(64,32,(1,2147483648))", "(4194304,2,8):(16,8,1)"), ("(64,2,(32,8)):(64,32,(1,17179869184))", "(64,2,8):(16,8,1)"),
                                          ("(64,2,256):(512,256,1)", "(64,2,8):(2,1,4294967296)")])
@pytest.mark.parametrize("queries", [1, 40])
def test_attention_walk_of_blocks_far_apart(codes, scales, queries):
    """A head's blocks lie as far apart as the pool is long: their offsets pass 32 bits."""
    L, M = lc.Layout(codes), lc.Layout(scales)
    plan = lc.MxAttentionPlan(_dense(queries, 4, 256), codes, scales, _dense(queries, 4, 256), "bf16", sequences=1, page=16, pages_per_sequence=4, max_queries=queries, scale=1.0)
    assert " linear=0" in plan.describe()
    pages, lengths = np.array([[3, 0, 2, 1]], np.int32), np.array([60], np.int32)
    sizes = (queries * 4 * 256 * 2, L.cosize // 2, M.cosize, queries * 4 * 256 * 2)
    want = _pairs(queries, 1, 16, 4, queries, lengths, None, 2, 4, True, 0)
    assert plan.debug_walk_on_host(pages, lengths, None, *sizes) == want


@pytest.mark.parametrize("page,each,window,none", [(16, 1, 0, True), (16, 2, 0, True), (32, 1, 5, True), (1, 32, 0, True), (11, 3, 0, False), (16, 3, 0, False), (64, 1, 1, False), (16, 200, 1, False)])
def test_attention_of_one_unit_needs_no_workspace(page, each, window, none):
    """32 cached tokens at most are never shared out, so nothing is joined.  (A window's first tile may begin before it.)"""
    for queries in (1, 8):
        plan = _attention(T=2 * queries, slots=page * 2 * each, page=page, pages_per_sequence=each, max_queries=queries, window=window)
        assert (plan.workspace_bytes == 0) == none and " kernel=few" in plan.describe()
        sizes = [t.cosize for t in (plan.q_layout, plan.codes_layout, plan.scales_layout, plan.o_layout)]
        starts, pages = np.array([0, queries, 2 * queries], np.int32), np.arange(2 * each, dtype=np.int32).reshape(2, each)
        for lengths in ([page * each] * 2, [1, page * each], [0, 1], [max(1, page * each // 2)] * 2):
            want = _pairs(2 * queries, 2, page, each, queries, lengths, starts, 4, 8, True, window)
            assert plan.debug_walk_on_host(pages, np.array(lengths, np.int32), starts, 2 * sizes[0], sizes[1] // 2, sizes[2], 2 * sizes[3]) == want


@pytest.mark.parametrize("rows,kernel", [(1, "few"), (16, "few"), (17, "few"), (32, "few"), (33, "tile"), (4096, "tile")])
def test_attention_kernel_by_rows(rows, kernel):
    assert " kernel=" + kernel in _attention(T=2 * rows, heads=2, kv=2, max_queries=rows).describe()


def test_attention_that_is_linear():
    """Pages of whole runs of 16 tokens, one stride apart, everything else one stride: what the kernel of few rows has a short way for."""
    assert " linear=1" in _attention(page=16).describe() and " linear=1" in _attention(page=16, order="tokens").describe()
    assert " linear=1" in _attention(page=16, codes="(64,2,64):(128,64,1)", scales="(64,2,2):(4,2,1)").describe()
    for change in (dict(page=8), dict(page=24, slots=96), dict(D=72), dict(q="((4,2),8,64):((512,4096),64,1)"), dict(o="(8,8,64):(1024,128,2)"),
                   dict(codes="((8,8),2,64):((64,1024),512,1)", scales="(64,2,2):(4,2,1)"), dict(scales="((2,32),2,2):((4,10),2,1)")):
        if change.get("D") == 72:
            assert " linear=1" in _attention(**change).describe()   # (whole vectors of eight)
        else:
            assert " linear=0" in _attention(**change).describe(), change
    assert " linear=0" in _attention(D=76).describe()
