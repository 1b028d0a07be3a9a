"""Attention over a microscaled 4-bit cache on the GPU against the definition in 64 bits.

Error bound.  H: half a step of q's type (2^-8 bf16, 2^-11 f16), u = 2^-24.
Scores: products of q and k are exact (k in q's type is what the oracle takes), a sum of D terms in fp32 is off by (D + 1) 2u of the sum of magnitudes (as for
lc_mx_gemm), times the scale, whose own rounding and product add 3u of the score: with Z the row's largest scale sum |q k|, a score is off by e <= (2 D + 5) u Z.
Probabilities: an exponential of a difference of such scores is off by 2 e, by u of its exponent (at most 2 Z / ln 2 of them) and by 2 u for the instruction:
r = 2 e + 3 u Z + 2 u relative.  Rounding to 16 bits: H relative, and in f16 2^-25 absolute against the row's maximum of 1.
Probabilities below 2^-126 of the row's largest, fp32's smallest, are zeros: 2^-126 absolute against it.
Sums of n terms in fp32, rescaled once a tile of 32: (2 n + n / 32 * 3 + 64) u relative to sum p |v| above and to sum p below (64: the joins).
Together |error| <= sum p |v| / sum p * (H + 2 r + 2 (2 n + n / 10 + 64) u) 1.01, 2^-126 sum |v| / sum p more (in f16 2^-25), and o's own rounding.
lse: e + r + (2 n + n / 10 + 64) u + 4 u |lse|."""
import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import serve_oracle as so
from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U = 2.0 ** -24


def _pool_texts(slots, heads, width, page, order):
    def text(w):
        pages = slots // page
        return {"heads": "((%d,%d),%d,%d):((%d,%d),%d,1)" % (page, pages, heads, w, w, heads * page * w, page * w),
                "tokens": "((%d,%d),%d,%d):((%d,%d),%d,1)" % (page, pages, heads, w, heads * w, page * heads * w, w),
                "flat": "(%d,%d,%d):(%d,%d,1)" % (slots, heads, w, heads * w, w),
                "gaps": "((%d,%d),%d,%d):((%d,%d),%d,1)" % (page, pages, heads, w, w + 32, heads * page * (w + 32) + 64, page * (w + 32))}[order]
    scales = text(width // 32)
    if order == "heads":   # scales of a page's tokens together, block by block
        blocks, pages = width // 32, slots // page
        scales = "((%d,%d),%d,%d):((1,%d),%d,%d)" % (page, pages, heads, blocks, heads * page * blocks, page * blocks, page)
    return text(width), scales


def _rows(T, H, D, order):
    return {"thd": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, H * D, D), "htd": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, D, T * D), "row": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, (H + 2) * D + 1, D),
            "dht": "(%d,%d,%d):(1,%d,%d)" % (T, H, D, T, T * H)}[order]


def _fill(rng, codes_text, scales_text, slots, low=123, high=128):
    """A pool whose every byte is noise, scales of 255 among it, but for the slots in use."""
    codes = rng.integers(0, 256, lc.Layout(codes_text).cosize // 2 + 16, dtype=np.uint8)
    scales = rng.integers(250, 256, lc.Layout(scales_text).cosize + 16, dtype=np.uint8)
    s = mx.mode_offsets(scales_text)
    at = s[0][slots][:, None, None] + s[1][None, :, None] + s[2][None, None, :]
    scales[at] = rng.integers(low, high, at.shape)
    return codes, scales


class Case:
    """One call's data; `run` makes it and compares."""

    def __init__(self, queries, lengths, heads, kv, D, page=16, dtype="bf16", o_dtype=None, order="heads", q_order="thd", o_order="thd", causal=True, window=0, table=True, starts=True,
                 extra_rows=0, max_queries=None, each=None, scale=None, seed=0, low=123, high=128):
        print("case", queries, lengths, heads, kv, D, page, dtype, o_dtype, order, q_order, o_order, causal, window, table, starts, flush=True)
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.queries, self.lengths, self.heads, self.kv, self.D = len(queries), queries, np.array(lengths, np.int32), heads, kv, D
        self.page, self.dtype, self.o_dtype, self.causal, self.window = page, dtype, o_dtype or dtype, causal, window
        self.each = each or max(1, -(-max(lengths) // page))
        self.max_queries = max_queries or max(max(queries), 1)
        self.T = sum(queries) + extra_rows
        self.scale = D ** -0.5 if scale is None else scale
        pages_n = self.B * self.each + (2 if table else 0)
        self.slots = pages_n * page
        width = (D + 31) // 32 * 32
        self.codes_text, self.scales_text = _pool_texts(self.slots, kv, width, page, order)
        self.q_text, self.o_text = _rows(self.T, heads, D, q_order), _rows(self.T, heads, D, o_order)
        self.pages = rng.permutation(pages_n)[:self.B * self.each].astype(np.int32).reshape(self.B, self.each) if table else None
        used = []
        for b in range(self.B):
            j = np.arange(min(max(lengths[b], 0), self.each * page))
            used.append((self.pages[b][j // page] if table else b * self.each + j // page) * page + j % page)
        self.used = used
        inside = np.concatenate(used).astype(np.int64)
        self.k, self.v = (list(_fill(rng, self.codes_text, self.scales_text, inside, low, high)) for _ in range(2))
        q = rng.standard_normal(lc.Layout(self.q_text).cosize).astype(np.float32) * 1.5
        self.q = torch.from_numpy(q).to(TORCH[dtype])
        self.starts = np.cumsum([0] + list(queries)).astype(np.int32) if starts else None

    def plan(self):
        return lc.MxAttentionPlan(self.q_text, self.codes_text, self.scales_text, self.o_text, self.dtype, self.o_dtype, sequences=self.B, page=self.page, pages_per_sequence=self.each,
                                  max_queries=self.max_queries, scale=self.scale, causal=self.causal, window=self.window)

    def on_gpu(self, workspace=None):
        dev = torch.device("cuda:0")
        g = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev)   # noqa: E731
        o = torch.full((lc.Layout(self.o_text).cosize + 8,), 77.0, dtype=TORCH[self.o_dtype], device=dev)
        lse = torch.full((self.T, self.heads), 77.0, device=dev)
        plan = self.plan()
        print(plan.describe(), flush=True)
        if workspace is None:   # what is in it does not matter
            workspace = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device=dev)
        lc.mx_attention_tensor(plan, self.q.to(dev), g(self.k[0]), g(self.k[1]), g(self.v[0]), g(self.v[1]), g(self.lengths), o, g(self.pages), g(self.starts), lse, workspace)
        torch.cuda.synchronize()
        return o, lse

    def want(self):
        # keys and values in q's type, as the call rounds them
        t = TORCH[self.dtype]
        pools = []
        for codes, scales in (self.k, self.v):
            pool = so.Pool(codes, self.codes_text, scales, self.scales_text, self.D)
            pools.append(type("Rounded", (), {"slots": pool.slots, "__call__": lambda _, s, pool=pool: torch.from_numpy(pool(s)).to(t).double().numpy()})())
        off = mx.offsets(self.q_text)
        o, lse = np.full((self.T, self.heads, self.D), 77.0), np.full((self.T, self.heads), 77.0)
        bound = so.attention(self.q.double().numpy()[off], *pools, self.heads // self.kv, self.B, self.page, self.each, self.max_queries, self.lengths, self.starts, self.pages,
                             float(np.float32(self.scale)), self.causal, self.window, o, lse)
        return o, lse, bound

    def run(self):
        o_t, lse_t = self.on_gpu()
        o, lse, (mass, loose, Z, n) = self.want()
        off = mx.offsets(self.o_text)
        got = o_t.double().cpu().numpy()
        H, D = HALF_STEP[self.dtype], self.D
        e = (2 * D + 5) * U * Z
        r = 2 * e + 3 * U * Z + 2 * U
        sums = (2 * n + n / 10 + 64) * U
        tol = mass * (H + 2 * r + 2 * sums)[..., None] * 1.01 + (2.0 ** -25 if self.dtype == "f16" else 2.0 ** -126) * loose
        tol = tol + HALF_STEP[self.o_dtype] * (np.abs(o) + tol) + (2.0 ** -25 if self.o_dtype == "f16" else 0.0)
        same = (got[off] == o) | (np.isnan(got[off]) & np.isnan(o))
        with np.errstate(invalid="ignore"):
            wrong = ~(same | (np.abs(got[off] - o) <= tol))
        assert not wrong.any(), (int(wrong.sum()), np.argwhere(wrong)[:5].tolist(), got[off][wrong][:5], o[wrong][:5], tol[wrong][:5])
        rest = np.ones(len(got), bool)
        rest[off.reshape(-1)] = False
        assert (got[rest] == 77.0).all()
        got = lse_t.double().cpu().numpy()
        same = (got == lse) | (np.isnan(got) & np.isnan(lse))
        with np.errstate(invalid="ignore"):
            assert (same | (np.abs(got - lse) <= e + r + sums + 4 * U * np.abs(lse))).all()
        return o_t, lse_t


# ---- few rows ----
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300, 1000])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_one_token(length, dtype):
    Case([1], [length], 8, 2, 128, dtype=dtype, each=70).run()


@pytest.mark.parametrize("D", [1, 31, 32, 33, 64, 80, 96, 128, 192, 200, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("queries", [1, 5])
def test_few_rows_of_every_width(D, dtype, queries):
    Case([queries] * 3, [70, queries, 333], 8, 2, D, dtype=dtype, seed=D).run()


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (7, 1), (16, 1), (17, 1), (32, 1), (12, 4), (64, 2)])
@pytest.mark.parametrize("page,order", [(16, "heads"), (64, "tokens"), (8, "heads"), (24, "tokens"), (1, "flat"), (3, "gaps"), (32, "gaps"), (128, "flat")])
def test_heads_and_pages(heads, kv, page, order):
    Case([1, 1], [200, 77], heads, kv, 64, page=page, order=order, seed=page).run()


@pytest.mark.parametrize("page,each,order", [(16, 20, "heads"), (40, 7, "flat"), (7, 41, "flat"), (1, 300, "flat"), (300, 1, "flat"), (304, 1, "heads")])
@pytest.mark.parametrize("queries", [1, 40])
def test_without_a_table(page, each, order, queries):
    Case([queries] * 2, [min(280, page * each), 55], 4, 2, 64, page=page, each=each, order=order, table=False).run()


# ---- many rows ----
@pytest.mark.parametrize("D", [1, 32, 33, 64, 80, 128, 192, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_rows_of_every_width(D, dtype):
    Case([130, 3, 40], [300, 64, 41], 4, 2, D, dtype=dtype, seed=D).run()


@pytest.mark.parametrize("queries,lengths", [([33], [33]), ([128], [128]), ([129], [1000]), ([64], [64]), ([65], [1]), ([200], [150]), ([100, 0, 1, 50], [100, 30, 1, 0]), ([40, 300, 7], [500, 301, 2000])])
@pytest.mark.parametrize("heads,kv", [(2, 2), (5, 1), (8, 2)])
def test_ragged_prompts(queries, lengths, heads, kv):
    """Sequences with fewer cached tokens than queries have rows that see nothing."""
    Case(queries, lengths, heads, kv, 64, seed=len(queries)).run()


@pytest.mark.parametrize("page,order", [(16, "tokens"), (1, "flat"), (3, "gaps"), (24, "heads"), (100, "tokens")])
def test_prompts_on_pages(page, order):
    Case([70, 20], [300, 90], 4, 2, 128, page=page, order=order).run()


# ---- masks ----
@pytest.mark.parametrize("window", [1, 2, 15, 64, 100, 5000])
@pytest.mark.parametrize("queries", [1, 4, 90])
def test_windows(window, queries):
    Case([queries] * 2, [400, 123], 4, 2, 64, window=window).run()


@pytest.mark.parametrize("queries", [1, 7, 60])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_token_for_every_query(queries, dtype):
    """Cross attention: queries of one length, cached states of another."""
    Case([queries, queries // 2, queries], [100, 333, 0], 4, 4, 80, causal=False, dtype=dtype).run()


@pytest.mark.parametrize("queries", [2, 4, 50, 140])
@pytest.mark.parametrize("window", [0, 37])
@pytest.mark.parametrize("dtype,byte", [("bf16", 255), ("bf16", 254), ("f16", 255), ("f16", 150)])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(queries, window, dtype, byte):
    """Scales of NaN, and such as make infinities of some codes, among the values of tokens that some queries see and others do not."""
    c = Case([queries, queries], [200, queries], 4, 2, 64, dtype=dtype, window=window, order="tokens")
    s = mx.mode_offsets(c.scales_text)
    for b in range(2):
        n = len(c.used[b])
        for j in {n - 1, n - 2, n - max(2, queries // 2), max(0, n - queries), max(0, n - queries - window + 1 if window else 0), max(0, n - 5)}:
            slot = c.used[b][min(max(j, 0), n - 1)]
            c.v[1][s[0][slot] + s[1][j % 2] + s[2][(j // 2) % 2]] = byte
    c.run()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_values_that_are_not_finite_in_the_first_tile(D, dtype):
    """Workgroups by the hundred, every wavefront of which finds a block of NaN in the first tile that it expands, each in a token of its own."""
    B, n, heads, blocks = 24, 130, 8, D // 32
    c = Case([n] * B, [64] * B, heads, heads, D, dtype=dtype, causal=False)
    s = mx.mode_offsets(c.scales_text)
    nan = np.zeros((B, heads, blocks), bool)
    for b in range(B):
        for h in range(heads):
            for block in range(blocks):
                if (b + h + block) % 3:
                    c.v[1][s[0][c.used[b][(7 * b + 13 * h + 8 * block) % 64]] + s[1][h] + s[2][block]] = 255
                    nan[b, h, block] = True
    o, _ = c.on_gpu()
    got = torch.isnan(o).cpu().numpy()[mx.offsets(c.o_text)].reshape(B, n, heads, blocks, 32)
    assert (got == nan[:, None, :, :, None]).all()


@pytest.mark.parametrize("queries", [1, 3, 60])
@pytest.mark.parametrize("what", ["k", "q"])
def test_nan_and_infinities_of_keys_and_queries(queries, what):
    c = Case([queries, queries], [100, queries + 3], 4, 2, 64)
    if what == "k":
        s = mx.mode_offsets(c.scales_text)
        c.k[1][s[0][c.used[0][-1]] + s[1][1] + s[2][0]] = 255   # seen by the last query only
    else:
        off = mx.offsets(c.q_text)
        c.q[off[0, 0, 3]] = float("nan")
        c.q[off[queries, 3, 5]] = float("inf")
    c.run()


@pytest.mark.parametrize("queries", [1, 5, 40])
@pytest.mark.parametrize("D", [33, 64, 96, 160, 192, 256])
@pytest.mark.parametrize("dtype,byte", [("bf16", 254), ("f16", 150)])
@pytest.mark.parametrize("block", [0, -1])
def test_a_score_of_minus_infinity_is_nothing(queries, D, dtype, byte, block):
    """A token whose key makes every score minus infinity leaves the bits as they are without it, also where the kernel's width is more than a head's blocks."""
    c = Case([queries, queries], [40, 39], 4, 2, D, dtype=dtype, causal=False)
    c.q = c.q.abs() + 0.5
    slot = c.used[0][39]
    codes, scales = mx.mode_offsets(c.codes_text), mx.mode_offsets(c.scales_text)
    d = block % len(scales[2])
    for head in range(2):
        at = (codes[0][slot] + codes[1][head] + codes[2][32 * d]) // 2
        c.k[0][at:at + 16] = 0xFF   # (all -6, those past D zeros: they have to be finite)
        left = D - 32 * d
        if left < 32:
            c.k[0][at + left // 2:at + 16] = 0
            if left % 2:
                c.k[0][at + left // 2] = 0x0F
        c.k[1][scales[0][slot] + scales[1][head] + scales[2][d]] = byte
    got = c.on_gpu()
    c.lengths[0] = 39
    want = c.on_gpu()
    assert not torch.isnan(want[0][:c.T * 4 * D]).any()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("queries", [1, 5, 40])
@pytest.mark.parametrize("dtype,byte", [("bf16", 254), ("f16", 150)])
@pytest.mark.parametrize("forced", [None, "64"])
def test_every_score_minus_infinity_gives_zeros_whatever_the_values(queries, dtype, byte, forced, monkeypatch):
    if forced:
        monkeypatch.setenv("LC_TUNE_MX_SHARES", forced)
        monkeypatch.setenv("LC_TUNE_MX_PART", forced)
    for D, page, order in ((64, 16, "heads"), (128, 3, "gaps"), (256, 16, "tokens")):
        c = Case([queries, queries], [200, 70], 4, 2, D, page=page, order=order, dtype=dtype, causal=False)
        off = mx.offsets(c.q_text)
        c.q = c.q.abs() + 0.5
        c.q[off[queries - 1, 3].reshape(-1)] *= -1   # one row's scores are infinite the other way: NaN
        codes, scales = mx.mode_offsets(c.codes_text), mx.mode_offsets(c.scales_text)
        c.k[0][(codes[0][c.used[0]][:, None, None] + codes[1][None, :, None] + codes[2][None, None, ::2]) // 2] = 0xFF
        c.k[1][scales[0][c.used[0]][:, None, None] + scales[1][None, :, None] + scales[2][None, None, :]] = byte
        for j, scale in ((0, 255), (64, byte), (199, 255)):
            c.v[1][scales[0][c.used[0][j]] + scales[1] + scales[2][j % 2]] = scale
        o, lse = c.on_gpu()
        o = o.double().cpu().numpy()[mx.offsets(c.o_text)]
        zero = np.ones((2 * queries, 4), bool)
        zero[queries - 1, 3] = False
        zero[queries:] = False
        assert (o[zero] == 0.0).all() and (lse.cpu().numpy()[zero] == -np.inf).all()
        assert np.isnan(o[queries - 1, 3]).all() and np.isfinite(o[queries:]).all()


@pytest.mark.parametrize("queries", [1, 4, 70])
@pytest.mark.parametrize("page", [4, 16])
def test_pages_outside_the_pool_are_seen_by_nobody(queries, page):
    c = Case([queries, queries, queries], [300, 200, 90], 4, 2, 64, page=page)
    c.pages[0, ::3] = -1
    c.pages[1, 1::2] = 2 ** 31 - 1
    c.pages[1, 0] = c.slots // page
    c.pages[2, :] = -2 ** 31
    c.run()


def test_equal_scores_give_the_mean():
    """q of zeros: every probability is 1, the sum of 2^n values of few bits is exact, and so is the result."""
    for queries in (1, 40):
        c = Case([queries], [256], 4, 2, 128, causal=False, dtype="bf16", o_dtype="f32", low=127, high=128)
        c.q.zero_()
        o_t, lse_t = c.on_gpu()
        o, lse, _ = c.want()
        assert (o_t.double().cpu().numpy()[mx.offsets(c.o_text)] == o).all()
        assert (np.abs(lse_t.double().cpu().numpy() - lse) <= 4 * U * np.abs(lse)).all()


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-42])
def test_a_scale_of_nothing_gives_the_mean(scale):
    """Scores of up to 1e35, none further from 0 than 2^-24 once they are scaled: as in the test above; what is masked stays so."""
    for queries in (1, 40):
        c = Case([queries], [256 + queries - 1], 4, 2, 64, causal=True, window=256, dtype="bf16", o_dtype="f32", low=127, high=128, scale=scale)
        c.q = c.q.clamp(-2, 2) * 2.0 ** 50 / (1 if abs(scale) < 1e-44 else 2 ** 20)
        c.k[1][mx.offsets(c.scales_text)[c.used[0]]] = 127 + 55
        o_t, lse_t = c.on_gpu()
        v = so.Pool(c.v[0], c.codes_text, c.v[1], c.scales_text, 64)(c.used[0])
        want = np.stack([np.repeat(v[i:i + 256].mean(0), 2, 0) for i in range(queries)])
        assert (o_t.double().cpu().numpy()[mx.offsets(c.o_text)] == want).all()
        assert (np.abs(lse_t.double().cpu().numpy() - np.log(256.0)) <= 4 * U * np.log(256.0)).all()


def test_one_cached_token_is_the_answer():
    for queries in (1, 40):
        c = Case([1] if queries == 1 else [1, queries], [1] if queries == 1 else [1, 1], 4, 2, 96, causal=False, low=120, high=134)
        o_t, _ = c.on_gpu()
        o, _, _ = c.want()
        assert (o_t.double().cpu().numpy()[mx.offsets(c.o_text)] == o).all()


def test_scores_of_every_size():
    """Maxima that grow from tile to tile, and scores so far apart that most probabilities are zero."""
    for queries in (1, 40):
        for scale in (0.0, 1e-3, 3.0, -0.5):
            Case([queries], [700], 4, 2, 64, scale=scale, low=126, high=131).run()


def _levels(rng, n):
    """Codes of n tokens, all of a token's elements alike: the largest and the smallest are shared by 2^k tokens each, in tiles of their own where there are several."""
    if n <= 2:
        yield np.full(n, rng.integers(9, 16))
        yield np.full(n, rng.integers(1, 8))
        return
    level = rng.choice([0, 1, 2, 3, 4, 5, 6, 9, 10, 11, 12, 13, 14], n)
    level[[70, n - 1]] = 7
    level[[3, 64, 130, 131]] = 15
    yield level
    level = rng.choice([9, 10, 11, 12, 13, 14], n)   # scores that reach 0 late, from far below (or begin at their largest)
    level[:64] = 15
    level[100:104] = 0
    yield level


@pytest.mark.parametrize("D,page,order", [(64, 16, "heads"), (128, 16, "tokens"), (256, 16, "heads"), (128, 3, "gaps")])
@pytest.mark.parametrize("queries", [1, 6, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_of_large_magnitude(D, page, order, queries, dtype, monkeypatch):
    """Scores of 1e3 to 3e38 of either sign, so far apart that only those that equal the largest count: the answer is the mean of 2^k values, exactly where the largest score's
    exponent of two lies beyond 2^10.  Up to there the exponent that is left of it is the rounding error of a product of that size, u times the exponent, 2^-14 u / u = 2^-15 at most: every
    probability that counts is 2^that, less than a quarter of a 16-bit step (2^-11) from 1, and is rounded to 1, and their sum holds it: the answer is off by ln 2 times it, u |score|,
    relative, and by 16 u of the mean magnitude for the sums, the reciprocal and the product with it.  (At 1e3 neighbouring scores are 24 apart, and the others' probabilities, e^-24 each, are allowed for twice.)
    lse: the scale's product with log2(e) (2 u), its product with a constant (2 u) and with the score (u), and one sum: 6 u."""
    values = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])
    rng = np.random.default_rng(D + queries)
    for size in (1e3, 1e4, 1e6, 1e9, 1e12, 1e30, 3e38):
        for n, forced in ((1, None), (2, None), (200, None), (200, "64")):
            if forced:
                monkeypatch.setenv("LC_TUNE_MX_SHARES", forced)
                monkeypatch.setenv("LC_TUNE_MX_PART", forced)
            for byte in (127, 217) if dtype == "bf16" else (127,):   # large by the scale, or by the keys
                for level in _levels(rng, n):
                    scale = float(np.float32(size * rng.uniform(0.5, 1) / (10.5 * D) * 2.0 ** (127 - byte)))
                    c = Case([queries], [n], 8, 2, D, page=page, order=order, dtype=dtype, o_dtype="f32", causal=False, scale=scale, low=125, high=129)
                    codes, scales = mx.mode_offsets(c.codes_text), mx.mode_offsets(c.scales_text)
                    at = (codes[0][c.used[0]][:, None, None] + codes[1][None, :, None] + codes[2][None, None, ::2]) // 2
                    c.k[0][at] = (level | level << 4)[:, None, None]
                    c.k[1][scales[0][c.used[0]][:, None, None] + scales[1][None, :, None] + scales[2][None, None, :]] = byte
                    a = rng.choice([1, 1.25, 1.5, 1.75, -1, -1.25, -1.5, -1.75], (queries, 8))
                    off = mx.offsets(c.q_text)
                    q = np.zeros(off.max() + 1, np.float32)
                    q[off] = a[:, :, None]
                    c.q = torch.from_numpy(q).to(TORCH[dtype])
                    score = scale * 2.0 ** (byte - 127) * D * a[:, :, None] * values[level]   # (queries, heads, tokens)
                    top = score == score.max(-1, keepdims=True)
                    v = so.Pool(c.v[0], c.codes_text, c.v[1], c.scales_text, D)(c.used[0])    # (tokens, key heads, D)
                    want = np.einsum("ihj,jhd->ihd", top / top.sum(-1, keepdims=True), np.repeat(v, 4, 1))
                    o, lse = c.on_gpu()
                    exponent = np.abs(score.max(-1))[..., None] / np.log(2.0)
                    mass = np.einsum("ihj,jhd->ihd", top / top.sum(-1, keepdims=True), np.repeat(np.abs(v), 4, 1))
                    tol = np.where(exponent <= 1024 * (1 + 4 * U), U * exponent * np.log(2.0) * np.abs(want) + 16 * U * mass, 0.0)
                    others = np.where(top, 0.0, np.exp(score - score.max(-1, keepdims=True)))
                    tol = tol + 2 * np.einsum("ihj,jhd->ihd", others, np.repeat(np.abs(v), 4, 1) + np.abs(v).max())
                    assert (np.abs(o.double().cpu().numpy()[mx.offsets(c.o_text)] - want) <= tol).all(), (size, n, forced, byte)
                    want = score.max(-1) + np.log(top.sum(-1))
                    assert (np.abs(lse.double().cpu().numpy() - want) <= 6.1 * U * np.abs(want) + others.sum(-1)).all(), (size, n, forced, byte)
            monkeypatch.delenv("LC_TUNE_MX_SHARES", raising=False)
            monkeypatch.delenv("LC_TUNE_MX_PART", raising=False)


# ---- layouts, types, rows that are nobody's ----
@pytest.mark.parametrize("q_order,o_order", [("htd", "thd"), ("row", "htd"), ("dht", "thd"), ("thd", "dht"), ("thd", "row")])
@pytest.mark.parametrize("queries", [1, 5, 40])
@pytest.mark.parametrize("D", [64, 72])
def test_layouts_of_queries(q_order, o_order, queries, D):
    Case([queries, queries], [50, 90], 4, 2, D, q_order=q_order, o_order=o_order, o_dtype="f32").run()


@pytest.mark.parametrize("queries", [1, 40])
def test_rows_that_are_nobodys_stay(queries):
    """Rows behind the last sequence, and queries past max_queries."""
    Case([queries, 2, queries], [100, 40, 300], 4, 2, 64, extra_rows=5).run()
    Case([queries + 2, 1], [100, 40], 4, 2, 64, max_queries=queries).run()
    Case([3] * 4, [10, 20, 30, 40], 4, 2, 64, starts=False).run()


def test_numbers_that_do_not_fit_are_cut():
    c = Case([4, 4], [60, 90], 4, 2, 64)
    c.lengths[:] = [2 ** 31 - 1, -7]
    full = np.arange(c.each * c.page)   # the first sequence now has every place of its row of the table
    slots = (c.pages[0][full // c.page] * c.page + full % c.page).astype(np.int64)
    for side in (c.k, c.v):
        s = mx.mode_offsets(c.scales_text)
        side[1][s[0][slots][:, None, None] + s[1][None, :, None] + s[2][None, None, :]] = 125
    c.starts = np.array([-3, 5, 2 ** 31 - 1], np.int32)
    c.run()


@pytest.mark.parametrize("queries", [1, 40])
def test_the_workspace_is_the_calls_alone(queries):
    """The same bits whatever it held, and for every run."""
    c = Case([queries] * 2, [5000, 4000], 4, 2, 64)
    need = c.plan().workspace_bytes
    assert need > 0
    first = c.on_gpu(torch.zeros(need, dtype=torch.uint8, device="cuda"))
    for fill in (255, 127):
        again = c.on_gpu(torch.full((need,), fill, dtype=torch.uint8, device="cuda"))
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("queries", [1, 8])
@pytest.mark.parametrize("page,each,D", [(16, 2, 64), (1, 32, 128), (16, 1, 256)])
def test_short_caches_need_no_workspace(queries, page, each, D):
    n = page * each
    c = Case([queries, queries, 0, queries], [n, 1, 3, n - 1], 8, 2, D, page=page, each=each, order="flat")
    assert c.plan().workspace_bytes == 0
    c.run()


def test_long_sequences_in_parts():
    Case([1, 1], [20000, 9999], 8, 2, 128, page=64).run()
    Case([40], [6000], 4, 1, 64, page=64, dtype="f16").run()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("queries,forced", [(1, "8"), (1, "64"), (1, "4096"), (9, "64"), (20, "64"), (20, "4096"), (70, "64"), (70, "1024")])
def test_parts_of_any_number(queries, forced, D, monkeypatch):
    """Few rows: wavefronts that a call's tokens are dealt out to; many rows: tokens of a part.  From one part of a row to one for each 32 or 64 tokens."""
    monkeypatch.setenv("LC_TUNE_MX_SHARES", forced)
    monkeypatch.setenv("LC_TUNE_MX_PART", forced)
    Case([queries, queries], [5000, 33 + queries], 2, 2, D, page=32).run()


@pytest.mark.parametrize("B", [64, 65, 128, 200])
@pytest.mark.parametrize("most", [1, 5, 60])
def test_more_sequences_than_a_wavefront_has_lanes(B, most):
    rng = np.random.default_rng(B)
    queries = rng.integers(0, most + 1, B).tolist()
    queries[B // 2] = most
    lengths = rng.integers(0, 150, B).tolist()
    lengths[B - 1] = 700
    Case(queries, lengths, 6, 3 if most > 5 else 2, 64, page=16, max_queries=most).run()


@pytest.mark.parametrize("queries", [1, 40])
def test_starts_that_decrease_end(queries):
    """Such a call's rows may hold anything, and nothing else is written."""
    B = 70
    c = Case([queries] * B, [100] * B, 2, 1, 64, extra_rows=5)
    c.starts = np.array([0, c.T - 5] * (B // 2) + [0], np.int32)
    c.max_queries = queries
    o, _ = c.on_gpu()
    off = mx.offsets(c.o_text)
    rest = np.ones(len(o), bool)
    rest[off[:c.T - 5].reshape(-1)] = False
    assert (o.float().cpu().numpy()[rest] == 77.0).all()


def test_offsets_past_32_bits():
    """A pool whose pages lie 2^28 + 1024 bytes apart."""
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(3)
    page, each, D = 16, 12, 64
    step = (1 << 29) + 2048
    codes_text, scales_text = "((16,%d),1,64):((64,%d),64,1)" % (each, step), "((16,%d),1,2):((2,32),2,1)" % each
    codes = torch.zeros((step * (each - 1) + 1024) // 2, dtype=torch.uint8, device=dev)
    small = rng.integers(0, 256, (each, page * 32), dtype=np.uint8)
    for i in range(each):
        codes[i * step // 2:i * step // 2 + page * 32] = torch.from_numpy(small[i]).to(dev)
    scales = rng.integers(124, 128, each * page * 2, dtype=np.uint8)
    pages = rng.permutation(each).astype(np.int32)
    for queries in (1, 40):
        q = torch.from_numpy(rng.standard_normal((queries, 2, D)).astype(np.float32)).bfloat16().to(dev)
        o = torch.empty(queries, 2, D, device=dev)
        plan = lc.MxAttentionPlan("(%d,2,64):(128,64,1)" % queries, codes_text, scales_text, "(%d,2,64):(128,64,1)" % queries, "bf16", "f32", sequences=1, page=page, pages_per_sequence=each,
                                  max_queries=queries, scale=0.125)
        g = lambda a: torch.from_numpy(a).to(dev)   # noqa: E731
        lc.mx_attention_tensor(plan, q, codes, g(scales), codes, g(scales), g(np.array([page * each], np.int32)), o, g(pages[None].copy()))
        near = "((16,%d),1,64):((64,1024),64,1)" % each
        plan2 = lc.MxAttentionPlan("(%d,2,64):(128,64,1)" % queries, near, scales_text, "(%d,2,64):(128,64,1)" % queries, "bf16", "f32", sequences=1, page=page, pages_per_sequence=each,
                                   max_queries=queries, scale=0.125)
        o2 = torch.empty_like(o)
        lc.mx_attention_tensor(plan2, q, g(small.reshape(-1)), g(scales), g(small.reshape(-1)), g(scales), g(np.array([page * each], np.int32)), o2, g(pages[None].copy()))
        assert torch.equal(o, o2)


@pytest.mark.parametrize("queries", [1, 5, 40])
def test_blocks_past_32_bits(queries):
    """A pool of 8 GiB whose heads have their eight blocks 2^30 bytes apart, scales 2^26 bytes: the bits of the same tokens in a small one."""
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(5)
    slots, kv, D, page, each = 1 << 22, 16, 256, 16, 5
    far, far_scales = "(%d,%d,(32,8)):(%d,32,(1,%d))" % (slots, kv, 32 * kv, slots * kv * 32), "(%d,%d,8):(%d,1,%d)" % (slots, kv, kv, slots * kv)
    near, near_scales = "(%d,%d,%d):(%d,%d,1)" % (page * each, kv, D, kv * D, D), "(%d,%d,8):(%d,8,1)" % (page * each, kv, 8 * kv)
    codes = rng.integers(0, 256, (page * each, kv, 8, 16), dtype=np.uint8)
    scales = rng.integers(122, 126, (page * each, kv, 8), dtype=np.uint8)
    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)   # noqa: E731
    q = g(rng.standard_normal((queries, 2 * kv, D)).astype(np.float32)).bfloat16()
    lengths, table = g(np.array([page * each - 3], np.int32)), rng.permutation(slots // page)[:each]
    big, big_scales = torch.zeros(8, slots, kv, 16, dtype=torch.uint8, device=dev), torch.full((8, slots, kv), 255, dtype=torch.uint8, device=dev)
    for i, at in enumerate(table):   # page i of the small pool is page `at` of the large one
        big[:, page * at:page * (at + 1)] = g(codes[page * i:page * (i + 1)].transpose(2, 0, 1, 3))
        big_scales[:, page * at:page * (at + 1)] = g(scales[page * i:page * (i + 1)].transpose(2, 0, 1))
    outs = []
    for c_text, s_text, c, s, pages in ((far, far_scales, big.view(-1), big_scales.view(-1), table), (near, near_scales, g(codes).view(-1), g(scales).view(-1), np.arange(each))):
        text = "(%d,%d,%d):(%d,%d,1)" % (queries, 2 * kv, D, 2 * kv * D, D)
        plan = lc.MxAttentionPlan(text, c_text, s_text, text, "bf16", "f32", sequences=1, page=page, pages_per_sequence=each, max_queries=queries, scale=0.0625)
        print(plan.describe(), flush=True)
        o = torch.full((queries, 2 * kv, D), 77.0, device=dev)
        lc.mx_attention_tensor(plan, q, c, s, c, s, lengths, o, g(pages[None].astype(np.int32)))
        outs.append(o)
    assert not (torch.isnan(outs[1]) | (outs[1] == 77.0)).any() and torch.equal(*outs)


def test_two_calls_at_once_and_a_captured_one():
    """A graph follows the arrays that it was captured with; an eager call on another stream with a workspace of its own does not disturb it."""
    dev = torch.device("cuda:0")
    c = Case([1, 1], [3000, 2000], 8, 2, 128)
    plan = c.plan()
    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)   # noqa: E731
    q, lengths, pages, starts = c.q.to(dev), g(c.lengths), g(c.pages), g(c.starts)
    pool = [g(a) for a in (*c.k, *c.v)]
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    spaces = [torch.empty(plan.workspace_bytes, dtype=torch.uint8, device=dev) for _ in range(2)]
    outs = [torch.empty(lc.Layout(c.o_text).cosize, dtype=torch.bfloat16, device=dev) for _ in range(2)]

    def call(i, stream):
        plan.execute(q.data_ptr(), *[p.data_ptr() for p in pool], pages.data_ptr(), lengths.data_ptr(), starts.data_ptr(), outs[i].data_ptr(), None, spaces[i].data_ptr(),
                     spaces[i].numel(), stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call(0, side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(0, torch.cuda.current_stream().cuda_stream)
    for n in ((3000, 2000), (1, 1999), (0, 64), (2500, 3000)):
        c.lengths[:] = n
        lengths.copy_(g(c.lengths))
        q.copy_(q * 0.9)
        torch.cuda.synchronize()
        for o in outs:
            o.fill_(77.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            call(1, other.cuda_stream)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and not torch.isnan(outs[0][:64]).any() if max(n) <= 3000 and n != (2500, 3000) else torch.equal(outs[0].isnan(), outs[1].isnan())


# ---- together, as they are used ----
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("pairs", ["half", "neighbours"])
def test_a_model_layer_step_by_step(dtype, pairs):
    """Prompts, then single tokens: queries and keys turned, keys and values written, attention over what is cached; every step against the same in 64 bits from the
    turned and quantised values."""
    rng = np.random.default_rng(12)
    dev = torch.device("cuda:0")
    B, heads, kv, D, page, each = 2, 4, 2, 64, 16, 8
    pages_n = B * each + 1
    codes_text, scales_text = _pool_texts(pages_n * page, kv, D, page, "tokens")
    pool = [torch.from_numpy(rng.integers(0, 256, lc.Layout(t).cosize // n, dtype=np.uint8)).to(dev) for t, n in ((codes_text, 2), (scales_text, 1)) * 2]
    pages = rng.permutation(pages_n)[:B * each].reshape(B, each).astype(np.int32)
    f = torch.tensor(lc.lc_rope_frequencies(D, 10000.0, "parts", 4.0, 64), device=dev)
    cached = np.zeros(B, np.int64)
    for counts in ([40, 23], [1, 1], [1, 1], [5, 3], [1, 1]):
        T = sum(counts)
        qkv = torch.from_numpy(rng.standard_normal((T, heads + 2 * kv, D)).astype(np.float32)).to(TORCH[dtype]).to(dev)
        positions = np.concatenate([np.arange(n) + cached[b] for b, n in enumerate(counts)]).astype(np.int32)
        which = np.repeat(np.arange(B), counts)
        slots = (pages[which, positions // page] * page + positions % page).astype(np.int32)
        cached += counts
        g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)   # noqa: E731
        row = (heads + 2 * kv) * D
        turned = "(%d,%d,%d):(%d,%d,1)" % (T, heads + kv, D, row, D)   # in place, inside the rows
        lc.rope_tensor(qkv, turned, g(positions), f, qkv, turned, D, pairs)
        k, v = qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        rows = "(%d,%d,%d):(%d,%d,1)" % (T, kv, D, row, D)
        lc.mx_cache_write_tensor(k, v, rows, pool[0], pool[2], codes_text, pool[1], pool[3], scales_text, g(slots))
        back = [torch.empty(T, kv, D, dtype=TORCH[dtype], device=dev) for _ in range(2)]
        lc.mx_cache_read_tensor(pool[0], pool[2], codes_text, pool[1], pool[3], scales_text, *back, "(%d,%d,%d):(%d,%d,1)" % (T, kv, D, kv * D, D), g(slots))
        for rows_in, rows_out in ((k, back[0]), (v, back[1])):
            want = mx.dequantize(*mx.quantize(rows_in.double().cpu().numpy().reshape(T * kv, D), D, "floor")).reshape(T, kv, D)
            assert (rows_out.double().cpu().numpy() == want).all()
        c = Case(counts, cached.tolist(), heads, kv, D, page=page, each=each, dtype=dtype, order="tokens")
        c.pages, c.codes_text, c.scales_text, c.slots = pages, codes_text, scales_text, pages_n * page
        c.q = qkv[:, :heads].contiguous().view(-1).cpu()
        c.k, c.v = [t.cpu().numpy() for t in pool[:2]], [t.cpu().numpy() for t in pool[2:]]
        c.run()
