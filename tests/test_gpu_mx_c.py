"""How the products with microscaled 4-bit operands write C: past the caches or not, as the plan says, and under modes of several leaves (the definition in 64
bits and the bounds there are test_gpu_mx_gemm's); and how dequantisation writes large tensors."""
import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx
from test_gpu_mx_gemm import TORCH, _codes_and_scales, _elements, _rows, _run, _scales

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

CODES = {64: "kernel=stream tile=64x64", 12864: "kernel=stream tile=128x64", 128: "kernel=stream tile=128x128", 256: "kernel=ring tile=256x256",
         128128: "kernel=ring tile=128x128"}
MIXED = {12864: "kernel=stream tile=128x64", 128: "kernel=stream tile=128x128", 256: "kernel=wide tile=256x256", 256128: "kernel=wide tile=256x128",
         128128: "kernel=wide tile=128x128", 128064: "kernel=wide tile=128x64"}
FORCED = [("mxfp4", t) for t in CODES] + [("bf16", t) for t in MIXED]


def _operands(M, N, K, a_dtype):
    a, a_s = (_rows(M, K), _scales(M, K)) if a_dtype == "mxfp4" else (_rows(M, K), None)
    return a, a_s, _rows(N, K), _scales(N, K)


def _words(plan):
    return dict(word.split("=", 1) for word in plan.describe().split(" [")[0].split() if "=" in word)


def _taken(plan, a_dtype, tile):
    words = _words(plan)
    return "kernel=%s tile=%s" % (words["kernel"], words["tile"]) == (CODES if a_dtype == "mxfp4" else MIXED)[tile]


def _large(plan, strides):
    """A plan's product of operands whose every partial sum fp32 holds, C filled with fives before: the whole of its memory, equal.  strides: C's."""
    rng = np.random.default_rng(plan.c_layout.cosize)
    b_packed, b_scales, b = _codes_and_scales(rng, str(plan.b_layout), str(plan.b_scales_layout), "exact")
    if plan.a_dtype == "mxfp4":
        a_packed, a_scales, a = _codes_and_scales(rng, str(plan.a_layout), str(plan.a_scales_layout), "exact")
        a_t, as_t = torch.from_numpy(a_packed).cuda(), torch.from_numpy(a_scales).cuda()
    else:
        a_t, a = _elements(rng, str(plan.a_layout), plan.a_dtype, "exact")
        a_t, as_t = a_t.cuda(), None
    b_t, bs_t = torch.from_numpy(b_packed).cuda(), torch.from_numpy(b_scales).cuda()
    expect = torch.full((plan.c_layout.cosize + 40,), 5.0, dtype=TORCH[plan.c_dtype])
    c_t = expect.cuda()
    assert c_t.data_ptr() % 128 == 0
    plan.execute(a_t.data_ptr(), None if as_t is None else as_t.data_ptr(), b_t.data_ptr(), bs_t.data_ptr(), c_t.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for l in range(a.shape[2]):   # (products of float32 matrices: exact here)
        want = torch.from_numpy(a[:, :, l]).float() @ torch.from_numpy(b[:, :, l]).float().T
        expect[l * strides[2]:].as_strided(want.shape, strides[:2]).copy_(want + 5 if plan.accumulate else want)
    assert torch.equal(c_t.cpu(), expect)


@pytest.mark.parametrize("a_dtype,tile", FORCED)
@pytest.mark.parametrize("M,N,pitch,c_dtype,accumulate,past", [
    (2101, 4124, 4128, "f32", False, 1), (2101, 4124, 4132, "f32", False, 0), (2101, 8252, 8256, "bf16", False, 1), (2101, 8252, 8256, "f16", False, 1),
    (2101, 4124, 4128, "f32", True, 0)])
def test_large_c_past_the_caches(a_dtype, tile, M, N, pitch, c_dtype, accumulate, past, monkeypatch):
    """More than 32 MiB of C in vectors, both sides past the last whole tile: past the caches where rows begin on lines and nothing is added to."""
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    K = 128   # (four blocks: a dword of scales)
    plan = lc.MxGemmPlan(*_operands(M, N, K, a_dtype), "(%d,%d):(%d,1)" % (M, N, pitch), a_dtype, c_dtype, accumulate)
    assert _taken(plan, a_dtype, tile) and _words(plan)["c_vec"] == "1" and _words(plan)["past_caches"] == str(past), plan.describe()
    _large(plan, (pitch, 1, 0))


@pytest.mark.parametrize("a_dtype,tile", FORCED)
def test_large_batches_past_the_caches(a_dtype, tile, monkeypatch):
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    M, N, K, L, pitch = 1030, 2052, 128, 5, 2080
    a, a_s = ("(%d,%d,%d):(%d,1,%d)" % (M, K, L, K, M * K), "(%d,%d,%d):(%d,1,%d)" % (M, K // 32, L, K // 32, M * K // 32))
    b, b_s = ("(%d,%d,%d):(%d,1,0)" % (N, K, L, K), "(%d,%d,%d):(%d,1,0)" % (N, K // 32, L, K // 32))
    plan = lc.MxGemmPlan(a, a_s if a_dtype == "mxfp4" else None, b, b_s, "(%d,%d,%d):(%d,1,%d)" % (M, N, L, pitch, M * pitch), a_dtype, "f32", False)
    assert _taken(plan, a_dtype, tile) and _words(plan)["past_caches"] == "1", plan.describe()
    _large(plan, (pitch, 1, M * pitch))


# C's modes; which of the two the kernel's vectors would lie along (n: of both operands in codes and of 16-bit elements beside codes; m: of two in codes)
LEAVES = {
    "vectors along n": ("((9,31),(8,33)):((520,4688),(1,16))", True),
    "vectors along m": ("((8,33),(9,31)):((1,16),(520,4688))", False),
    "single elements along n": ("((9,31),(7,37)):((335,3017),(1,9))", False),
    "single elements along m": ("((7,37),(9,31)):((1,9),(335,3017))", False),
    "one leaf beside two": ("(260,(8,33)):(520,(1,16))", True),
    "two leaves beside one": ("((9,31),264):((268,2416),1)", True),
}


@pytest.mark.parametrize("a_dtype,tile", FORCED)
@pytest.mark.parametrize("case", LEAVES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_c_under_modes_of_several_leaves(case, a_dtype, tile, accumulate, monkeypatch):
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    c, vectors = LEAVES[case]
    vectors = vectors or (case == "vectors along m" and a_dtype == "mxfp4")
    M, N = mx.offsets(c).shape
    for kind, c_dtype in (("exact", "f32"), ("wide", "bf16")):
        args = _operands(M, N, 160, a_dtype) + (c, a_dtype, c_dtype, accumulate)
        plan = lc.MxGemmPlan(*args)
        assert _taken(plan, a_dtype, tile) and _words(plan)["c_vec"] == str(int(vectors))
        text = plan.describe().split(" C=[")[1]
        assert text.count(",") == c.count(",") - 2, text   # every leaf is still there
        _run(*args, kind, seed=tile)


@pytest.mark.parametrize("R,K,x", [(2101, 8203, "k"), (2101, 8300, "r"), (2104, 8300, "r")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("origin", [0, 1])
def test_large_16_bit_tensors_dequantised(R, K, x, dtype, origin):
    """More than 32 MiB, rows or columns that begin on lines where the tensor does: past the caches, and (origin 1) not."""
    text = {"k": "(%d,%d):(8256,1)" % (R, K), "r": "(%d,%d):(1,2112)" % (R, K)}[x]
    P = (K + 31) // 32 * 32
    torch_dtype = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    plan = lc.MxDequantizePlan(_rows(R, P), _rows(R, P // 32), text, dtype)
    assert "large_lines=1" in plan.describe() and ("access=k-vectors" if x == "k" else "access=row-vectors") in plan.describe()
    g = torch.Generator().manual_seed(K)
    codes = torch.randint(0, 256, (R, P // 2), dtype=torch.uint8, generator=g)
    scales = torch.randint(100, 150, (R, P // 32), dtype=torch.uint8, generator=g)
    size = lc.Layout(text).cosize + origin + 9
    dst = torch.full((size,), 77.0, dtype=torch_dtype, device="cuda")
    lc.mx_dequantize_tensor(codes.cuda(), _rows(R, P), scales.cuda(), _rows(R, P // 32), dst, text, dst_origin=origin)
    torch.cuda.synchronize()
    levels = torch.from_numpy(mx.LEVELS).float()   # (codes times powers of two: exact in fp32, then rounded once)
    want = (levels[torch.stack([codes & 15, codes >> 4], 2).long().reshape(R, P)] * torch.exp2(scales.float() - 127).repeat_interleave(32, 1)).to(torch_dtype)
    expect = torch.full((size,), 77.0, dtype=torch_dtype)
    expect[torch.from_numpy(mx.offsets(text)).reshape(R, K) + origin] = want[:, :K]
    assert torch.equal(dst.cpu(), expect)
