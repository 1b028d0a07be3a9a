"""GEMM with microscaled 4-bit operands on the GPU against the definition in 64 bits.

Where every partial sum is a multiple of a power of two that fp32 holds ("exact" values) the result has to equal the 64-bit one, rounded
once to C's type.  Otherwise ("wide" values) the products are exact (codes: 4 significant bits; codes times 16-bit elements: 13 at most),
and a sum of K terms and C's old value in fp32, in whatever order, is off by at most (K + 1) 2^-23 of the sum of magnitudes (each of the
K additions rounds by 2^-24 of a partial sum; the factor of two covers sums inside an instruction that drop bits below the largest term
instead of rounding); the rounding to C's type adds half a step, 2^-8 (bf16) or 2^-11 (f16) of the value, and f16's smallest step 2^-25."""
import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _offsets(text):
    o = mx.offsets(text)
    return o if o.ndim == 3 else o[:, :, None]


def _codes_and_scales(rng, codes_text, scales_text, kind, blocked=1):
    """Random codes and scales under their layouts: packed bytes, scale bytes, values (rows, k, batch) in 64 bits."""
    off, s_off = _offsets(codes_text), _offsets(scales_text)
    codes = rng.integers(0, 16, off.shape)
    low, high = {"exact": (126, 129), "wide": (110, 135), "f16": (113, 127)}[kind]
    scales = rng.integers(low, high, s_off.shape)
    packed = rng.integers(0, 256, (int(off.max()) // 32 + 1) * 16, dtype=np.uint8)
    s_bytes = rng.integers(0, 256, int(s_off.max()) + 1, dtype=np.uint8)
    for l in range(off.shape[2]):
        for parity in (0, 1):
            at = off[:, :, l] % 2 == parity
            byte = off[:, :, l][at] // 2
            packed[byte] = (packed[byte] & (0xF0 if parity == 0 else 0x0F)) | (codes[:, :, l][at].astype(np.uint8) << (4 * parity))
    s_bytes[s_off] = scales
    # what lies there now (a layout with strides of 0 shares elements)
    codes = (packed[off // 2] >> (4 * (off % 2)).astype(np.uint8)) & 15
    scales = s_bytes[s_off].astype(np.int64)
    return packed, s_bytes, mx.LEVELS[codes] * np.repeat(np.where(scales == 255, np.nan, np.ldexp(1.0, scales - 127)), 32, axis=blocked)


def _elements(rng, text, dtype, kind):
    off = _offsets(text)
    v = rng.integers(-4, 5, int(off.max()) + 1).astype(np.float32) if kind == "exact" else \
        (rng.standard_normal(int(off.max()) + 1) * np.exp2(rng.integers(-6, 1 if kind == "f16" else 6, int(off.max()) + 1))).astype(np.float32)
    t = torch.from_numpy(v).to(TORCH[dtype])
    return t, t.double().numpy()[off]


def _run(a_text, a_s_text, b_text, b_s_text, c_text, a_dtype, c_dtype, accumulate, kind, blocked=1, seed=0):
    rng = np.random.default_rng(seed)
    dev = torch.device("cuda:0")
    codes = a_dtype == "mxfp4"
    wide = "f16" if kind == "wide" and "f16" in (a_dtype, c_dtype) else kind   # (short of what overflows there)
    b_packed, b_scales, b = _codes_and_scales(rng, b_text, b_s_text, wide, blocked)
    b_t, bs_t = torch.from_numpy(b_packed).to(dev), torch.from_numpy(b_scales).to(dev)
    if codes:
        a_packed, a_scales, a = _codes_and_scales(rng, a_text, a_s_text, wide)
        a_t, as_t = torch.from_numpy(a_packed).to(dev), torch.from_numpy(a_scales).to(dev)
    else:
        a_t, a = _elements(rng, a_text, a_dtype, wide)
        a_t, as_t = a_t.to(dev), None
    c_off = _offsets(c_text)
    M, N, L = c_off.shape
    c0 = torch.from_numpy(rng.integers(-8, 9, int(c_off.max()) + 33).astype(np.float32)).to(TORCH[c_dtype])
    c_t = c0.to(dev)
    plan = lc.MxGemmPlan(a_text, a_s_text, b_text, b_s_text, c_text, a_dtype, c_dtype, accumulate)
    print("case", plan.describe(), kind, flush=True)
    plan.execute(a_t.data_ptr(), as_t.data_ptr() if codes else None, b_t.data_ptr(), bs_t.data_ptr(), c_t.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    K = a.shape[1]
    # B blocked along k may be padded beyond K, B blocked along its rows beyond N
    b = b[:N, :K]
    with np.errstate(invalid="ignore"):
        want = np.einsum("mkl,nkl->mnl", a, b)
        size = np.einsum("mkl,nkl->mnl", np.abs(a), np.abs(b))
    got_all, c0 = c_t.double().cpu().numpy(), c0.double().numpy()
    old = c0[c_off]
    if accumulate:
        want, size = want + old, size + np.abs(old)
    got = got_all[c_off]
    if kind == "exact":
        assert (torch.from_numpy(got) == torch.from_numpy(want).to(TORCH[c_dtype]).double()).all()
    else:
        bound = (K + 1) * 2.0 ** -23 * size * (1 + HALF_STEP[c_dtype]) + HALF_STEP[c_dtype] * np.abs(want) + (2.0 ** -25 if c_dtype == "f16" else 0)
        with np.errstate(invalid="ignore"):
            assert (np.abs(got - want) <= bound).all(), np.nanmax(np.abs(got - want) / bound)
    rest = np.ones(len(c0), bool)
    rest[c_off.reshape(-1)] = False
    assert (got_all[rest] == c0[rest]).all()   # nothing else was written


def _rows(r, p):
    return "(%d,%d):(%d,1)" % (r, p, p)


def _scales(r, p, tiles=False, blocked=1):
    text = str(lc.lc_mx_scale_layout(r, p // 32)) if tiles else _rows(r, p // 32)
    if blocked == 1:
        return text
    shape, stride = text.split(":")
    flip = lambda t: "(" + t[t.index(",") + 1:-1] + "," + t[1:t.index(",")] + ")"   # noqa: E731
    return flip(shape) + ":" + flip(stride)


# M, N, K (whole blocks)
CODES = [(1, 1, 32), (1, 40, 64), (3, 17, 96), (16, 16, 128), (17, 33, 160), (64, 64, 256), (65, 130, 288), (128, 128, 512), (129, 200, 544),
         (200, 64, 1024), (300, 260, 2080), (31, 1001, 4128)]


@pytest.mark.parametrize("M,N,K", CODES)
@pytest.mark.parametrize("tile", [0, 16, 3216, 32, 64, 12864, 128, 256, 128128])
def test_codes_by_codes(M, N, K, tile, monkeypatch):
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    for i, (kind, c_dtype, accumulate, tiles, c_text) in enumerate((
            ("exact", "f32", True, False, _rows(M, N)), ("exact", "bf16", False, True, "(%d,%d):(1,%d)" % (M, N, M)), ("wide", "f32", False, True, _rows(M, N)),
            ("wide", "f16", True, False, "(%d,%d):(%d,3)" % (M, N, 3 * N)))):
        P = (K + 255) // 256 * 256 if tiles else K
        _run(_rows(M, P), _scales(M, P, tiles), _rows(N, P), _scales(N, P, tiles), c_text, "mxfp4", c_dtype, accumulate, kind, seed=i)


@pytest.mark.parametrize("a,a_s,b,b_s,c", [
    # rows apart, scales apart and transposed
    ("(70,320):(384,1)", "(70,10):(1,70)", "(90,320):(352,1)", "(90,10):(11,1)", "(70,90):(100,1)"),
    # blocks of all rows together: the k mode has leaves of one block
    ("(70,(32,10)):(32,(1,2240))", "(70,10):(1,70)", "(90,(32,10)):(32,(1,2880))", "(90,10):(10,1)", "(70,90):(1,80)"),
    # leaves of 8 blocks
    ("(70,(256,3)):(256,(1,17920))", "(70,(4,6)):(4,(1,280))", "(90,(256,3)):(768,(1,256))", "(90,(8,3)):(8,(1,720))", "(70,90):(90,1)"),
    # rows in two leaves on all tensors, C as well
    ("((7,10),320):((320,3200),1)", "((7,10),10):((10,100),1)", "((9,10),320):((3200,320),1)", "(90,10):(10,1)", "((7,10),(9,10)):((1,7),(70,630))"),
    # one row of A shared by all of M; scales shared by all blocks
    ("(70,320):(0,1)", "(70,10):(0,1)", "(90,320):(320,1)", "(90,10):(1,0)", "(70,90):(90,1)"),
    # batches: A's matrices apart, B's shared, scales shared
    ("(33,320,3):(320,1,16000)", "(33,10,3):(10,1,330)", "(50,320,3):(320,1,0)", "(50,10,3):(10,1,0)", "(33,50,3):(50,1,1700)"),
])
@pytest.mark.parametrize("tile", [0, 32, 64, 128, 256, 128128])
def test_layouts_of_codes(a, a_s, b, b_s, c, tile, monkeypatch):
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    _run(a, a_s, b, b_s, c, "mxfp4", "f32", True, "exact", seed=3)
    _run(a, a_s, b, b_s, c, "mxfp4", "bf16", False, "wide", seed=4)


MIXED = [(1, 1, 1), (1, 40, 64), (1, 1000, 1024), (2, 17, 100), (5, 33, 33), (16, 130, 256), (17, 64, 520), (40, 300, 1000), (64, 256, 2048), (129, 200, 77),
         (200, 129, 640), (300, 520, 136)]


@pytest.mark.parametrize("M,N,K", MIXED)
@pytest.mark.parametrize("a_dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tile", [0, 16, 3216, 32, 12864, 128, 256, 256128, 128128, 128064])
def test_weights(M, N, K, a_dtype, tile, monkeypatch):
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    for i, (kind, c_dtype, accumulate, tiles, c_text) in enumerate((
            ("exact", "f32", True, False, _rows(M, N)), ("exact", a_dtype, False, True, "(%d,%d):(1,%d)" % (M, N, M)), ("wide", a_dtype, False, True, _rows(M, N)))):
        P = (K + 255) // 256 * 256 if tiles else (K + 31) // 32 * 32
        _run(_rows(M, K), None, _rows(N, P), _scales(N, P, tiles), c_text, a_dtype, c_dtype, accumulate, kind, seed=i)


@pytest.mark.parametrize("M,K,N", MIXED)
@pytest.mark.parametrize("a_dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tile", [0, 12864, 128, 256, 256128, 128128, 128064])
def test_transposed_weights(M, N, K, a_dtype, tile, monkeypatch):
    """The gradient of the forward product's A: the sum runs over N, B is blocked along the rows of the result."""
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    for i, (kind, c_dtype, accumulate, tiles) in enumerate((("exact", "f32", True, False), ("exact", a_dtype, False, True), ("wide", a_dtype, False, True))):
        P = (K + 255) // 256 * 256 if tiles else (K + 31) // 32 * 32
        _run(_rows(M, N), None, "(%d,%d):(1,%d)" % (P, N, P), _scales(N, P, tiles, blocked=0), _rows(M, K), a_dtype, c_dtype, accumulate, kind, blocked=0, seed=i)


@pytest.mark.parametrize("a,b,b_s,c,blocked", [
    ("(70,300):(1,70)", "(90,320):(352,1)", "(90,10):(1,90)", "(70,90):(100,1)", 1),              # A contiguous along its rows
    ("(70,300):(2,150)", "(90,320):(320,1)", "(90,10):(10,1)", "(70,90):(1,70)", 1),              # not contiguous
    ("(70,300):(301,1)", "(90,(32,10)):(32,(1,2880))", "(90,10):(10,1)", "(70,90):(90,1)", 1),    # rows at any alignment, codes by blocks
    ("(70,(20,16)):(20,(1,1400))", "(90,320):(320,1)", "(90,10):(10,1)", "(70,90):(90,1)", 1),    # a k mode of two leaves
    ("((7,10),304):((304,3040),1)", "((9,10),320):((3200,320),1)", "(90,10):(10,1)", "((7,10),(9,10)):((1,7),(70,630))", 1),
    ("(70,304):(0,1)", "(90,320):(0,1)", "(90,10):(0,1)", "(70,90):(90,1)", 1),                   # shared rows
    ("(33,304,3):(304,1,16000)", "(50,320,3):(320,1,0)", "(50,10,3):(10,1,0)", "(33,50,3):(50,1,1700)", 1),
    ("(33,301,3):(301,1,16001)", "(50,320,3):(320,1,16000)", "(50,10,3):(10,1,512)", "(33,50,3):(50,1,1700)", 1),
    ("(70,90):(90,1)", "(320,90):(1,320)", "(10,90):(1,10)", "(70,300):(300,1)", 0),
    ("(70,90):(1,70)", "((32,10),90):((1,2880),32)", "(10,90):(90,1)", "(70,300):(1,70)", 0),
    ("(33,50,3):(56,1,2000)", "(320,50,3):(1,320,0)", "(10,50,3):(1,10,0)", "(33,304,3):(304,1,10032)", 0),
])
@pytest.mark.parametrize("tile", [0, 32, 128, 256, 256128, 128128, 128064])
@pytest.mark.parametrize("a_dtype", ["bf16", "f16"])
def test_layouts_of_mixed_operands(a, b, b_s, c, blocked, tile, a_dtype, monkeypatch):
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    _run(a, None, b, b_s, c, a_dtype, "f32", True, "exact", blocked=blocked, seed=5)
    _run(a, None, b, b_s, c, a_dtype, a_dtype, False, "wide", blocked=blocked, seed=6)


@pytest.mark.parametrize("a_dtype,blocked", [("mxfp4", 1), ("bf16", 1), ("f16", 1), ("bf16", 0), ("f16", 0)])
@pytest.mark.parametrize("tile", [0, 32, 128, 256, 256128, 128128, 128064])
def test_nan_scales_reach_what_they_enter_and_nothing_else(a_dtype, tile, blocked, monkeypatch):
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    dev = torch.device("cuda:0")
    M, N, K = 40, 96, 320   # blocked along k: K codes of N rows; along the rows: N codes of K rows
    stored = (N, K) if blocked else (K, N)
    codes = torch.full((stored[0] * stored[1] // 2,), 0x22, dtype=torch.uint8, device=dev)   # ones
    scales = torch.full((stored[0], stored[1] // 32), 127, dtype=torch.uint8, device=dev)
    scales[5, 1] = 255
    b_text = _rows(*stored) if blocked else "(%d,%d):(1,%d)" % (N, K, N)
    s_text = _scales(*stored) if blocked else "(%d,%d):(1,%d)" % (N // 32, K, N // 32)
    if a_dtype == "mxfp4":
        a, a_s = torch.full((M * K // 2,), 0x22, dtype=torch.uint8, device=dev), torch.full((M * K // 32,), 127, dtype=torch.uint8, device=dev)
        a_s_text = _scales(M, K)
    else:
        a, a_s, a_s_text = torch.ones(M * K, dtype=TORCH[a_dtype], device=dev), None, None
    c = torch.zeros(M, N, device=dev)
    lc.mx_gemm_tensor(a, _rows(M, K), a_s, a_s_text, codes, b_text, scales, s_text, c, _rows(M, N), accumulate=False)
    torch.cuda.synchronize()
    want = torch.full((M, N), float(K))
    want[:, slice(5, 6) if blocked else slice(32, 64)] = float("nan")
    assert torch.equal(torch.isnan(c.cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(c.cpu()), torch.nan_to_num(want))


@pytest.mark.parametrize("a_dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tile", [0, 32, 128, 256, 256128, 128128, 128064])
def test_blocks_past_k_are_not_used(a_dtype, tile, monkeypatch):
    """K = 72 of 256: what lies in the blocks past it, NaN scales among it, stays out of the sum."""
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    dev = torch.device("cuda:0")
    M, N, K, P = 20, 70, 72, 256
    codes = torch.full((N, P // 2), 0x22, dtype=torch.uint8, device=dev)
    scales = torch.full((N, P // 32), 255, dtype=torch.uint8, device=dev)
    scales[:, :3] = 127
    c = torch.zeros(M, N, device=dev)
    lc.mx_gemm_tensor(torch.ones(M * K, dtype=TORCH[a_dtype], device=dev), _rows(M, K), None, None, codes, _rows(N, P), scales, _rows(N, P // 32), c, _rows(M, N))
    torch.cuda.synchronize()
    assert (c.cpu() == K).all()


@pytest.mark.parametrize("a_dtype,low,high", [("bf16", 1, 254), ("f16", 100, 141)])
def test_weights_take_the_other_operands_type(a_dtype, low, high):
    """One term per sum: the product with 1 is B's element rounded to A's type, at every scale (bf16: short of what overflows)."""
    dev = torch.device("cuda:0")
    scales = np.arange(low, high).astype(np.uint8)
    N = len(scales)
    for c in range(16):
        codes = np.zeros((N, 16), np.uint8)
        codes[:, 0] = c
        want = torch.from_numpy(mx.LEVELS[c] * np.ldexp(1.0, scales.astype(np.int64) - 127)).to(TORCH[a_dtype]).float()
        keep = torch.isfinite(want) & ((want.abs() >= 2.0 ** -126) | (want == 0))
        out = torch.zeros(1, N, device=dev)
        a = torch.zeros(32, dtype=TORCH[a_dtype], device=dev)
        a[0] = 1
        lc.mx_gemm_tensor(a, _rows(1, 32), None, None, torch.from_numpy(codes).reshape(-1).to(dev), _rows(N, 32), torch.from_numpy(scales).to(dev), _rows(N, 1), out,
                          _rows(1, N), accumulate=False)
        assert torch.equal(out.cpu()[0][keep], want[keep]), c


def test_graph_and_second_stream():
    dev = torch.device("cuda:0")
    M, N, K = 40, 320, 512
    x_text, c_text, s = _rows(M, K), _rows(M, N), torch.cuda.Stream()
    q = lc.MxQuantizePlan(x_text, _rows(M, K), _scales(M, K, True), "bf16")
    plans = [lc.MxGemmPlan(_rows(M, K), _scales(M, K, True), _rows(N, K), _scales(N, K, True), c_text, accumulate=False),
             lc.MxGemmPlan(x_text, None, _rows(N, K), _scales(N, K, True), c_text, a_dtype="bf16", accumulate=True)]
    rng = np.random.default_rng(1)
    b_packed, b_scales, b = _codes_and_scales(rng, _rows(N, K), _scales(N, K, True), "exact")
    b_t, bs_t = torch.from_numpy(b_packed).to(dev), torch.from_numpy(b_scales).to(dev)
    x, c = torch.zeros(M, K, dtype=torch.bfloat16, device=dev), torch.zeros(M, N, device=dev)
    a, a_s = torch.zeros(M * K // 2, dtype=torch.uint8, device=dev), torch.zeros(M * K // 32, dtype=torch.uint8, device=dev)

    def launch(stream):
        q.execute(x.data_ptr(), a.data_ptr(), a_s.data_ptr(), stream)
        plans[0].execute(a.data_ptr(), a_s.data_ptr(), b_t.data_ptr(), bs_t.data_ptr(), c.data_ptr(), stream)
        plans[1].execute(x.data_ptr(), None, b_t.data_ptr(), bs_t.data_ptr(), c.data_ptr(), stream)

    torch.cuda.synchronize()
    launch(s.cuda_stream)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        launch(torch.cuda.current_stream().cuda_stream)
    for rep in range(4):
        v = torch.from_numpy(np.random.default_rng(rep).integers(-4, 5, (M, K)).astype(np.float32))   # whole numbers to 4: held exactly
        x.copy_(v)
        c.fill_(1e6)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (c.cpu().double().numpy() == 2 * (v.double().numpy() @ b[:, :, 0].T)).all(), rep


def test_a_layer_forward_and_backward():
    """The operators together as a training step uses them, against the products of the same rounded operands in 64 bits; and the rounded
    layer's gradients against differences: the loss is linear in x and in w (the operands are what is rounded, not the sums), so a
    difference of two losses is the gradient times the step."""
    dev = torch.device("cuda:0")
    T, I, O = 96, 160, 224   # tokens, inputs, outputs
    rng = np.random.default_rng(2)
    x, w, dy = (torch.from_numpy(rng.standard_normal(s)).to(torch.bfloat16) for s in ((T, I), (O, I), (T, O)))

    def quantized(v, transposed):
        rows, k = (v.shape[1], v.shape[0]) if transposed else v.shape
        codes, scales = torch.zeros(rows * k // 2, dtype=torch.uint8, device=dev), torch.zeros(rows * k // 32, dtype=torch.uint8, device=dev)
        src = "(%d,%d):(1,%d)" % (rows, k, rows) if transposed else _rows(rows, k)
        lc.mx_quantize_tensor(v.to(dev), src, codes, _rows(rows, k), scales, _rows(rows, k // 32), "cover")
        exact = (v.t() if transposed else v).double().numpy()
        return (codes, _rows(rows, k), scales, _rows(rows, k // 32)), mx.dequantize(*mx.quantize(exact, k, "cover"))

    def product(a, b, shape):
        c = torch.zeros(shape, device=dev)
        lc.mx_gemm_tensor(a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3], c, _rows(*shape), accumulate=False)
        return c.cpu().double().numpy()

    def near(got, a, b):
        want, size = a @ b.T, np.abs(a) @ np.abs(b).T
        assert (np.abs(got - want) <= (a.shape[1] + 1) * 2.0 ** -23 * size).all()

    (xq, xv), (wq, wv), (gq, gv) = quantized(x, False), quantized(w, False), quantized(dy, False)
    (xtq, xtv), (wtq, wtv), (gtq, gtv) = quantized(x, True), quantized(w, True), quantized(dy, True)
    y, dx, dw = product(xq, wq, (T, O)), product(gq, wtq, (T, I)), product(gtq, xtq, (O, I))
    near(y, xv, wv)
    near(dx, gv, wtv)
    near(dw, gtv, xtv)
    # frozen weights: forward and the input's gradient with x and dy in 16 bits
    y16, dx16 = torch.zeros(T, O, device=dev), torch.zeros(T, I, device=dev)
    lc.mx_gemm_tensor(x.to(dev), _rows(T, I), None, None, wq[0], wq[1], wq[2], wq[3], y16, _rows(T, O), accumulate=False)
    lc.mx_gemm_tensor(dy.to(dev), _rows(T, O), None, None, wq[0], "(%d,%d):(1,%d)" % (I, O, I), wq[2], "(%d,%d):(1,%d)" % (I // 32, O, I // 32), dx16, _rows(T, I),
                      accumulate=False)
    near(y16.cpu().double().numpy(), x.double().numpy(), wv)
    near(dx16.cpu().double().numpy(), dy.double().numpy(), wv.T)
    # differences: the loss sum(dy * y) of the frozen layer, x moved by a power of two along single inputs (held exactly in bf16 next to 0)
    for t, i in ((0, 0), (5, 33), (95, 159)):
        losses = []
        for step in (2.0, -2.0):
            moved = torch.zeros(T, I, dtype=torch.bfloat16)
            moved[t, i] = step
            out = torch.zeros(T, O, device=dev)
            lc.mx_gemm_tensor(moved.to(dev), _rows(T, I), None, None, wq[0], wq[1], wq[2], wq[3], out, _rows(T, O), accumulate=False)
            losses.append((out.cpu().double() * dy.double()).sum().item())
        slope = (losses[0] - losses[1]) / 4.0
        assert abs(slope - dx16[t, i].item()) <= (O + 1) * 2.0 ** -23 * float(np.abs(dy.double().numpy()[t]) @ np.abs(wv[:, i]))


def test_offsets_past_32_bits():
    """Codes that end 3 GiB behind their first, rows of C 2 GiB apart."""
    dev = torch.device("cuda:0")
    N, K, M = 4, 64, 4
    step = 1 << 31   # codes: 1 GiB from row to row
    codes = torch.zeros((N - 1) * step // 2 + K // 2, dtype=torch.uint8, device=dev)
    for r in range(N):
        codes[r * step // 2:r * step // 2 + K // 2] = 0x22 * (1 + (r == 2))   # ones; the third row twos
    scales = torch.full((N * 2,), 127, dtype=torch.uint8, device=dev)
    c_step = 1 << 29
    c = torch.full(((M - 1) * c_step + N,), 5.0, device=dev)
    a = torch.ones(M * K, dtype=torch.bfloat16, device=dev)
    for a_dtype in ("bf16", "mxfp4"):
        if a_dtype == "bf16":
            args = (a, _rows(M, K), None, None)
        else:
            args = (torch.full((M * K // 2,), 0x22, dtype=torch.uint8, device=dev), _rows(M, K), torch.full((M * 2,), 127, dtype=torch.uint8, device=dev), _rows(M, 2))
        lc.mx_gemm_tensor(*args, codes, "(%d,%d):(%d,1)" % (N, K, step), scales, _rows(N, 2), c, "(%d,%d):(%d,1)" % (M, N, c_step), accumulate=False)
        torch.cuda.synchronize()
        for m in range(M):
            assert c[m * c_step:m * c_step + N].tolist() == [K, K, 2.0 * K, K]
        assert c[N].item() == 5.0 and c[c_step - 1].item() == 5.0


def test_helper_refusals():
    dev = torch.device("cuda:0")
    a, b = torch.zeros(64, dtype=torch.bfloat16, device=dev), torch.zeros(32, dtype=torch.uint8, device=dev)
    s, c = torch.zeros(2, dtype=torch.uint8, device=dev), torch.zeros(4, device=dev)
    args = dict(a=a, a_layout="(2,32):(32,1)", a_scales=None, a_scales_layout=None, b=b, b_layout="(2,32):(32,1)", b_scales=s, b_scales_layout="(2,1):(1,1)", c=c,
                c_layout="(2,2):(2,1)")
    lc.mx_gemm_tensor(**args)
    for key, value, error in (("a", a[:63], ValueError), ("a", a.float(), ValueError), ("b", b[:31], ValueError), ("b", b.to(torch.int32), ValueError),
                              ("b_scales", s[:1], ValueError), ("c", c[:3], ValueError), ("c", c.double(), ValueError), ("b", b.cpu(), RuntimeError),
                              ("c_layout", "(2,2):(1,1)", lc.LayoutCopyError)):
        with pytest.raises(error):
            lc.mx_gemm_tensor(**dict(args, **{key: value}))


@pytest.mark.parametrize("a_dtype", ["mxfp4", "bf16"])
@pytest.mark.parametrize("M", [1, 20])
@pytest.mark.parametrize("s_text", ["(20,2304):(2304,1)", "(20,2304):(1,20)"])
def test_long_k(a_dtype, M, s_text):
    """More scales than the direct kernel keeps in LDS (2304 blocks), and just as many as it does (1020, 2044)."""
    for blocks in (2304, 2044, 1020):
        K, N = 32 * blocks, 20
        s = s_text.replace("2304", str(blocks))
        a, a_s = (_rows(M, K), _scales(M, K)) if a_dtype == "mxfp4" else (_rows(M, K), None)
        _run(a, a_s, _rows(N, K), s, _rows(M, N), a_dtype, "f32", False, "wide", seed=blocks)


@pytest.mark.parametrize("M,N,K,pitch", [(3, 40, 65, 70), (20, 70, 72, 80), (33, 100, 264, 272), (130, 140, 520, 528), (16, 128, 301, 301), (200, 129, 640, 648)])
@pytest.mark.parametrize("order", ["k", "r"])
@pytest.mark.parametrize("blocked", [1, 0])
@pytest.mark.parametrize("tile", [0, 32, 12864, 128, 256, 256128, 128128, 128064])
def test_nan_around_the_operands_stays_out(M, N, K, pitch, order, blocked, tile, monkeypatch):
    """NaN before, behind and between the rows of A, scales of 255 between and behind B's, an origin of A off any vector for odd M."""
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(K)
    pitch = pitch if order == "k" else M + 8
    a_text = "(%d,%d):(%d,1)" % (M, K, pitch) if order == "k" else "(%d,%d):(1,%d)" % (M, K, pitch)
    a = rng.integers(-4, 5, (M, K)).astype(np.float32)
    before = 8 + M % 2
    flat = np.full(before + lc.Layout(a_text).cosize + 600, np.nan, np.float32)
    flat[before + mx.offsets(a_text)] = a
    P = (K + 31) // 32 * 32 if blocked else (N + 31) // 32 * 32
    rows, k = (N, P) if blocked else (K, P)
    s_pitch = P // 32 + 3
    codes = rng.integers(0, 16, (rows, k))
    scales = np.full((rows + 9) * s_pitch + 1, 255, np.uint8)
    used = 1 + np.arange(rows)[:, None] * s_pitch + np.arange(P // 32)   # at an odd address
    scales[used] = rng.integers(126, 129, used.shape)
    packed = np.zeros((rows, k // 2), np.uint8)
    packed |= (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
    values = mx.LEVELS[codes] * np.repeat(np.ldexp(1.0, scales[used].astype(np.int64) - 127), 32, axis=1)
    b_text, s_text = ("(%d,%d):(%d,1)" % (N, P, P), "(%d,%d):(%d,1)" % (N, P // 32, s_pitch)) if blocked else \
                     ("(%d,%d):(1,%d)" % (P, K, P), "(%d,%d):(1,%d)" % (P // 32, K, s_pitch))
    want = a.astype(np.float64) @ (values[:, :K].T if blocked else values[:, :N])
    a_t = torch.from_numpy(flat).to(torch.bfloat16).to(dev)
    b_t, s_t, c = torch.from_numpy(packed).to(dev), torch.from_numpy(scales).to(dev), torch.full((M, N), np.nan, device=dev)
    lc.lc_mx_gemm(a_t.data_ptr() + 2 * before, a_text, None, None, b_t.data_ptr(), b_text, s_t.data_ptr() + 1, s_text, c.data_ptr(), _rows(M, N), "bf16", "f32", False,
                  torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (c.cpu().double().numpy() == want).all()


@pytest.mark.parametrize("M,N,K", [(5, 20, 96), (40, 70, 320), (130, 140, 544), (300, 260, 1056)])
@pytest.mark.parametrize("tile", [0, 32, 64, 128, 256, 128128])
def test_scales_between_the_rows_of_codes_stay_out(M, N, K, tile, monkeypatch):
    """Scales of 255 between, before and behind the rows' own, which start at an odd address."""
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    dev = torch.device("cuda:0")
    rng = np.random.default_rng(K)
    sides, s_pitch = [], K // 32 + 3
    for rows in (M, N):
        codes = rng.integers(0, 16, (rows, K))
        scales = np.full((rows + 9) * s_pitch + 1, 255, np.uint8)
        used = 1 + np.arange(rows)[:, None] * s_pitch + np.arange(K // 32)
        scales[used] = rng.integers(126, 129, used.shape)
        packed = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
        values = mx.LEVELS[codes] * np.repeat(np.ldexp(1.0, scales[used].astype(np.int64) - 127), 32, axis=1)
        sides.append((torch.from_numpy(packed).to(dev), _rows(rows, K), torch.from_numpy(scales).to(dev), "(%d,%d):(%d,1)" % (rows, K // 32, s_pitch), values))
    (a, a_l, a_s, a_sl, av), (b, b_l, b_s, b_sl, bv) = sides
    c = torch.full((M, N), np.nan, device=dev)
    lc.lc_mx_gemm(a.data_ptr(), a_l, a_s.data_ptr() + 1, a_sl, b.data_ptr(), b_l, b_s.data_ptr() + 1, b_sl, c.data_ptr(), _rows(M, N), "mxfp4", "f32", False,
                  torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (c.cpu().double().numpy() == av @ bv.T).all()


@pytest.mark.parametrize("a_dtype", ["mxfp4", "bf16"])
@pytest.mark.parametrize("tile", [0, 12864, 128, 256, 256128, 128128, 128064])
@pytest.mark.parametrize("pitch,c_dtype", [(4128, "f32"), (4130, "f32"), (8256, "f16")])
def test_large_c(a_dtype, tile, pitch, c_dtype, monkeypatch):
    """More than 32 MiB of C, with rows that begin on cache lines and with ones that do not."""
    if tile:
        monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    M, N, K = 2101, pitch - 5, 64
    a, a_s = (_rows(M, K), _scales(M, K)) if a_dtype == "mxfp4" else (_rows(M, K), None)
    _run(a, a_s, _rows(N, K), _scales(N, K), "(%d,%d):(%d,1)" % (M, N, pitch), a_dtype, c_dtype, False, "exact")


def test_large_c_off_a_cache_line():
    dev = torch.device("cuda:0")
    M, N, K = 2050, 4096, 32
    a, b = torch.full((M * K // 2,), 0x22, dtype=torch.uint8, device=dev), torch.full((N * K // 2,), 0x22, dtype=torch.uint8, device=dev)
    s = torch.full((4096,), 127, dtype=torch.uint8, device=dev)
    c = torch.zeros(M * N + 64, device=dev)
    plan = lc.MxGemmPlan(_rows(M, K), _scales(M, K), _rows(N, K), _scales(N, K), _rows(M, N), accumulate=False)
    plan.execute(a.data_ptr(), s.data_ptr(), b.data_ptr(), s.data_ptr(), c.data_ptr() + 16, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert (c[:4] == 0).all() and (c[4:4 + M * N] == K).all() and (c[4 + M * N:] == 0).all()
