"""Quantisation to and from microscaled 4-bit tensors on the GPU against the oracle: every code, scale and value equal, bytes that
belong to nobody left as they were."""
import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _values(rng, rows, k, dtype, kind):
    """(R, K) values of the type, as a float32 tensor: `kind` picks what they are near."""
    if kind == "normal":
        v = rng.standard_normal((rows, k)) * np.exp2(rng.integers(-20, 12, (rows, 1)))
    elif kind == "ties":      # values on the borders between codes, at scales of every size
        v = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, 6.0, 7.0, 7.5, 1.0, 3.0, 4.0], (rows, k)) * rng.choice([-1.0, 1.0], (rows, k))
        v = v * np.exp2(rng.integers(-10, 10, (rows, 1)))
    elif kind == "extremes":  # the type's smallest and largest, zeros of both signs, whole blocks of zeros
        low, high = {"f32": (-149, 126), "bf16": (-133, 126), "f16": (-24, 14)}[dtype]
        v = rng.choice([-1.0, 1.0, 0.0, -0.0, 1.5], (rows, k)) * np.exp2(rng.integers(low, high, (rows, k)).astype(np.float64))
        v[rng.random((rows, k)) < 0.3] = 0.0
        v[::3] = 0.0
        v[1::5] = np.exp2(low)
    else:                     # infinities and NaN in some blocks, the type's lowest value in others
        v = rng.standard_normal((rows, k))
        v[rng.random((rows, k)) < 0.01] = np.nan
        v[rng.random((rows, k)) < 0.01] = np.inf
        v[rng.random((rows, k)) < 0.01] = -np.inf
        v[rng.random((rows, k)) < 0.01] = torch.finfo(TORCH[dtype]).min
    return torch.from_numpy(v.astype(np.float32)).to(TORCH[dtype])


def _same(a, b):
    return ((a == b) & (np.signbit(a) == np.signbit(b))) | (np.isnan(a) & np.isnan(b))


def _check(R, K, P, dtype, x_text, codes_text, scales_text, rule, kind, seed):
    print("case", R, K, P, dtype, x_text, codes_text, scales_text, rule, kind, flush=True)
    rng = np.random.default_rng(seed)
    dev = torch.device("cuda:0")
    v = _values(rng, R, K, dtype, kind)
    X = lc.Layout(x_text)
    origin, size = -X.min_offset + 5, -X.min_offset + X.cosize + 11   # values before and behind, an origin off any vector
    off = torch.from_numpy(mx.offsets(x_text) + origin)
    src = torch.full((size,), 77.0, dtype=TORCH[dtype])
    src[off] = v
    codes = rng.integers(0, 256, lc.Layout(codes_text).cosize // 2 + 16, dtype=np.uint8)
    scales = rng.integers(0, 256, lc.Layout(scales_text).cosize + 16, dtype=np.uint8)
    codes_t, scales_t, src_t = torch.from_numpy(codes).to(dev), torch.from_numpy(scales).to(dev), src.to(dev)
    lc.mx_quantize_tensor(src_t, x_text, codes_t, codes_text, scales_t, scales_text, rule, src_origin=origin)
    torch.cuda.synchronize()
    want_codes, want_scales = mx.quantize(v.double().numpy(), P, rule)
    mx.put_codes(codes, codes_text, want_codes)
    scales[mx.offsets(scales_text)] = want_scales
    assert (scales_t.cpu().numpy() == scales).all()
    assert (codes_t.cpu().numpy() == codes).all()
    # and back
    dst_t = torch.full((size,), 77.0, dtype=TORCH[dtype], device=dev)
    lc.mx_dequantize_tensor(codes_t, codes_text, scales_t, scales_text, dst_t, x_text, dst_origin=origin)
    torch.cuda.synchronize()
    want = torch.full((size,), 77.0, dtype=TORCH[dtype])
    values = mx.dequantize(want_codes, want_scales)[:, :K]
    with np.errstate(over="ignore"):
        want[off] = torch.from_numpy(values).to(TORCH[dtype])
    assert _same(dst_t.float().cpu().numpy(), want.float().numpy()).all()


def _layout(R, K, order):
    return {"k": "(%d,%d):(%d,1)" % (R, K, K), "k_padded": "(%d,%d):(%d,1)" % (R, K, K + 5), "r": "(%d,%d):(1,%d)" % (R, K, R),
            "r_padded": "(%d,%d):(1,%d)" % (R, K, R + 3), "strided": "(%d,%d):(%d,3)" % (R, K, 3 * K + 1), "reversed": "(%d,%d):(-%d,1)" % (R, K, K),
            "reversed_k": "(%d,%d):(%d,-1)" % (R, K, K)}[order]


SIZES = [(1, 1), (1, 32), (2, 7), (3, 33), (5, 64), (8, 100), (17, 256), (64, 520), (65, 1023), (131, 96), (257, 2048), (40, 4099)]


@pytest.mark.parametrize("R,K", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["k", "r", "strided"])
def test_sizes(R, K, dtype, order):
    for seed, (rule, tiles) in enumerate((("floor", False), ("cover", True))):
        P = (K + 255) // 256 * 256 if tiles else (K + 31) // 32 * 32
        scales = str(lc.lc_mx_scale_layout(R, P // 32)) if tiles else "(%d,%d):(%d,1)" % (R, P // 32, P // 32)
        _check(R, K, P, dtype, _layout(R, K, order), "(%d,%d):(%d,1)" % (R, P, P), scales, rule, "normal", seed)


@pytest.mark.parametrize("kind", ["ties", "extremes", "bad"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rule", ["floor", "cover"])
@pytest.mark.parametrize("order", ["k", "r", "reversed"])
def test_values(kind, dtype, rule, order):
    R, K = 48, 160
    _check(R, K, K, dtype, _layout(R, K, order), "(%d,%d):(%d,1)" % (R, K, K), "(%d,%d):(%d,1)" % (R, K // 32, K // 32), rule, kind, 7)


@pytest.mark.parametrize("x", ["k_padded", "r_padded", "reversed", "reversed_k", "((8,3),(64,2)):((64,4000),(1,512))", "((8,3),(4,32)):((1,8),(24,96))",
                               "(24,(16,8)):(16,(1,400))", "((2,12),128):((128,1000),1)"])
@pytest.mark.parametrize("codes,scales", [
    ("(24,128):(160,1)", "(24,4):(7,1)"),                      # rows apart
    ("(24,(32,4)):(32,(1,768))", "(24,4):(1,24)"),             # the same block of all rows together
    ("((4,6),(64,2)):((64,1000000),(1,512))", "((4,6),(2,2)):((2,1000),(1,100))"),
    ("(24,256):(256,1)", "(24,(8,1)):(8,(1,0))"),              # padded by whole blocks
])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts(x, codes, scales, dtype):
    R, K = 24, 128
    codes = codes.replace("1000000", "1024")
    text = x if ":" in x else _layout(R, K, x)
    P = lc.Layout(codes).size // R
    _check(R, K, P, dtype, text, codes, scales, "floor", "normal", 3)


def test_rows_of_nothing_but_zeros_and_one_element():
    _check(1, 1, 32, "bf16", "(1,1):(1,1)", "(1,32):(32,1)", "(1,1):(1,1)", "floor", "bad", 1)
    _check(3, 32, 32, "f16", "(3,32):(32,1)", "(3,32):(32,1)", "(3,1):(1,1)", "cover", "extremes", 2)


def test_offsets_past_32_bits():
    """A source whose rows lie 2^29 + 1 fp32 elements apart (over 4 GiB to the third row), codes 2 GiB apart."""
    dev = torch.device("cuda:0")
    R, K, step = 3, 64, (1 << 29) + 1
    x = torch.zeros((R - 1) * step + K, dtype=torch.float32, device=dev)
    rng = np.random.default_rng(5)
    v = rng.standard_normal((R, K)).astype(np.float32)
    for r in range(R):
        x[r * step:r * step + K] = torch.from_numpy(v[r]).to(dev)
    q_step = 1 << 32
    codes = torch.zeros((R - 1) * q_step // 2 + K // 2, dtype=torch.uint8, device=dev)
    scales = torch.zeros(R * 2, dtype=torch.uint8, device=dev)
    lc.mx_quantize_tensor(x, "(%d,%d):(%d,1)" % (R, K, step), codes, "(%d,%d):(%d,1)" % (R, K, q_step), scales, "(%d,2):(2,1)" % R)
    want_codes, want_scales = mx.quantize(v.astype(np.float64), K, "floor")
    got = np.stack([codes[r * q_step // 2:r * q_step // 2 + K // 2].cpu().numpy() for r in range(R)])
    assert (got == (want_codes[:, 0::2] | (want_codes[:, 1::2] << 4))).all()
    assert (scales.cpu().numpy().reshape(R, 2) == want_scales).all()
    x.fill_(9.0)
    lc.mx_dequantize_tensor(codes, "(%d,%d):(%d,1)" % (R, K, q_step), scales, "(%d,2):(2,1)" % R, x, "(%d,%d):(%d,1)" % (R, K, step))
    values = mx.dequantize(want_codes, want_scales)
    for r in range(R):
        assert (x[r * step:r * step + K].cpu().numpy() == values[r]).all()
    assert float(x[K]) == 9.0 and float(x[step - 1]) == 9.0


def test_in_a_graph_and_on_another_stream():
    dev = torch.device("cuda:0")
    R, K = 33, 512
    text, codes_text, scales_text = "(%d,%d):(1,%d)" % (R, K, R), "(%d,%d):(%d,1)" % (R, K, K), str(lc.lc_mx_scale_layout(R, K // 32))
    q, d = lc.MxQuantizePlan(text, codes_text, scales_text, "bf16"), lc.MxDequantizePlan(codes_text, scales_text, text, "bf16")
    x, y = torch.zeros(R * K, dtype=torch.bfloat16, device=dev), torch.zeros(R * K, dtype=torch.bfloat16, device=dev)
    codes, scales = torch.zeros(R * K // 2, dtype=torch.uint8, device=dev), torch.zeros(R * K // 32, dtype=torch.uint8, device=dev)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def launch(stream):
        q.execute(x.data_ptr(), codes.data_ptr(), scales.data_ptr(), stream)
        d.execute(codes.data_ptr(), scales.data_ptr(), y.data_ptr(), stream)

    launch(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        launch(torch.cuda.current_stream().cuda_stream)
    for rep in range(4):
        rng = np.random.default_rng(rep)
        v = _values(rng, R, K, "bf16", "normal")
        x[torch.from_numpy(mx.offsets(text)).to(dev)] = v.to(dev)
        y.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = mx.dequantize(*mx.quantize(v.double().numpy(), K, "floor"))
        got = y.float().cpu().numpy()[mx.offsets(text)]
        assert _same(got, want.astype(np.float32)).all(), rep


def test_tensor_helpers_refuse_what_does_not_fit():
    dev = torch.device("cuda:0")
    x, codes, scales = torch.zeros(128, device=dev), torch.zeros(64, dtype=torch.uint8, device=dev), torch.zeros(4, dtype=torch.uint8, device=dev)
    text = "(2,64):(64,1)"
    with pytest.raises(ValueError):
        lc.mx_quantize_tensor(x[:127], text, codes, text, scales, "(2,2):(2,1)")
    with pytest.raises(ValueError):
        lc.mx_quantize_tensor(x, text, codes[:63], text, scales, "(2,2):(2,1)")
    with pytest.raises(ValueError):
        lc.mx_quantize_tensor(x, text, codes, text, scales[:3], "(2,2):(2,1)")
    with pytest.raises(ValueError):
        lc.mx_quantize_tensor(x.to(torch.int32), text, codes, text, scales, "(2,2):(2,1)")
    with pytest.raises(ValueError):
        lc.mx_dequantize_tensor(codes.to(torch.int32), text, scales, "(2,2):(2,1)", x, text)
    with pytest.raises(RuntimeError):
        lc.mx_dequantize_tensor(codes.cpu(), text, scales, "(2,2):(2,1)", x, text)
    with pytest.raises(lc.LayoutCopyError):
        lc.mx_quantize_tensor(x, text, codes.repeat(2)[8:], text, scales, "(2,2):(2,1)")   # codes off the 16-byte grid


@pytest.mark.parametrize("R,K,x", [(2101, 4100, "k"), (2101, 4128, "k"), (2101, 4100, "r"), (2104, 4100, "r"), (3, 2900000, "r3"), (4100, 2050, "strided")])
@pytest.mark.parametrize("origin", [0, 1])
def test_large_tensors_on_and_off_cache_lines(R, K, x, origin):
    """More than 32 MiB of fp32, rows or columns that begin on lines and (origin 1) that do not."""
    dev = torch.device("cuda:0")
    text = {"k": "(%d,%d):(%d,1)" % (R, K, 4128), "r": "(%d,%d):(1,%d)" % (R, K, 2112), "r3": "(%d,%d):(1,4)" % (R, K),
            "strided": "(%d,%d):(%d,1)" % (R, K, 2051)}[x]
    P = (K + 31) // 32 * 32
    g = torch.Generator().manual_seed(K)
    codes = torch.randint(0, 256, (R, P // 2), dtype=torch.uint8, generator=g)
    scales = torch.randint(100, 150, (R, P // 32), dtype=torch.uint8, generator=g)
    size = lc.Layout(text).cosize + origin + 9
    dst = torch.full((size,), 77.0, device=dev)
    lc.mx_dequantize_tensor(codes.to(dev), "(%d,%d):(%d,1)" % (R, P, P), scales.to(dev), "(%d,%d):(%d,1)" % (R, P // 32, P // 32), dst, text, dst_origin=origin)
    torch.cuda.synchronize()
    levels = torch.from_numpy(mx.LEVELS).float()   # (codes times powers of two: exact in fp32)
    want = levels[torch.stack([codes & 15, codes >> 4], 2).long().reshape(R, P)] * torch.exp2(scales.float() - 127).repeat_interleave(32, 1)
    off = torch.from_numpy(mx.offsets(text)).reshape(R, K) + origin
    expect = torch.full((size,), 77.0)
    expect[off] = want[:, :K]
    assert torch.equal(dst.cpu(), expect)
