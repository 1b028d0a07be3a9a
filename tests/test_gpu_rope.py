"""Rotary positions on the GPU against the definition in 64 bits.

A result is a c - b s in fp32 with c and s within 2^-24 of their value relative to it (they are rounded once; the series behind them is far below), one product
rounded by 2^-24 of itself and one sum by 2^-24 of itself: three times 2^-24 of |a c| + |b s| in all, to first order; 1 % covers the rest.  Rounding to 16 bits
adds half a step, 2^-8 (bf16) or 2^-11 (f16) of the value, and f16's smallest step 2^-25.  What is copied is copied bit for bit."""
import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx
from oracle import serve_oracle as so

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _dense(T, H, D, order):
    return {"thd": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, H * D, D), "htd": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, D, T * D), "row": "(%d,%d,%d):(%d,%d,1)" % (T, H, D, (H + 3) * D + 1, D),
            "dht": "(%d,%d,%d):(1,%d,%d)" % (T, H, D, T, T * H), "back": "(%d,%d,%d):(-%d,%d,1)" % (T, H, D, H * D, D), "wide": "(%d,%d,%d):(%d,%d,3)" % (T, H, D, 3 * H * D, 3 * D),
            "batch": "((%d,1),%d,%d):((%d,7),%d,1)" % (T, H, D, H * D, D)}[order]


def _tolerance(want, size, dtype):
    tol = 3.03 * 2.0 ** -24 * size
    return tol + HALF_STEP[dtype] * (np.abs(want) + tol) + (2.0 ** -25 if dtype == "f16" else 0.0)


def _run(T, H, D, rotary, pairs, dtype, x_order="thd", y_order="thd", transposed=False, factor=1.0, far=5000, rule="plain", in_place=False, seed=0):
    print("case", T, H, D, rotary, pairs, dtype, x_order, y_order, transposed, factor, far, in_place, flush=True)
    rng = np.random.default_rng(seed)
    dev = torch.device("cuda:0")
    x_text, y_text = _dense(T, H, D, x_order), _dense(T, H, D, y_order)
    X, Y = lc.Layout(x_text), lc.Layout(y_text)
    origin, y_origin = 3 - X.min_offset, 5 - Y.min_offset
    x_off, y_off = mx.offsets(x_text) + origin, mx.offsets(y_text) + y_origin
    src = torch.from_numpy(rng.standard_normal(origin + X.cosize + 9).astype(np.float32)).to(TORCH[dtype])
    positions = rng.integers(-far, far, T).astype(np.int32)
    positions[0] = 0
    frequencies = np.array(lc.lc_rope_frequencies(rotary, 10000.0, rule, 1.0 if rule == "plain" else 8.0, 4096), np.float32)
    x = src.double().numpy()[x_off]
    want, size = so.rotate(x, positions, frequencies, rotary, pairs, transposed, factor)
    src_t = src.to(dev)
    dst_t = src_t if in_place else torch.full((y_origin + Y.cosize + 9,), 77.0, dtype=TORCH[dtype], device=dev)
    lc.rope_tensor(src_t, x_text, torch.from_numpy(positions).to(dev), torch.from_numpy(frequencies).to(dev), dst_t, x_text if in_place else y_text, rotary, pairs, transposed, factor,
                   x_origin=origin, y_origin=origin if in_place else y_origin)
    torch.cuda.synchronize()
    got = dst_t.double().cpu().numpy()
    at = x_off if in_place else y_off
    assert (np.abs(got[at] - want) <= _tolerance(want, size, dtype)).all(), np.abs(got[at] - want).max()
    assert (got[at][..., rotary:] == x[..., rotary:]).all()
    rest = np.ones(len(got), bool)
    rest[at.reshape(-1)] = False
    assert (got[rest] == (src.double().numpy() if in_place else np.full(len(got), 77.0))[rest]).all()   # bytes that are nobody's


SIZES = [(1, 1, 2, 2), (1, 1, 3, 2), (1, 40, 128, 128), (5, 3, 64, 64), (64, 40, 128, 128), (33, 9, 80, 40), (7, 2, 96, 96), (130, 1, 32, 16), (3, 2, 513, 512), (300, 12, 80, 80), (2, 70, 256, 192),
         (2049, 8, 64, 32), (17, 5, 66, 66)]


@pytest.mark.parametrize("T,H,D,rotary", SIZES)
@pytest.mark.parametrize("pairs", ["half", "neighbours"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_sizes(T, H, D, rotary, pairs, dtype):
    _run(T, H, D, rotary, pairs, dtype)


@pytest.mark.parametrize("x_order,y_order", [("row", "thd"), ("htd", "thd"), ("thd", "htd"), ("dht", "thd"), ("thd", "dht"), ("back", "thd"), ("thd", "back"), ("wide", "row"), ("batch", "thd")])
@pytest.mark.parametrize("pairs", ["half", "neighbours"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layouts(x_order, y_order, pairs, dtype):
    _run(21, 4, 72, 48, pairs, dtype, x_order, y_order)


@pytest.mark.parametrize("pairs", ["half", "neighbours"])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_the_other_way_stretched_and_scaled(pairs, dtype):
    _run(40, 3, 64, 64, pairs, dtype, transposed=True, factor=0.75, rule="parts")
    _run(40, 3, 64, 48, pairs, dtype, transposed=True, rule="bands")
    _run(40, 3, 64, 64, pairs, dtype, factor=1.25, rule="base")


@pytest.mark.parametrize("far", [1 << 20, 1 << 29])
def test_far_positions(far):
    """(products of a position below 2^29 and an fp32 frequency have 53 bits: the oracle's angle is exact)"""
    _run(64, 2, 128, 128, "half", "f32", far=far)


@pytest.mark.parametrize("T,H,D,rotary", [(5, 3, 64, 64), (33, 9, 80, 40), (300, 12, 66, 66)])
@pytest.mark.parametrize("pairs", ["half", "neighbours"])
@pytest.mark.parametrize("x_order", ["thd", "dht"])
def test_in_place(T, H, D, rotary, pairs, x_order):
    _run(T, H, D, rotary, pairs, "bf16", x_order, in_place=True)


def test_infinities_and_nan_stay_in_their_pair():
    dev = torch.device("cuda:0")
    x = torch.ones(4, 2, 64, device=dev)
    x[1, 0, 5], x[2, 1, 40], x[3, 0, 60] = float("inf"), float("nan"), float("-inf")
    f = torch.tensor(lc.lc_rope_frequencies(48), device=dev)
    y = torch.empty_like(x)
    lc.rope_tensor(x, _dense(4, 2, 64, "thd"), torch.arange(4, dtype=torch.int32, device=dev), f, y, _dense(4, 2, 64, "thd"), 48)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1, 0, [5, 29]], want[2, 1, [16, 40]], want[3, 0, 60] = True, True, True
    assert (bad == want).all() and y[3, 0, 60] == float("-inf")


def test_gradient_against_differences():
    """The transposed call gives the gradient of the plain one: of w . rope(x), element by element, by differences in steps that both rounding and the
    (linear) function leave exact to 2^-18."""
    rng = np.random.default_rng(4)
    T, H, D, rotary = 2, 2, 16, 12
    dev = torch.device("cuda:0")
    text = _dense(T, H, D, "thd")
    p = torch.tensor([3, 100], dtype=torch.int32, device=dev)
    f = torch.tensor(lc.lc_rope_frequencies(rotary), device=dev)
    x, w = (torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(dev) for _ in range(2))
    for pairs in ("half", "neighbours"):
        def rope(v, transposed=False):
            y = torch.empty_like(v)
            lc.rope_tensor(v, text, p, f, y, text, rotary, pairs, transposed, factor=1.5)
            return y
        grad = rope(w, True).double().cpu()
        for i in range(0, T * H * D, 7):
            step = torch.zeros(T * H * D, device=dev)
            step[i] = 1.0
            step = step.view(T, H, D)
            slope = (w.double() * (rope(x + step).double() - rope(x - step).double())).sum() / 2
            assert abs(slope.item() - grad.view(-1)[i].item()) < 2.0 ** -18


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(5)
    dev = torch.device("cuda:0")
    T, H, D = 64, 8, 128
    text = _dense(T, H, D, "thd")
    plan = lc.RopePlan(text, text, "bf16", D)
    f = torch.tensor(lc.lc_rope_frequencies(D), device=dev)
    x, p = torch.empty(T, H, D, dtype=torch.bfloat16, device=dev), torch.empty(T, dtype=torch.int32, device=dev)
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan.execute(x.data_ptr(), p.data_ptr(), f.data_ptr(), y.data_ptr(), stream=side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        plan.execute(x.data_ptr(), p.data_ptr(), f.data_ptr(), y.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(dev))
        p.copy_(torch.from_numpy(rng.integers(0, 1000, T).astype(np.int32)).to(dev))
        graph.replay()
        torch.cuda.synchronize()
        want, size = so.rotate(x.double().cpu().numpy(), p.cpu().numpy(), f.cpu().numpy(), D, "half")
        assert (np.abs(y.double().cpu().numpy() - want) <= _tolerance(want, size, "bf16")).all()
        eager = torch.empty_like(x)
        lc.rope_tensor(x, text, p, f, eager, text, D)
        assert torch.equal(eager, y)


@pytest.mark.parametrize("pairs", ["half", "neighbours"])
def test_angles_up_to_the_largest(pairs):
    """Angles of 2^20 to 2^64 radians, whose products with 23 bits of position and 24 of frequency 64 bits hold exactly: 2^-40 more than elsewhere."""
    rng = np.random.default_rng(7)
    dev = torch.device("cuda:0")
    T, rotary = 64, 88
    positions = (rng.integers(1 << 22, 1 << 23, T) << 8).astype(np.int32) * rng.choice([-1, 1], T).astype(np.int32)
    frequencies = np.ldexp(rng.uniform(1, 2, rotary // 2).astype(np.float32), np.arange(rotary // 2) - 11).astype(np.float32)
    x = rng.standard_normal((T, 2, rotary)).astype(np.float32)
    want, size = so.rotate(x, positions, frequencies, rotary, pairs)
    y, text = torch.empty(T, 2, rotary, device=dev), "(%d,2,%d):(%d,%d,1)" % (T, rotary, 2 * rotary, rotary)
    lc.rope_tensor(torch.from_numpy(x).to(dev), text, torch.from_numpy(positions).to(dev), torch.from_numpy(frequencies).to(dev), y, text, rotary, pairs)
    assert (np.abs(y.double().cpu().numpy() - want) <= _tolerance(want, size, "f32") + 2.0 ** -40 * 2 * np.abs(x).max()).all()
