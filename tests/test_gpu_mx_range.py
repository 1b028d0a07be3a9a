"""Products with microscaled 4-bit operands over the whole range of scales, one term to a sum: what comes out is the exact product of the two elements
rounded once to fp32 (subnormal results included; infinite from 2^128 on), so everything is compared for equality.  Beside 16-bit elements the code's
element is first rounded to their type, where it is infinite from 2^128 (bf16) or 65520 (fp16) on."""
import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
SCALES = np.arange(255)   # 2^-127 .. 2^127


def _rows(r, p):
    return "(%d,%d):(%d,1)" % (r, p, p)


def _first_of_row(code, rows, k):
    """Packed rows of k codes that are zeros but for the first."""
    packed = np.zeros((rows, k // 2), np.uint8)
    packed[:, 0] = code
    return torch.from_numpy(packed).reshape(-1).cuda()


def _run(plan, *tensors):
    plan.execute(*(None if t is None else t.data_ptr() for t in tensors), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("a_dtype,powers", [("bf16", (-133, -127, -126, -100, -60, -10, 0, 10, 60, 100, 126)), ("f16", (-24, -15, -14, -4, 0, 10, 15))])
@pytest.mark.parametrize("tile,want", [(16, "kernel=direct"), (3216, "kernel=direct"), (32, "kernel=direct"), (12864, "kernel=stream"), (128, "kernel=stream"),
                                       (256, "kernel=wide"), (256128, "kernel=wide"), (128128, "kernel=wide"), (128064, "kernel=wide")])
def test_weights(a_dtype, powers, tile, want, monkeypatch):
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    M, N, K = len(powers), len(SCALES), 32
    a = torch.zeros(M, K, dtype=TORCH[a_dtype])
    a[:, 0] = torch.from_numpy(np.ldexp(1.0, np.array(powers))).to(TORCH[a_dtype])
    assert (a[:, 0].double().numpy() == np.ldexp(1.0, np.array(powers))).all()
    plan = lc.MxGemmPlan(_rows(M, K), None, _rows(N, K), _rows(N, 1), _rows(M, N), a_dtype, "f32", False)
    assert want in plan.describe()
    scales = torch.from_numpy(SCALES.astype(np.uint8)).cuda()
    for code in range(1, 16):
        weights = torch.from_numpy(mx.LEVELS[code] * np.ldexp(1.0, SCALES - 127)).to(TORCH[a_dtype]).double()
        c = torch.full((M, N), 7.0, device="cuda")
        _run(plan, a.cuda(), None, _first_of_row(code, N, K), scales, c)
        assert torch.equal(c.cpu().nan_to_num(nan=-7.0), torch.outer(a[:, 0].double(), weights).float().nan_to_num(nan=-7.0)), code


@pytest.mark.parametrize("tile,want", [(16, "kernel=direct"), (3216, "kernel=direct"), (32, "kernel=direct"), (64, "kernel=stream"), (12864, "kernel=stream"),
                                       (128, "kernel=stream"), (256, "kernel=ring"), (128128, "kernel=ring")])
def test_codes_by_codes(tile, want, monkeypatch):
    """Every scale by every scale, 2^-127 times 2^127 among them, whose product is an ordinary number."""
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    M = N = len(SCALES)
    K = 128
    scales = np.full((M, K // 32), 127, np.uint8)
    scales[:, 0] = SCALES
    s = torch.from_numpy(scales).reshape(-1).cuda()
    plan = lc.MxGemmPlan(_rows(M, K), _rows(M, K // 32), _rows(N, K), _rows(N, K // 32), _rows(M, N), accumulate=False)
    assert want in plan.describe()
    for a, b in ((1, 1), (2, 2), (3, 3), (7, 7), (1, 7), (7, 9), (11, 7), (13, 15), (2, 0)):
        values = [torch.from_numpy(mx.LEVELS[code] * np.ldexp(1.0, SCALES - 127)) for code in (a, b)]
        c = torch.full((M, N), 7.0, device="cuda")
        _run(plan, _first_of_row(a, M, K), s, _first_of_row(b, N, K), s, c)
        assert torch.equal(c.cpu(), torch.outer(*values).float()), (a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_largest_values_quantised(dtype):
    """From 3.5 2^126 on, COVER's nearest code is 4 at 2^126: 2^128, which neither type holds.  FLOOR saturates at 6 at 2^125."""
    torch_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.tensor([3.4375 * 2.0 ** 126, 3.5 * 2.0 ** 126, torch.finfo(torch_dtype).max], dtype=torch_dtype, device="cuda")
    src = torch.zeros(3, 32, dtype=torch_dtype, device="cuda")
    src[:, 0] = x
    one = torch.zeros(32, dtype=torch.bfloat16, device="cuda")
    one[0] = 1
    inf = float("inf")
    for rule, want in (("cover", [3 * 2.0 ** 126, inf, inf]), ("floor", [6 * 2.0 ** 125] * 3)):
        codes, scales = torch.zeros(48, dtype=torch.uint8, device="cuda"), torch.zeros(3, dtype=torch.uint8, device="cuda")
        back, c = torch.zeros(3, 32, dtype=torch_dtype, device="cuda"), torch.zeros(3, device="cuda")
        lc.mx_quantize_tensor(src, _rows(3, 32), codes, _rows(3, 32), scales, _rows(3, 1), rule)
        lc.mx_dequantize_tensor(codes, _rows(3, 32), scales, _rows(3, 1), back, _rows(3, 32))
        lc.mx_gemm_tensor(one, _rows(1, 32), None, None, codes, _rows(3, 32), scales, _rows(3, 1), c, _rows(1, 3), accumulate=False)
        assert back[:, 0].tolist() == want and c.tolist() == want
