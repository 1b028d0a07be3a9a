"""Microscaled 4-bit tensors (MXFP4), as measurable cases: quantisation, dequantisation, and the products that read them.

An MXFP4 tensor holds elements of 4 bits (sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
negatives), two to a byte with the even element in the low half, in blocks of 32 along one mode; every block has one scale of
8 bits s that stands for 2^(s - 127), 255 for NaN.  The blocked mode is padded to whole blocks with zeros.

A case is a dict of plain values; its `kind` names the path:
  round     R x K values quantised and dequantised again (training that imitates 4 bits, checks of a quantiser)
  expand    a quantised matrix back to 16 or 32 bits
  product   C(m,n) = sum_k A(m,k) B(n,k), both operands quantised
  linear    a layer's forward pass: activations quantised, then multiplied with quantised weights
  train     that layer's backward pass: the gradients of the input and of the weights, each a product of operands quantised
            along the mode it sums over
  weights   C(m,n) = sum_k A(m,k) B(n,k), A in 16 bits, B quantised along k (weights of a served model)
  grad      dX(m,k) = sum_n dY(m,n) W(n,k), dY in 16 bits, W quantised along k, which is not summed over here (tuning with
            frozen 4-bit weights)
`order`: k (a row's elements are neighbours) or r (a column's are).  `rule`: the block's scale 2^e from its largest magnitude
a: floor (e = floor(log2 a) - 2) or cover (the smallest e with a <= 6 * 2^e).  `scales`: how a matrix's scales lie: rows (as a
row-major matrix) or tiles (eight neighbouring blocks of a row together, then the next row's eight).
"""
import math

import torch

own = False   # set from outside: True takes the framework's kernels, False the plain form

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_BLOCK = 32


def listed():
    return [
        # a decoding step's activations between two layers: latency of two launches
        {"name": "round_small_bf16", "kind": "round", "R": 16, "K": 4096, "dtype": "bf16", "order": "k", "rule": "floor", "scales": "rows"},
        # a weight matrix imitated in 4 bits during training
        {"name": "round_large_bf16", "kind": "round", "R": 8192, "K": 8192, "dtype": "bf16", "order": "k", "rule": "cover", "scales": "tiles"},
        # fp32 master weights quantised along the mode they are not stored by, sides nobody padded
        {"name": "round_columns_f32", "kind": "round", "R": 4100, "K": 5003, "dtype": "f32", "order": "r", "rule": "floor", "scales": "rows"},
        # quantised weights brought back to 16 bits, transposed on the way
        {"name": "expand_bf16", "kind": "expand", "R": 8192, "K": 8192, "dtype": "bf16", "order": "r", "scales": "tiles"},
        # a small layer on a ragged batch: launch and fill of the chip
        {"name": "product_odd_bf16", "kind": "product", "M": 123, "N": 1001, "K": 544, "out": "bf16", "scales": "rows"},
        # prefill / training size, fp32 result
        {"name": "product_large_f32", "kind": "product", "M": 8192, "N": 8192, "K": 8192, "out": "f32", "scales": "tiles"},
        # a layer's forward pass on a long prompt, quantisation of the activations included
        {"name": "linear_bf16", "kind": "linear", "M": 4096, "N": 8192, "K": 4096, "dtype": "bf16", "out": "bf16", "rule": "floor", "scales": "tiles"},
        # the backward pass of a square layer over 4096 tokens
        {"name": "train_bf16", "kind": "train", "M": 4096, "N": 2048, "K": 2048, "dtype": "bf16", "out": "f32", "rule": "cover", "scales": "tiles"},
        # one token through a served layer: all of the weights for one row
        {"name": "weights_one_bf16", "kind": "weights", "M": 1, "N": 8192, "K": 8192, "dtype": "bf16", "out": "bf16", "scales": "rows"},
        # a decoding batch
        {"name": "weights_batch_f16", "kind": "weights", "M": 32, "N": 8192, "K": 8192, "dtype": "f16", "out": "f32", "scales": "rows"},
        # a prompt through a served layer
        {"name": "weights_prompt_bf16", "kind": "weights", "M": 2048, "N": 8192, "K": 4096, "dtype": "bf16", "out": "bf16", "scales": "tiles"},
        # the input's gradient through frozen 4-bit weights
        {"name": "grad_bf16", "kind": "grad", "M": 2048, "N": 4096, "K": 4096, "dtype": "bf16", "out": "bf16", "scales": "tiles"},
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer in [lo, hi], a multiple of step, spread over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def _side(rng, lo, hi):
    """A side of a matrix: every third one odd, the others multiples of 8."""
    return _log_int(rng, lo, hi) | 1 if rng.random() < 1 / 3 else _log_int(rng, lo, hi, 8)


def draw(rng):
    kind = rng.choice(["round", "round", "expand", "product", "linear", "train", "weights", "weights", "grad"])
    half, tiles = rng.choice(["bf16", "f16"]), rng.choice(["tiles", "rows"])
    case = {"kind": kind, "scales": tiles}
    if kind in ("round", "expand"):
        case.update(R=_side(rng, 1, 8191), K=_side(rng, 32, 8191), dtype=rng.choice(["f32", "bf16", "f16"]), order=rng.choice(["k", "r"]))
    elif kind == "product":
        case.update(M=_side(rng, 16, 8191), N=_side(rng, 16, 8191), K=_log_int(rng, 64, 8192, 32), out=rng.choice(["f32", "bf16", "f16"]))
    elif kind == "linear":
        case.update(M=_side(rng, 16, 4095), N=_side(rng, 256, 8191), K=_side(rng, 256, 8191), dtype=half, out=half)
    elif kind == "train":
        case.update(M=_side(rng, 64, 4095), N=_side(rng, 64, 4095), K=_side(rng, 64, 4095), dtype=half, out="f32")
    elif kind == "weights":
        case.update(M=_log_int(rng, 1, 2048), N=_side(rng, 256, 8191), K=_side(rng, 256, 8191), dtype=half, out=rng.choice(["f32", half]))
    else:
        case.update(M=_log_int(rng, 16, 2048), N=_side(rng, 256, 4095), K=_side(rng, 256, 4095), dtype=half, out=rng.choice(["f32", half]))
    if kind in ("round", "linear", "train"):
        case["rule"] = rng.choice(["floor", "cover"])
    return case


# ---- layouts of a quantised R x K matrix: codes row-major over whole blocks, scales by `scales` ----
def _padded(k, scales):
    step = 8 * _BLOCK if scales == "tiles" else _BLOCK
    return (k + step - 1) // step * step


def _codes(rows, k, scales, blocked=1):
    """Layout of the codes, counted in elements of 4 bits; blocked: which mode the blocks run along."""
    kp = _padded(k, scales)
    return "(%d,%d):(%d,1)" % (rows, kp, kp) if blocked == 1 else "(%d,%d):(1,%d)" % (kp, rows, kp)


def _scale_modes(rows, k, scales):
    blocks = _padded(k, scales) // _BLOCK
    return (str(rows), "8", "(8,%d)" % (blocks // 8), "(1,%d)" % (8 * rows)) if scales == "tiles" else (str(rows), str(blocks), str(blocks), "1")


def _scales(rows, k, scales, blocked=1):
    r, rd, b, bd = _scale_modes(rows, k, scales)
    return "(%s,%s):(%s,%s)" % ((r, b, rd, bd) if blocked == 1 else (b, r, bd, rd))


def _dense(rows, k, order):
    return "(%d,%d):(%d,1)" % (rows, k, k) if order == "k" else "(%d,%d):(1,%d)" % (rows, k, rows)


# ---- the plain form ----
def _levels(device):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=device)


def _power_of_two(e):
    """2^e in 64 bits for whole e, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _plain_blocks(x, scales):
    """x (R, K) with zeros up to whole blocks, as (R, blocks, 32), in 64 bits: values next to a border between two codes decide."""
    kp = _padded(x.shape[1], scales)
    return torch.nn.functional.pad(x.double(), (0, kp - x.shape[1])).view(x.shape[0], kp // _BLOCK, _BLOCK)


def _plain_quantize(x, rule, scales):
    """Codes as numbers 0 .. 15 (R, blocks, 32), exponents of the scales (R, blocks); a block that holds infinities or NaN gets 128."""
    v = _plain_blocks(x, scales)
    largest = v.abs().amax(-1)
    fraction, power = torch.frexp(largest)   # largest = fraction * 2^power, fraction in [1/2, 1)
    e = power - 3
    if rule == "cover":
        e = e + (fraction > 0.75)
    e = torch.where(largest > 0, e, -127).clamp(-127, 127)
    bad = ~torch.isfinite(largest)
    e = torch.where(bad, 128, e)
    y = torch.where(bad[..., None], 0.0, v.abs() * _power_of_two(-e)[..., None])
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    y = (torch.round(y / step) * step).clamp(max=6.0)
    code = torch.where(y < 2, y * 2, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8)
    negative = torch.signbit(v) & ~bad[..., None]
    return code + 8 * negative.to(torch.uint8), e.to(torch.int32)


def _plain_values(code, e):
    """(R, blocks, 32) codes and (R, blocks) exponents -> (R, K) values in 32 bits."""
    scale = torch.where(e == 128, math.nan, _power_of_two(e)).float()
    return (_levels(code.device)[code.long()] * scale[..., None]).reshape(code.shape[0], -1)


def _pack(code, e, scales):
    """The bytes that a program holds: codes two to a byte (R, K / 2), scales in their order."""
    code = code.reshape(code.shape[0], -1, 2)
    packed = (code[..., 0] | (code[..., 1] << 4)).contiguous()
    s = (e + 127).to(torch.uint8)
    if scales == "tiles":
        s = s.view(s.shape[0], -1, 8).transpose(0, 1)
    return packed, s.contiguous()


def _unpack(packed, s, scales):
    code = torch.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[0], -1, _BLOCK)
    if scales == "tiles":
        s = s.transpose(0, 1).reshape(packed.shape[0], -1)
    return code, s.to(torch.int32) - 127


# ---- inputs ----
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(rows, k, g):
    """N(0,1) with a few channels that are far larger, as layers' inputs have them."""
    loud = torch.exp2(torch.randn(k, device="cuda", generator=g).abs().sub_(2).clamp_(min=0).mul_(3))
    return torch.randn(rows, k, device="cuda", generator=g).mul_(loud)


def _weights(rows, k, g):
    return torch.randn(rows, k, device="cuda", generator=g).mul_(1 / math.sqrt(k))


def _packed_weights(rows, k, scales, g):
    """Weights that are quantised already, at random: every code, scales of a layer's size."""
    kp = _padded(k, scales)
    code = torch.randint(0, 16, (rows, kp // _BLOCK, _BLOCK), device="cuda", generator=g, dtype=torch.uint8)
    code.view(rows, kp)[:, k:] = 0
    e = torch.randint(-9, -4, (rows, kp // _BLOCK), device="cuda", generator=g, dtype=torch.int32)
    return _pack(code, e, scales)


def _inputs(case, seed):
    """What a program has in hand: tensors by name; quantised ones as (codes, scales)."""
    g, kind, scales = _generator(seed), case["kind"], case["scales"]
    if kind == "round":
        x = _activations(case["R"], case["K"], g).to(_TORCH[case["dtype"]])
        return {"x": x.t().contiguous() if case["order"] == "r" else x}   # order r: stored (K, R)
    if kind == "expand":
        return {"x": _packed_weights(case["R"], case["K"], scales, g)}
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "product":
        return {"a": _packed_weights(M, K, scales, g), "b": _packed_weights(N, K, scales, g)}
    half = _TORCH[case["dtype"]]
    if kind == "linear":
        return {"x": _activations(M, K, g).to(half), "b": _packed_weights(N, K, scales, g)}
    if kind == "train":   # W^T is quantised along n once a step, with the update
        return {"x": _activations(M, K, g).to(half), "dy": _weights(M, N, g).to(half), "wt": _packed_weights(K, N, scales, g)}
    if kind == "weights":
        return {"a": _activations(M, K, g).to(half), "b": _packed_weights(N, K, scales, g)}
    return {"a": _weights(M, N, g).to(half), "b": _packed_weights(N, K, scales, g)}


def _empty_mx(rows, k, scales):
    kp = _padded(k, scales)
    return torch.empty(rows * kp // 2, dtype=torch.uint8, device="cuda"), torch.empty(rows * kp // _BLOCK, dtype=torch.uint8, device="cuda")


def _plans(case):
    """The framework's plans of one case and the buffers that a program keeps beside them."""
    import paper_2603_02298_amd as lc
    kind, how = case["kind"], case["scales"]
    if kind in ("round", "expand"):
        R, K = case["R"], case["K"]
        codes, scales, dense = _codes(R, K, how), _scales(R, K, how), _dense(R, K, case["order"])
        # the padding is dropped on the way back: the blocks' first K elements
        plans = {"back": lc.MxDequantizePlan(codes, scales, dense, case["dtype"]), "y": torch.empty(R * K, dtype=_TORCH[case["dtype"]], device="cuda")}
        if kind == "round":
            plans.update(quantize=lc.MxQuantizePlan(dense, codes, scales, case["dtype"], case["rule"]), q=_empty_mx(R, K, how))
        return plans
    M, N, K = case["M"], case["N"], case["K"]
    out = _TORCH[case["out"]]
    if kind == "train":
        x, dy = "(%d,%d):(%d,1)" % (M, K, K), "(%d,%d):(%d,1)" % (M, N, N)
        xt, dyt = "(%d,%d):(1,%d)" % (K, M, K), "(%d,%d):(1,%d)" % (N, M, N)
        return {
            "q_dy": lc.MxQuantizePlan(dy, _codes(M, N, how), _scales(M, N, how), case["dtype"], case["rule"]),
            "q_dyt": lc.MxQuantizePlan(dyt, _codes(N, M, how), _scales(N, M, how), case["dtype"], case["rule"]),
            "q_xt": lc.MxQuantizePlan(xt, _codes(K, M, how), _scales(K, M, how), case["dtype"], case["rule"]),
            "dx_of": lc.MxGemmPlan(_codes(M, N, how), _scales(M, N, how), _codes(K, N, how), _scales(K, N, how), x, c_dtype=case["out"], accumulate=False),
            "dw_of": lc.MxGemmPlan(_codes(N, M, how), _scales(N, M, how), _codes(K, M, how), _scales(K, M, how), "(%d,%d):(%d,1)" % (N, K, K),
                                   c_dtype=case["out"], accumulate=False),
            "dy_q": _empty_mx(M, N, how), "dyt_q": _empty_mx(N, M, how), "xt_q": _empty_mx(K, M, how),
            "dx": torch.empty(M, K, dtype=out, device="cuda"), "dw": torch.empty(N, K, dtype=out, device="cuda")}
    if kind in ("product", "linear"):
        plans = {"gemm": lc.MxGemmPlan(_codes(M, K, how), _scales(M, K, how), _codes(N, K, how), _scales(N, K, how), "(%d,%d):(%d,1)" % (M, N, N),
                                       c_dtype=case["out"], accumulate=False), "c": torch.empty(M, N, dtype=out, device="cuda")}
        if kind == "linear":
            plans.update(quantize=lc.MxQuantizePlan("(%d,%d):(%d,1)" % (M, K, K), _codes(M, K, how), _scales(M, K, how), case["dtype"], case["rule"]),
                         q=_empty_mx(M, K, how))
        return plans
    if kind == "weights":
        return {"gemm": lc.MxGemmPlan("(%d,%d):(%d,1)" % (M, K, K), None, _codes(N, K, how), _scales(N, K, how), "(%d,%d):(%d,1)" % (M, N, N),
                                      a_dtype=case["dtype"], c_dtype=case["out"], accumulate=False), "c": torch.empty(M, N, dtype=out, device="cuda")}
    return {"gemm": lc.MxGemmPlan("(%d,%d):(%d,1)" % (M, N, N), None, _codes(N, K, how, blocked=0), _scales(N, K, how, blocked=0), "(%d,%d):(%d,1)" % (M, K, K),
                                  a_dtype=case["dtype"], c_dtype=case["out"], accumulate=False), "c": torch.empty(M, K, dtype=out, device="cuda")}


def prepare(case, seed):
    state = {"case": case, "in": _inputs(case, seed), "stream": torch.cuda.current_stream().cuda_stream}
    if own:
        state["plans"] = _plans(case)
    return state


def _addresses(*tensors):
    return [t.data_ptr() for t in tensors]


def _run_own(state):
    p, t, kind, stream = state["plans"], state["in"], state["case"]["kind"], state["stream"]
    if kind in ("round", "expand"):
        q = t["x"]
        if kind == "round":
            q = p["q"]
            p["quantize"].execute(*_addresses(t["x"], *q), stream)
        p["back"].execute(*_addresses(*q, p["y"]), stream)
        return p["y"]
    if kind == "train":
        p["q_dy"].execute(*_addresses(t["dy"], *p["dy_q"]), stream)
        p["q_dyt"].execute(*_addresses(t["dy"], *p["dyt_q"]), stream)
        p["q_xt"].execute(*_addresses(t["x"], *p["xt_q"]), stream)
        p["dx_of"].execute(*_addresses(*p["dy_q"], *t["wt"], p["dx"]), stream)
        p["dw_of"].execute(*_addresses(*p["dyt_q"], *p["xt_q"], p["dw"]), stream)
        return {"dx": p["dx"], "dw": p["dw"]}
    if kind in ("product", "linear"):
        a = t.get("a")
        if kind == "linear":
            a = p["q"]
            p["quantize"].execute(*_addresses(t["x"], *a), stream)
        p["gemm"].execute(*_addresses(*a, *t["b"], p["c"]), stream)
    else:
        p["gemm"].execute(t["a"].data_ptr(), None, *_addresses(*t["b"], p["c"]), stream)
    return p["c"]


def _matmul(a, b):
    return torch.mm(a, b.contiguous())


def _run_plain(state):
    case, t = state["case"], state["in"]
    kind, how = case["kind"], case["scales"]
    values = lambda q: _plain_values(*_unpack(*q, how))   # noqa: E731
    if kind in ("round", "expand"):
        x = t["x"]
        if kind == "round":
            y = _plain_values(*_plain_quantize(x.t() if case["order"] == "r" else x, case["rule"], how))
        else:
            y = values(x)
        y = y[:, :case["K"]].to(_TORCH[case["dtype"]])
        return (y.t() if case["order"] == "r" else y).contiguous().view(-1)
    out = _TORCH[case["out"]]
    if kind == "train":
        again = lambda v: _plain_values(*_plain_quantize(v, case["rule"], how))   # noqa: E731
        dx = _matmul(again(t["dy"]), values(t["wt"]).t())
        dw = _matmul(again(t["dy"].t()), again(t["x"].t()).t())
        return {"dx": dx.to(out), "dw": dw.to(out)}
    if kind in ("product", "linear"):
        a = _plain_values(*_plain_quantize(t["x"], case["rule"], how)) if kind == "linear" else values(t["a"])
        return _matmul(a, values(t["b"]).t()).to(out)
    w = values(t["b"])[:, :case["K"]]
    return (_matmul(t["a"].float(), w.t()) if kind == "weights" else _matmul(t["a"].float(), w)).to(out)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _mx_bytes(rows, k, scales):
    """Codes and scales of a quantised matrix, without its padding."""
    return rows * k / 2 + rows * ((k + _BLOCK - 1) // _BLOCK)


def work(case):
    kind, how = case["kind"], case["scales"]
    if kind in ("round", "expand"):
        R, K, e = case["R"], case["K"], _BYTES[case["dtype"]]
        return {"bytes": R * K * e + (R * K * e + 2 * _mx_bytes(R, K, how) if kind == "round" else _mx_bytes(R, K, how)), "flops": 0}
    M, N, K, o = case["M"], case["N"], case["K"], _BYTES[case["out"]]
    if kind == "train":   # dY once, X once; the quantised copies written and read; two products
        made = _mx_bytes(M, N, how) + _mx_bytes(N, M, how) + _mx_bytes(K, M, how)
        return {"bytes": 2 * M * (N + K) + 2 * made + _mx_bytes(K, N, how) + o * (M * K + N * K), "flops": 4 * M * N * K}
    if kind == "product":
        return {"bytes": _mx_bytes(M, K, how) + _mx_bytes(N, K, how) + o * M * N, "flops": 2 * M * N * K}
    if kind == "linear":
        return {"bytes": 2 * M * K + 2 * _mx_bytes(M, K, how) + _mx_bytes(N, K, how) + o * M * N, "flops": 2 * M * N * K}
    if kind == "weights":
        return {"bytes": 2 * M * K + _mx_bytes(N, K, how) + o * M * N, "flops": 2 * M * N * K}
    return {"bytes": 2 * M * N + _mx_bytes(N, K, how) + o * M * K, "flops": 2 * M * N * K}


# ---- the definition in 64 bits, written apart from the plain form ----
def _exact_read(q, scales, k):
    """Packed codes and scales -> (R, k) values in 64 bits, from the bits of each code."""
    packed, s = q[0].int(), q[1].int()
    rows = packed.shape[0]
    nibble = torch.empty(rows, 2 * packed.shape[1], dtype=torch.int32, device=packed.device)
    nibble[:, 0::2] = packed & 15
    nibble[:, 1::2] = packed >> 4
    exponent, mantissa = (nibble >> 1) & 3, nibble & 1
    magnitude = torch.where(exponent == 0, mantissa * 0.5, (1 + mantissa * 0.5) * torch.exp2(exponent - 1.0)).double()
    if scales == "tiles":
        s = torch.cat([part for part in s.view(-1, rows, 8)], 1)
    s = s.repeat_interleave(_BLOCK, 1)
    v = torch.where(nibble >= 8, -magnitude, magnitude) * torch.exp2((s - 127).double())
    v[s == 255] = math.nan
    return v[:, :k]


def _exact_round(x, rule):
    """(R, K) -> the nearest values that 4 bits and a scale hold, in 64 bits; block by block."""
    x = x.double()
    rows, k = x.shape
    out = torch.empty_like(x)
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for first in range(0, k, _BLOCK):
        v = x[:, first:first + _BLOCK]
        top = v.abs().max(1, keepdim=True).values
        if rule == "floor":
            e = torch.floor(torch.log2(top.clamp(min=1e-300)))
            e = torch.where(torch.exp2(e) > top, e - 1, e)
            e = torch.where(torch.exp2(e + 1) <= top, e + 1, e) - 2
        else:
            e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 6))
            e = torch.where(6 * torch.exp2(e) < top, e + 1, e)
            e = torch.where(6 * torch.exp2(e - 1) >= top, e - 1, e)
        scale = torch.exp2(e.clamp(-127, 127))
        u = v.abs() / scale
        nearest = torch.zeros_like(u)
        for i in range(7):   # past the middle of two neighbours, or on it where the upper one's code is even
            middle = (grid[i] + grid[i + 1]) / 2
            nearest = torch.where((u >= middle) if i % 2 else (u > middle), torch.full_like(u, grid[i + 1]), nearest)
        r = torch.copysign(nearest * scale, v)
        out[:, first:first + _BLOCK] = torch.where(torch.isfinite(top), r, torch.full_like(r, math.nan))
    return out


def _exact_product(a, b):
    """sum_k a(m,k) b(n,k)"""
    return torch.mm(a.contiguous(), b.t().contiguous())


def exact(case, seed):
    t, kind, how = _inputs(case, seed), case["kind"], case["scales"]
    if kind in ("round", "expand"):
        turned = case["order"] == "r"
        y = _exact_round(t["x"].t() if turned else t["x"], case["rule"]) if kind == "round" else _exact_read(t["x"], how, case["K"])
        return (y.t() if turned else y).reshape(-1)
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "train":
        return {"dx": _exact_product(_exact_round(t["dy"], case["rule"]), _exact_read(t["wt"], how, N)),
                "dw": _exact_product(_exact_round(t["dy"].t(), case["rule"]), _exact_round(t["x"].t(), case["rule"]))}
    w = _exact_read(t["b"], how, K)
    if kind == "product":
        return _exact_product(_exact_read(t["a"], how, K), w)
    if kind == "linear":
        return _exact_product(_exact_round(t["x"], case["rule"]), w)
    return _exact_product(t["a"].double(), w if kind == "weights" else w.t())
