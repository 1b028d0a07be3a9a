"""The tensor helpers' checks without a GPU: stand-ins for GPU tensors, and the C call behind each helper replaced by a recorder."""
import contextlib

import pytest

import paper_2603_02298_amd as lc
from paper_2603_02298_amd import binding

torch = pytest.importorskip("torch")


class OnGpu(torch.Tensor):
    """A host tensor, and any view of it, that says it is on a GPU."""
    is_cuda = True


def _tensor(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    """The names of the C calls that the helpers made."""
    made = []
    for name in ("lc_copy", "lc_gemm", "lc_mx_quantize", "lc_mx_dequantize", "lc_mx_gemm"):
        monkeypatch.setattr(binding, name, lambda *args, name=name, **more: made.append(name))

    class Stream:
        cuda_stream = 0

    monkeypatch.setattr(torch.cuda, "current_stream", lambda *args: Stream)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    return made


U8, BF16 = torch.uint8, torch.bfloat16
# helper, its arguments with every tensor as large as its layout
CALLS = {
    "copy": (lc.copy_tensor, dict(src=_tensor(4, 96), src_layout="(4,96):(96,1)", dst=_tensor(4, 96), dst_layout="(4,96):(96,1)")),
    "gemm": (lc.gemm_tensor, dict(a=_tensor(4, 96, dtype=BF16), a_layout="(4,96):(96,1)", b=_tensor(5, 96, dtype=BF16), b_layout="(5,96):(96,1)", c=_tensor(4, 5),
                                  c_layout="(4,5):(5,1)")),
    "quantize": (lc.mx_quantize_tensor, dict(src=_tensor(4, 96), src_layout="(4,96):(96,1)", codes=_tensor(4, 48, dtype=U8), codes_layout="(4,96):(96,1)",
                                             scales=_tensor(4, 3, dtype=U8), scales_layout="(4,3):(3,1)")),
    "dequantize": (lc.mx_dequantize_tensor, dict(codes=_tensor(4, 48, dtype=U8), codes_layout="(4,96):(96,1)", scales=_tensor(4, 3, dtype=U8),
                                                 scales_layout="(4,3):(3,1)", dst=_tensor(4, 96), dst_layout="(4,96):(96,1)")),
    "product of codes": (lc.mx_gemm_tensor, dict(a=_tensor(4, 48, dtype=U8), a_layout="(4,96):(96,1)", a_scales=_tensor(4, 3, dtype=U8), a_scales_layout="(4,3):(3,1)",
                                                 b=_tensor(5, 48, dtype=U8), b_layout="(5,96):(96,1)", b_scales=_tensor(5, 3, dtype=U8),
                                                 b_scales_layout="(5,3):(3,1)", c=_tensor(4, 5), c_layout="(4,5):(5,1)")),
    "product": (lc.mx_gemm_tensor, dict(a=_tensor(4, 96, dtype=BF16), a_layout="(4,96):(96,1)", a_scales=None, a_scales_layout=None, b=_tensor(5, 48, dtype=U8),
                                        b_layout="(5,96):(96,1)", b_scales=_tensor(5, 3, dtype=U8), b_scales_layout="(5,3):(3,1)", c=_tensor(4, 5),
                                        c_layout="(4,5):(5,1)")),
}
EACH = [(call, key) for call, (_, args) in CALLS.items() for key, t in args.items() if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("call", CALLS)
def test_tensors_as_large_as_their_layouts(call, calls):
    helper, args = CALLS[call]
    helper(**args)
    assert len(calls) == 1


@pytest.mark.parametrize("call,key", EACH)
def test_a_view_that_repeats_its_memory_covers_only_that(call, key, calls):
    """One row expanded to all of them has as many elements as the layout, in a row's worth of memory."""
    helper, args = CALLS[call]
    t = args[key]
    with pytest.raises(ValueError, match="cover|smaller"):
        helper(**dict(args, **{key: t[:1].expand(t.shape)}))
    assert calls == []


@pytest.mark.parametrize("call,key", EACH)
def test_a_view_with_gaps_covers_them(call, key, calls):
    """A matrix whose rows are part of wider ones, under the layout of just that: its elements are fewer than the layout's cosize, its memory is not.  A
    row less does not do."""
    helper, args = CALLS[call]
    t = args[key]
    unit = 2 if t.dtype == U8 and "scales" not in key else 1   # codes: two to a byte
    wide = torch.zeros(t.shape[0], t.shape[1] + 16, dtype=t.dtype).as_subclass(OnGpu)[:, :t.shape[1]]
    layout = "(%d,%d):(%d,1)" % (t.shape[0], unit * t.shape[1], unit * wide.stride(0))
    helper(**dict(args, **{key: wide, key + "_layout": layout}))
    assert len(calls) == 1
    with pytest.raises(ValueError, match="cover|smaller"):
        helper(**dict(args, **{key: wide[:-1], key + "_layout": layout}))
    assert len(calls) == 1


@pytest.mark.parametrize("call,key", EACH)
def test_other_orders_of_the_same_memory_and_empty_tensors(call, key, calls):
    helper, args = CALLS[call]
    t = args[key]
    helper(**dict(args, **{key: torch.zeros(t.shape[1], t.shape[0], dtype=t.dtype).as_subclass(OnGpu).t()}))
    assert len(calls) == 1
    with pytest.raises(ValueError, match="cover|smaller"):
        helper(**dict(args, **{key: t[:0]}))
    assert len(calls) == 1


def test_scales_and_their_layout_come_together(calls):
    """A layout without scales, or scales without a layout, is refused as the C call refuses it, not left out."""
    for call, change in (("product", dict(a_scales_layout="(4,3):(3,1)")), ("product of codes", dict(a_scales=None)), ("product of codes", dict(a_scales_layout=None))):
        helper, args = CALLS[call]
        with pytest.raises(ValueError, match="a_scales and a_scales_layout"):
            helper(**dict(args, **change))
    assert calls == []
