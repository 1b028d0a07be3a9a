"""The checks of the tensor helpers of rotary positions, the 4-bit cache and the attention over it, without a GPU: stand-ins for GPU tensors, and the C call behind each helper
replaced by a recorder."""
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
    made = []
    for name in ("lc_rope", "lc_mx_cache_write", "lc_mx_cache_read"):
        monkeypatch.setattr(binding, name, lambda *args, name=name: made.append(name))
    monkeypatch.setattr(lc.MxAttentionPlan, "execute", lambda *args: made.append("execute"))

    class Stream:
        cuda_stream = 0

    monkeypatch.setattr(torch.cuda, "current_stream", lambda *args: Stream)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    return made


U8, BF16, I32 = torch.uint8, torch.bfloat16, torch.int32
ROWS, CODES, SCALES = "(4,2,64):(128,64,1)", "(32,2,64):(128,64,1)", "(32,2,2):(4,2,1)"


def _plan():
    return lc.MxAttentionPlan(ROWS, CODES, SCALES, ROWS, "bf16", sequences=2, page=16, pages_per_sequence=1, max_queries=3, scale=1.0)


def _cache():
    return dict(k_codes=_tensor(32, 64, dtype=U8), v_codes=_tensor(32, 64, dtype=U8), codes_layout=CODES, k_scales=_tensor(32, 4, dtype=U8), v_scales=_tensor(32, 4, dtype=U8), scales_layout=SCALES,
                k=_tensor(4, 128, dtype=BF16), v=_tensor(4, 128, dtype=BF16), x_layout=ROWS, slots=_tensor(4, dtype=I32))


# helper, its arguments with every tensor as large as its layout, and those that are arrays of numbers
CALLS = {
    "rope": (lc.rope_tensor, lambda: dict(x=_tensor(4, 128), x_layout=ROWS, positions=_tensor(4, dtype=I32), frequencies=_tensor(32), y=_tensor(4, 128), y_layout=ROWS, rotary=64),
             ("positions", "frequencies")),
    "write": (lc.mx_cache_write_tensor, _cache, ("slots",)),
    "read": (lc.mx_cache_read_tensor, _cache, ("slots",)),
    "attention": (lc.mx_attention_tensor, lambda: dict(plan=_plan(), q=_tensor(4, 128, dtype=BF16), k_codes=_tensor(32, 64, dtype=U8), k_scales=_tensor(32, 4, dtype=U8),
                                                       v_codes=_tensor(32, 64, dtype=U8), v_scales=_tensor(32, 4, dtype=U8), lengths=_tensor(2, dtype=I32),
                                                       o=_tensor(4, 128, dtype=BF16), pages=_tensor(2, 1, dtype=I32), starts=_tensor(3, dtype=I32), lse=_tensor(4, 2)),
                  ("lengths", "pages", "starts", "lse")),
}
EACH = [(call, key) for call, (_, args, _) in CALLS.items() for key, t in args().items() if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("call", CALLS)
def test_tensors_as_large_as_their_layouts(call, calls):
    helper, args, _ = CALLS[call]
    helper(**args())
    assert len(calls) == 1


@pytest.mark.parametrize("call,key", EACH)
def test_what_is_too_small_or_elsewhere(call, key, calls):
    helper, args, arrays = CALLS[call]
    args = args()
    t = args[key]
    short = t.reshape(-1)[:-1] if key in arrays else t[:1].expand(t.shape)   # an array that ends early; one row that stands for all of them
    with pytest.raises(ValueError):
        helper(**dict(args, **{key: short}))
    with pytest.raises(RuntimeError, match="needs GPU tensors"):
        helper(**dict(args, **{key: t.as_subclass(torch.Tensor)}))
    if key in arrays:
        with pytest.raises(ValueError):
            helper(**dict(args, **{key: t.double()}))
        with pytest.raises(ValueError):
            helper(**dict(args, **{key: torch.cat([t.reshape(-1), t.reshape(-1)])[::2]}))
    else:
        with pytest.raises(ValueError):
            helper(**dict(args, **{key: t.to(torch.int16)}))
    assert calls == []


@pytest.mark.parametrize("call", ["write", "read"])
def test_a_second_tensor_comes_whole(call, calls):
    helper, args, _ = CALLS[call]
    helper(**dict(args(), v=None, v_codes=None, v_scales=None))
    for some in (("v",), ("v_codes",), ("v", "v_scales")):
        with pytest.raises(ValueError, match="all or none"):
            helper(**dict(args(), **{key: None for key in some}))
    with pytest.raises(ValueError, match="one type"):
        helper(**dict(args(), v=_tensor(4, 128)))
    assert len(calls) == 1


@pytest.mark.parametrize("call,origin,key", [("rope", "x_origin", "x"), ("rope", "y_origin", "y"), ("write", "x_origin", "k"), ("attention", "q_origin", "q"), ("attention", "o_origin", "o")])
def test_origins(call, origin, key, calls):
    """Offset 0 may lie inside the tensor, as far as what the layout reaches does."""
    helper, args, _ = CALLS[call]
    for at in (1, -1):
        with pytest.raises(ValueError, match="cover"):
            helper(**dict(args(), **{origin: at}))
    assert calls == []


def test_what_a_plan_is_not_for(calls):
    helper, args, _ = CALLS["attention"]
    for key in ("q", "o"):
        with pytest.raises(ValueError, match="types"):
            helper(**dict(args(), **{key: _tensor(4, 128, dtype=torch.float16)}))
    with pytest.raises(ValueError, match="tokens, heads"):
        lc.rope_tensor(**dict(CALLS["rope"][1](), x_layout="(4,128):(128,1)"))
    with pytest.raises(ValueError, match="one type"):
        lc.rope_tensor(**dict(CALLS["rope"][1](), y=_tensor(4, 128, dtype=BF16)))
    helper(**dict(args(), pages=None, starts=None, lse=None))
    assert len(calls) == 1
