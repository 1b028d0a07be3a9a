"""Microscaled 4-bit tensors without a GPU: the oracle against the format's own values, plans and their refusals, and every
plan's accesses walked on the host against the buffers."""
import ctypes

import numpy as np
import pytest

import paper_2603_02298_amd as lc
from oracle import mx_oracle as mx


# ---- the oracle ----
def test_oracle_rounds_to_the_nearest_level_with_ties_to_even():
    #        ties: 0.25 0.75 1.25 1.75 2.5 3.5 5.0 go to the even code of the two
    y = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2499, 0.2501, 4.99, 5.01, 7.9, 0.0])
    want = np.array([0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, 0.5, 4.0, 6.0, 6.0, 0.0])
    assert (mx.LEVELS[mx.nearest_codes(y)] == want).all()


@pytest.mark.parametrize("largest,floor,cover", [
    (1.0, 125, 125), (6.0, 127, 127), (6.0001, 127, 128), (4.0, 127, 127), (7.99, 127, 128), (8.0, 128, 128), (3.0, 126, 126), (3.01, 126, 127),
    (0.0, 0, 0), (2.0 ** -149, 0, 0), (3.4e38, 252, 253), (2.0 ** -124, 1, 1), (2.0 ** -125, 0, 0)])
def test_oracle_scales(largest, floor, cover):
    assert mx.scale_bytes(np.array([largest]), "floor")[0] == floor
    assert mx.scale_bytes(np.array([largest]), "cover")[0] == cover


def test_oracle_of_infinities_and_nan():
    x = np.ones((2, 64))
    x[0, 3], x[1, 40] = np.inf, np.nan
    codes, scales = mx.quantize(x, 64, "floor")
    assert scales.tolist() == [[255, 125], [125, 255]] and (codes[0, :32] == 0).all() and (codes[0, 32:] == 6).all()
    v = mx.dequantize(codes, scales)
    assert np.isnan(v[0, :32]).all() and (v[0, 32:] == 1).all()


def test_oracle_offsets_are_the_layout_function():
    for text in ("((2,3),(4,2)):((1,100),(2,50))", "(5,8):(8,1)", "(3,(2,2),2):(40,(1,7),1000)"):
        L, off = lc.Layout(text), mx.offsets(text)
        assert [L(i) for i in range(L.size)] == off.reshape(-1, order="F").tolist()


# ---- plans ----
def _rows(r, p):
    return "(%d,%d):(%d,1)" % (r, p, p), "(%d,%d):(%d,1)" % (r, p // 32, p // 32)


@pytest.mark.parametrize("x,dtype,access", [
    ("(5,96):(96,1)", "bf16", "k-vectors"), ("(5,96):(1,5)", "f32", "row-vectors"), ("(5,96):(1,5)", "bf16", "elements"), ("(5,96):(2,10)", "f32", "elements"),
    ("(5,90):(97,1)", "f16", "k-vectors"), ("((2,4),96):((96,1000),1)", "f32", "k-vectors"), ("((8,2),96):((1,4000),8)", "f16", "row-vectors"),
    ("(16,(16,6)):(96,(1,16))", "bf16", "k-vectors"), ("(16,(16,6)):(16,(1,1600))", "bf16", "elements"), ("(9,96):(-96,1)", "f32", "k-vectors"),
    ("(5,1):(1,1)", "f32", "row-vectors"), ("(1,1):(1,1)", "bf16", "elements")])
def test_access(x, dtype, access):
    L = lc.Layout(x)
    r = {1: 1}.get(L.size) or (8 if "(2,4)" in x else 16 if "(8,2)" in x or x.startswith("(16") else 9 if x.startswith("(9") else 5)
    k = L.size // r
    codes, scales = _rows(r, (k + 31) // 32 * 32)
    for plan in (lc.MxQuantizePlan(x, codes, scales, dtype), lc.MxDequantizePlan(codes, scales, x, dtype)):
        assert "access=" + access in plan.describe(), plan.describe()


def test_scale_layout():
    assert str(lc.lc_mx_scale_layout(5, 16)) == "(5,(8,2)):(8,(1,40))"
    assert str(lc.lc_mx_scale_layout(5, 12)) == "(5,12):(12,1)"
    for rows, blocks in ((3, 8), (7, 40), (1, 1), (4, 9)):
        off = mx.offsets(str(lc.lc_mx_scale_layout(rows, blocks)))
        assert sorted(off.reshape(-1)) == list(range(rows * blocks))
    h = ctypes.c_void_p()
    assert lc.lib().lc_mx_scale_layout(0, 4, ctypes.byref(h)) == 4 and lc.lib().lc_mx_scale_layout(4, 1 << 31, ctypes.byref(h)) == 14
    assert lc.lib().lc_mx_scale_layout(4, 4, None) == 1 and not h


@pytest.mark.parametrize("x,codes,scales,dtype,status", [
    ("(4,96):(96,1)", "(4,80):(80,1)", "(4,3):(3,1)", "f32", "SIZE_MISMATCH"),               # not whole blocks
    ("(4,96):(96,1)", "(4,96):(96,1)", "(4,4):(4,1)", "f32", "SIZE_MISMATCH"),               # scales of another size
    ("(4,96):(96,1)", "(5,96):(96,1)", "(5,3):(3,1)", "f32", "SIZE_MISMATCH"),               # rows
    ("(4,97):(97,1)", "(4,96):(96,1)", "(4,3):(3,1)", "f32", "SIZE_MISMATCH"),               # K beyond the blocks
    ("(4,96):(96,1)", "(4,96):(100,1)", "(4,3):(3,1)", "f32", "BLOCK_LAYOUT"),               # rows off the 16-byte grid
    ("(4,96):(96,1)", "(4,96):(1,4)", "(4,3):(3,1)", "f32", "BLOCK_LAYOUT"),                 # blocks not contiguous
    ("(4,96):(96,1)", "(4,(16,6)):(96,(1,32))", "(4,3):(3,1)", "f32", "BLOCK_LAYOUT"),
    ("(4,96):(96,1)", "(4,(32,3)):(96,(1,48))", "(4,3):(3,1)", "f32", "BLOCK_LAYOUT"),
    ("(4,96):(96,1)", "(4,96):(-96,1)", "(4,3):(3,1)", "f32", "NEGATIVE_STRIDE"),
    ("(4,96):(96,1)", "(4,96):(96,1)", "(4,3):(3,-1)", "f32", "NEGATIVE_STRIDE"),
    ("(4,96):(96,1)", "(4,96):(0,1)", "(4,3):(3,1)", "f32", "DST_ALIASES"),
    ("(4,96):(96,1)", "(4,96):(64,1)", "(4,3):(3,1)", "f32", "DST_ALIASES"),
    ("(4,96):(96,1)", "(4,96):(96,1)", "(4,3):(2,1)", "f32", "DST_ALIASES"),
    ("(4,96):(96,1)", "(4,96):(96,1)", "(4,3):(3,1)", "b16", "UNSUPPORTED_DTYPE"),
    ("(4,96,1):(96,1,0)", "(4,96):(96,1)", "(4,3):(3,1)", "f32", "INVALID_ARG"),
    ("384:1", "(4,96):(96,1)", "(4,3):(3,1)", "f32", "INVALID_ARG"),
    ("(4,96):(96,1)", "(4,96,1):(96,1,0)", "(4,3):(3,1)", "f32", "INVALID_ARG"),
    ("(4,96):(96,1)", "(4,96):(96,1)", "12:1", "f32", "INVALID_ARG"),
    ("((2,2,2,2,2),96):((1,4,16,64,1000),4096)", "(32,96):(96,1)", "(32,3):(3,1)", "f32", "TOO_LARGE"),   # five leaves
    ("(1073741824,96):(96,1)", "(1073741824,96):(96,1)", "(1073741824,3):(3,1)", "f32", "TOO_LARGE"),     # 2^31 blocks and more
])
def test_quantize_refusals(x, codes, scales, dtype, status):
    with pytest.raises(lc.LayoutCopyError) as e:
        lc.MxQuantizePlan(x, codes, scales, dtype)
    assert e.value.status_name == status


def test_dequantize_refusals_and_what_it_takes():
    codes, scales = _rows(4, 96)
    for dst, status in (("(4,96):(0,1)", "DST_ALIASES"), ("(4,96):(50,1)", "DST_ALIASES"), ("(4,100):(100,1)", "SIZE_MISMATCH"), ("(3,96):(96,1)", "SIZE_MISMATCH")):
        with pytest.raises(lc.LayoutCopyError) as e:
            lc.MxDequantizePlan(codes, scales, dst, "bf16")
        assert e.value.status_name == status
    lc.MxDequantizePlan("(4,96):(0,1)", "(4,3):(0,0)", "(4,96):(96,1)", "bf16")   # codes and scales that rows share are read only
    lc.MxDequantizePlan(codes, scales, "(4,96):(-96,-1)", "bf16")


def test_null_arguments_wrong_directions_and_misaligned_pointers():
    L = lc.lib()
    x, (codes, scales) = lc.Layout("(4,96):(96,1)"), (lc.Layout(t) for t in _rows(4, 96))
    h = ctypes.c_void_p()
    assert L.lc_mx_quantize_plan_create(None, codes._h, scales._h, 0, 0, ctypes.byref(h)) == 1
    assert L.lc_mx_quantize_plan_create(x._h, codes._h, scales._h, 0, 0, None) == 1
    assert L.lc_mx_quantize_plan_create(x._h, codes._h, scales._h, 0, 2, ctypes.byref(h)) == 1   # no such rule
    assert L.lc_mx_dequantize_plan_create(codes._h, None, x._h, 0, ctypes.byref(h)) == 1 and not h
    assert L.lc_mx_plan_describe(None, None, 0, None) == 1
    q, d = lc.MxQuantizePlan(x, codes, scales, "f32"), lc.MxDequantizePlan(codes, scales, x, "f32")
    # refused before anything is launched: addresses that are never touched
    assert L.lc_mx_quantize_plan_execute(None, 256, 256, 256, None) == 1
    assert L.lc_mx_quantize_plan_execute(q._h, None, 256, 256, None) == 1
    assert L.lc_mx_quantize_plan_execute(d._h, 256, 256, 256, None) == 1
    assert L.lc_mx_dequantize_plan_execute(q._h, 256, 256, 256, None) == 1
    assert L.lc_mx_quantize_plan_execute(q._h, 258, 256, 256, None) == 15
    assert L.lc_mx_quantize_plan_execute(q._h, 256, 264, 256, None) == 15
    assert L.lc_mx_dequantize_plan_execute(d._h, 256, 256, 258, None) == 15
    assert L.lc_mx_quantize(None, x._h, 256, codes._h, 256, scales._h, 0, 0, None) == 1
    assert L.lc_mx_dequantize(256, codes._h, 256, scales._h, 256, None, 0, None) == 1
    assert L.lc_dtype_bytes(8) == 0
    assert L.lc_plan_create(x._h, x._h, 8, 256, 256, ctypes.byref(h)) == 13


WALKS = [(1, 1), (1, 31), (3, 32), (5, 33), (8, 64), (17, 100), (33, 255), (64, 256), (65, 1000), (130, 2048), (300, 40), (2, 4100)]


@pytest.mark.parametrize("R,K", WALKS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["k", "r", "strided", "reversed"])
@pytest.mark.parametrize("tiles", [False, True])
def test_every_access_lies_inside_and_every_byte_is_written_once(R, K, dtype, order, tiles):
    P = (K + 255) // 256 * 256 if tiles else (K + 31) // 32 * 32
    es = lc.DTYPE_BYTES[dtype]
    x = {"k": "(%d,%d):(%d,1)" % (R, K, K + 3), "r": "(%d,%d):(1,%d)" % (R, K, R + 1), "strided": "(%d,%d):(%d,3)" % (R, K, 3 * K),
         "reversed": "(%d,%d):(%d,-1)" % (R, K, K)}[order]
    codes = "(%d,%d):(%d,1)" % (R, P, P + 32)
    scales = str(lc.lc_mx_scale_layout(R, P // 32))
    X, Q, S = lc.Layout(x), lc.Layout(codes), lc.Layout(scales)
    before, behind = -X.min_offset * es, X.cosize * es
    q = lc.MxQuantizePlan(x, codes, scales, dtype)
    reads, written = q.debug_walk_on_host(before, behind, Q.cosize // 2, S.cosize)
    assert written == R * P // 2 + R * P // 32 and reads >= R * K * es
    d = lc.MxDequantizePlan(codes, scales, x, dtype)
    reads, written = d.debug_walk_on_host(before, behind, Q.cosize // 2, S.cosize)
    assert written == R * K * es
    # a buffer that is one byte short is noticed
    with pytest.raises(lc.LayoutCopyError):
        q.debug_walk_on_host(before, behind, Q.cosize // 2, S.cosize - 1)
    with pytest.raises(lc.LayoutCopyError):
        d.debug_walk_on_host(before, behind - 1, Q.cosize // 2, S.cosize)


# ---- products ----
def _gemm(a, a_s, b, b_s, c, a_dtype="mxfp4", c_dtype="f32", **more):
    return lc.MxGemmPlan(a, a_s, b, b_s, c, a_dtype, c_dtype, **more)


@pytest.mark.parametrize("a,a_s,b,b_s,c,a_dtype,c_dtype,status", [
    ("(4,96):(96,1)", "(4,3):(3,1)", "(5,96):(96,1)", "(5,3):(3,1)", "(4,6):(6,1)", "mxfp4", "f32", "SIZE_MISMATCH"),       # N
    ("(4,96):(96,1)", "(4,3):(3,1)", "(5,64):(64,1)", "(5,2):(2,1)", "(4,5):(5,1)", "mxfp4", "f32", "SIZE_MISMATCH"),       # K
    ("(4,96):(96,1)", "(4,3):(3,1)", "(5,96):(96,1)", "(5,3):(3,1)", "(3,5):(5,1)", "mxfp4", "f32", "SIZE_MISMATCH"),       # M
    ("(4,96):(96,1)", "(4,2):(2,1)", "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "mxfp4", "f32", "SIZE_MISMATCH"),       # A's scales
    ("(4,96):(96,1)", "(4,3):(3,1)", "(5,96):(96,1)", "(4,3):(3,1)", "(4,5):(5,1)", "mxfp4", "f32", "SIZE_MISMATCH"),       # B's scales
    ("(4,96):(96,1)", "(4,3):(3,1)", "(32,96):(1,32)", "(1,96):(1,1)", "(4,32):(32,1)", "mxfp4", "f32", "SIZE_MISMATCH"),   # codes by codes blocked along the rows
    ("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "mxfp4", "f32", "INVALID_ARG"),                  # no scales
    ("(4,96):(96,1)", "(4,3):(3,1)", "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "INVALID_ARG"),          # scales for 16 bits
    ("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "f32", "f32", "UNSUPPORTED_DTYPE"),
    ("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "b16", "UNSUPPORTED_DTYPE"),
    ("(4,97):(97,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "SIZE_MISMATCH"),                 # K beyond B's
    ("(4,97):(97,1)", None, "(96,97):(1,96)", "(3,97):(1,3)", "(4,97):(97,1)", "bf16", "f32", "SIZE_MISMATCH"),             # N beyond B's
    ("(4,96):(96,1)", None, "(96,97):(1,96)", "(3,97):(1,3)", "(4,90):(90,1)", "bf16", "f32", "SIZE_MISMATCH"),             # K differs
    ("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(0,1)", "bf16", "f32", "DST_ALIASES"),
    ("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(4,1)", "bf16", "f32", "DST_ALIASES"),
    ("(4,96):(-96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "NEGATIVE_STRIDE"),
    ("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,-1)", "bf16", "f32", "NEGATIVE_STRIDE"),
    ("(4,96):(96,1)", None, "(5,96):(98,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "BLOCK_LAYOUT"),
    ("(4,96):(96,1)", None, "(5,96):(1,5)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "BLOCK_LAYOUT"),
    ("(4,96,2):(96,1,384)", None, "(5,96,2):(96,1,500)", "(5,3,2):(3,1,15)", "(4,5,2):(5,1,20)", "bf16", "f32", "BLOCK_LAYOUT"),   # a batch off the grid
    ("(4,96,2):(96,1,384)", None, "(5,96,3):(96,1,480)", "(5,3,3):(3,1,15)", "(4,5,2):(5,1,20)", "bf16", "f32", "SIZE_MISMATCH"),
    ("(4,96,2):(96,1,384)", None, "(5,96,2):(96,1,480)", "(5,3,1):(3,1,15)", "(4,5,2):(5,1,20)", "bf16", "f32", "SIZE_MISMATCH"),
    ("(4,96,2):(96,1,384)", None, "(5,96,2):(96,1,480)", "(5,3,2):(3,1,15)", "(4,5,2):(5,1,10)", "bf16", "f32", "DST_ALIASES"),
    ("(4,96):(96,1)", None, "(5,96,2):(96,1,480)", "(5,3,2):(3,1,15)", "(4,5):(5,1)", "bf16", "f32", "INVALID_ARG"),
    ("(4,96,2):(96,1,384)", None, "(5,96,2):(96,1,480)", "(5,3):(3,1)", "(4,5,2):(5,1,20)", "bf16", "f32", "INVALID_ARG"),
    ("384:1", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "INVALID_ARG"),
    ("(4,96):(1073741824,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "TOO_LARGE"),
    ("(4,96):(96,1)", None, "(5,96):(4294967296,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", "TOO_LARGE"),
])
def test_gemm_refusals(a, a_s, b, b_s, c, a_dtype, c_dtype, status):
    with pytest.raises(lc.LayoutCopyError) as e:
        _gemm(a, a_s, b, b_s, c, a_dtype, c_dtype)
    assert e.value.status_name == status


def test_gemm_alignments_and_null_arguments():
    for more, status in (({"b_align": 8}, "MISALIGNED"), ({"a_align": 1}, "MISALIGNED"), ({"c_align": 2}, "MISALIGNED"), ({"a_align": 24}, "INVALID_ARG"),
                         ({"a_align": 0}, "INVALID_ARG")):
        with pytest.raises(lc.LayoutCopyError) as e:
            _gemm("(4,96):(96,1)", None, "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", "bf16", "f32", **more)
        assert e.value.status_name == status
    with pytest.raises(lc.LayoutCopyError) as e:
        _gemm("(4,96):(96,1)", "(4,3):(3,1)", "(5,96):(96,1)", "(5,3):(3,1)", "(4,5):(5,1)", a_align=8)
    assert e.value.status_name == "MISALIGNED"
    L = lc.lib()
    mixed = _gemm("(4,96):(96,1)", None, "(8,96):(96,1)", "(8,3):(3,1)", "(4,8):(8,1)", "bf16", "f32")
    codes = _gemm("(4,96):(96,1)", "(4,3):(3,1)", "(8,96):(96,1)", "(8,3):(3,1)", "(4,8):(8,1)")
    assert mixed.flops == codes.flops == 2 * 4 * 8 * 96
    # refused before anything is launched: addresses that are never touched
    assert L.lc_mx_gemm_plan_execute(None, 256, None, 256, 256, 256, None) == 1
    assert L.lc_mx_gemm_plan_execute(mixed._h, 256, 256, 256, 256, 256, None) == 1   # scales for 16-bit elements
    assert L.lc_mx_gemm_plan_execute(codes._h, 256, None, 256, 256, 256, None) == 1
    assert L.lc_mx_gemm_plan_execute(mixed._h, 256, None, 256, 256, None, None) == 1
    assert L.lc_mx_gemm_plan_execute(mixed._h, 258, None, 256, 256, 256, None) == 15   # planned for 16-byte vectors
    assert L.lc_mx_gemm_plan_execute(mixed._h, 256, None, 264, 256, 256, None) == 15
    assert L.lc_mx_gemm_plan_execute(mixed._h, 256, None, 256, 256, 260, None) == 15
    assert L.lc_mx_gemm_plan_execute(codes._h, 264, 256, 256, 256, 256, None) == 15
    assert L.lc_mx_gemm_plan_flops(None) == -1 and L.lc_mx_gemm_plan_describe(None, None, 0, None) == 1
    ms = ctypes.c_float()
    assert L.lc_mx_gemm_plan_time(mixed._h, 256, None, 256, 256, 256, 0, 0, None, ctypes.byref(ms)) == 1
    a, b, s, c = (lc.Layout(t) for t in ("(4,96):(96,1)", "(8,96):(96,1)", "(8,3):(3,1)", "(4,8):(8,1)"))
    assert L.lc_mx_gemm(256, a._h, None, None, 256, b._h, 256, s._h, None, c._h, 2, 0, 0, None) == 1
    assert L.lc_mx_gemm(256, a._h, 256, None, 256, b._h, 256, s._h, 256, c._h, 2, 0, 0, None) == 1
    assert L.lc_mx_gemm(256, a._h, None, None, 264, b._h, 256, s._h, 256, c._h, 2, 0, 0, None) == 15


@pytest.mark.parametrize("a,a_dtype,load", [
    ("(40,320):(320,1)", "bf16", "load=k-vectors "), ("(40,317):(320,1)", "bf16", "load=unaligned-k-vectors"), ("(40,320):(321,1)", "f16", "load=unaligned-k-vectors"),
    ("(40,320):(1,40)", "bf16", "load=elements"), ("(40,(8,40)):(8,(1,320))", "bf16", "load=elements"), ("(40,7):(7,1)", "bf16", "load=elements")])
def test_gemm_loads(a, a_dtype, load):
    k = lc.Layout(a).size // 40
    p = (k + 31) // 32 * 32
    codes, scales = _rows(50, p)
    assert load in _gemm(a, None, codes, scales, "(40,50):(50,1)", a_dtype).describe()
