"""Which kernel and tile the products with microscaled 4-bit operands are planned for: a tile asked for is the tile taken wherever its kernel applies (the GPU
tests that ask for tiles would otherwise repeat the default choice), and the default choice where one kernel was measured well ahead of the others."""
import pytest

import paper_2603_02298_amd as lc


def _rows(r, p):
    return "(%d,%d):(%d,1)" % (r, p, p)


def _scales(r, p, tiles):
    return str(lc.lc_mx_scale_layout(r, p // 32)) if tiles else _rows(r, p // 32)


def _plan(M, N, K, a_dtype="mxfp4", tiles=True):
    """Rows of whole blocks; A's rows K elements apart."""
    P = (K + 31) // 32 * 32
    a, a_s = (_rows(M, P), _scales(M, P, tiles)) if a_dtype == "mxfp4" else (_rows(M, K), None)
    return lc.MxGemmPlan(a, a_s, _rows(N, P), _scales(N, P, tiles), _rows(M, N), a_dtype, "f32", False)


def _along_rows(M, N, K, a_dtype):
    """The sum over K of A (M,K) and B stored as K rows of N codes."""
    P = (N + 31) // 32 * 32
    return lc.MxGemmPlan(_rows(M, K), None, "(%d,%d):(1,%d)" % (P, K, P), "(%d,%d):(1,%d)" % (P // 32, K, P // 32), _rows(M, N), a_dtype, "f32", False)


def _words(plan):
    return dict(word.split("=", 1) for word in plan.describe().split(" [")[0].split() if "=" in word)


def _choice(plan):
    words = _words(plan)
    return words["kernel"] + " " + words["tile"]


SIZES = [(1, 1, 128), (1, 40, 160), (16, 16, 128), (65, 130, 288), (129, 200, 544), (300, 260, 2080), (31, 1001, 4128)]
CODES = {16: "direct 16x16", 3216: "direct 32x16", 32: "direct 32x32", 64: "stream 64x64", 12864: "stream 128x64", 128: "stream 128x128", 256: "ring 256x256",
         128128: "ring 128x128"}
MIXED = {16: "direct 16x16", 3216: "direct 32x16", 32: "direct 32x32", 12864: "stream 128x64", 128: "stream 128x128", 256: "wide 256x256", 256128: "wide 256x128",
         128128: "wide 128x128", 128064: "wide 128x64"}


@pytest.mark.parametrize("tile", CODES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_a_tile_asked_for_of_codes(M, N, K, tile, monkeypatch):
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    for tiles in (False, True):
        assert _choice(_plan(M, N, K, tiles=tiles)) == CODES[tile]   # (four blocks of a row and more, their scales neighbours)


@pytest.mark.parametrize("tile", MIXED)
@pytest.mark.parametrize("M,N,K", SIZES + [(1, 1, 8), (2, 17, 104), (17, 64, 520), (200, 129, 640)])
@pytest.mark.parametrize("a_dtype", ["bf16", "f16"])
def test_a_tile_asked_for_beside_16_bits(M, N, K, tile, a_dtype, monkeypatch):
    monkeypatch.setenv("LC_TUNE_MX_TILE", str(tile))
    for tiles in (False, True):
        assert _choice(_plan(M, N, K, a_dtype, tiles)) == MIXED[tile]   # (rows of A begin on 16 bytes)
    if not MIXED[tile].startswith("direct"):
        assert _choice(_along_rows(M, N, K, a_dtype)) == MIXED[tile]
    if MIXED[tile].startswith("stream"):   # what the others do not take
        assert _choice(_plan(M, N, K + 3, a_dtype)) == _choice(_along_rows(M, N, K + 3, a_dtype)) == MIXED[tile]


@pytest.mark.parametrize("M,N,K,want", [
    # us of the choice and of the next: 256 x 4096 x 4096 13.4, 14.7; 1024 x 4096 x 4096 19.3, 20.8; 2048 x 4096 x 4096 28.8, 37.0; 4096 x 8192 x 4096 89, 101; 8192^3 299,
    # 363; 64 x 4096 x 4096 9.8, 13.7; 256^3 4.6, 5.6; 256^2 x 2048 6.0, 7.5
    (256, 4096, 4096, "stream 64x64"), (1024, 4096, 4096, "ring 128x128"), (2048, 4096, 4096, "ring 128x128"), (4096, 8192, 4096, "ring 256x256"),
    (8192, 8192, 8192, "ring 256x256"), (64, 4096, 4096, "direct 32x32"), (256, 256, 256, "stream 64x64"), (256, 256, 2048, "direct 16x16")])
def test_choice_of_codes(M, N, K, want):
    assert _choice(_plan(M, N, K)) == want


@pytest.mark.parametrize("M,N,K", [(1, 8192, 8192), (1, 32768, 8192), (4, 8192, 8192), (16, 8192, 8192), (16, 16384, 4096), (16, 32768, 8192), (32, 8192, 8192), (32, 16384, 8192)])
@pytest.mark.parametrize("a_dtype", ["bf16", "f16"])
def test_few_rows_beside_16_bits_share_out_k(M, N, K, a_dtype):
    """Up to 32 rows: wavefronts share out k, and every CU has a workgroup.  (us, direct and 128 x 64: 1 x 32768 x 8192 28.4, 59; 16 x 32768 x 8192 44.6, 60.6;
    16 x 16384 x 4096 16.4, 31.5; 32 x 16384 x 8192 31.9, 58.)"""
    words = _words(_plan(M, N, K, a_dtype))
    m, n = (int(t) for t in words["tiles"].split("x"))
    assert words["kernel"] == "direct" and words["waves"] == "8" and m * n >= 256


def test_many_rows_beside_16_bits():
    """(us of the choice and of the next: 2048 x 8192 x 4096 116, 144; 3000 x 5000 x 1024 40, 43; along the rows 2048 x 4096 x 4096 82, 92.)"""
    assert _choice(_plan(2048, 8192, 4096, "bf16")) == _choice(_plan(3000, 5000, 1024, "bf16")) == "wide 256x256"
    assert _choice(_along_rows(2048, 4096, 4096, "bf16")) == "wide 256x128"
