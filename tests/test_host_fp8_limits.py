"""CPU tests of the largest sizes that the 8-bit operators take: what is refused is refused as a size."""
import ctypes

import pytest

import paper_2604_16893_amd as vp
from paper_2604_16893_amd import fp8
from test_host_fp8 import P, held, refused

BIG = vp.VP_MAX_DIM


def workspace(m, n, k, dtype=1):
    b = ctypes.c_int64(-1)
    return fp8._entry("vp_fp8_matmul_workspace")(m, n, k, dtype, ctypes.byref(b)), b.value


def test_products_of_the_largest_sizes():
    for m, n, k in ((BIG, 1, 1), (1, BIG, 1), (BIG, 128, 0), (1 << 19, 1 << 18, 128), (1, 1, vp.VP_MAX_SUM),
                    (5000, 5000, vp.VP_MAX_SUM)):
        for dtype in (0, 1):
            status, size = workspace(m, n, k, dtype)
            assert status == vp.VP_OK and size >= 0
    for m, n, k in ((BIG, 129, 1), (BIG, BIG, 0), (1 << 20, 1 << 19, 128), (1 << 19, 1 << 19, 1 << 25)):
        for dtype in (0, 1):
            assert workspace(m, n, k, dtype)[0] == vp.VP_ERR_DIMS and vp.lib().vp_last_error_message()
        assert refused("vp_fp8_matmul", held(m, k), held(n, k, 128), P, 1, n, P, 1 << 62, 0) == vp.VP_ERR_DIMS


def test_conversions_of_too_many_tiles():
    many = 1 << 24      # rows and columns: 2^17 tiles of 128 each way
    for call in (("vp_fp8_quantize", P, 1, many, many, many, held(many, many, 128), None, 0),
                 ("vp_fp8_quantize", P, 1, many, many, many, None, held(many, many), 0),
                 ("vp_fp8_transpose", held(many, many), held(many, many), 0)):
        assert refused(*call) == vp.VP_ERR_DIMS


def test_a_refused_workspace_raises():
    with pytest.raises(vp.VPError):
        vp.vp_fp8_matmul_workspace(BIG, BIG, 128)


def test_the_kernels_of_a_product():
    for dtype in (vp.VP_OUT_BF16, vp.VP_OUT_F32):
        assert vp.vp_fp8_matmul_kernels(0, 5, 128, dtype).shape == (0, 4)
        kinds = {int(r[0]) for s in ((1, 4096, 4096), (8192, 8192, 8192), (300, 8192, 16384))
                 for r in vp.vp_fp8_matmul_kernels(*s, dtype)}
        assert kinds == {vp.VP_PRODUCT_TILES, vp.VP_PRODUCT_WAVES, vp.VP_PRODUCT_JOIN}
        # pieces take workspace, and a result whose rows are too far apart for the widest tiles goes to the next ones
        for m, n, k in ((300, 8192, 16384), (77, 1001, 1176), (8192, 8192, 8192), (6, 301, 6000)):
            rows = vp.vp_fp8_matmul_kernels(m, n, k, dtype)
            assert (rows[0, 3] > 1) == (vp.vp_fp8_matmul_workspace(m, n, k, dtype) > 0)
        assert vp.vp_fp8_matmul_kernels(8192, 8192, 8192, dtype, 1 << 21).tolist() == [[vp.VP_PRODUCT_TILES, 128, 128, 1]]
    count, rows = ctypes.c_int32(-1), (ctypes.c_int32 * 8)(*[-7] * 8)
    call = fp8._entry("vp_fp8_matmul_kernels")
    assert call(300, 8192, 16384, 1, 8192, rows, 1, ctypes.byref(count)) == vp.VP_OK
    assert count.value == 2 and rows[0] == vp.VP_PRODUCT_TILES and list(rows)[4:] == [-7] * 4
    assert refused("vp_fp8_matmul_kernels", 1, 1, 1, 1, 1, None, 0, None) == vp.VP_ERR_NULL
    for m, n, k, dtype, ld, buf, capacity, status in ((1, 5, 1, 1, 4, rows, 2, vp.VP_ERR_ARG), (1, 5, 1, 1, 5, None, 2, vp.VP_ERR_ARG),
                                                      (1, 5, 1, 1, 5, rows, -1, vp.VP_ERR_ARG), (1, 5, 1, 4, 5, rows, 2, vp.VP_ERR_ARG),
                                                      (-1, 5, 1, 1, 5, rows, 2, vp.VP_ERR_DIMS), (BIG, BIG, 1, 1, BIG, rows, 2, vp.VP_ERR_DIMS)):
        assert refused("vp_fp8_matmul_kernels", m, n, k, dtype, ld, buf, capacity, ctypes.byref(count)) == status
