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
