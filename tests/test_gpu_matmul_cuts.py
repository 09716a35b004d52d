"""GPU tests of the products by the kernel that takes them: results into rows that are further apart than they are
long, between values that no one may touch.

Tolerances are those of test_gpu_fp8.py.
"""
import pytest
import torch

import fp8_reference as R
import paper_2604_16893_amd as vp
from test_gpu_fp8 import DEV, TYPES, check_product, rand

pytestmark = pytest.mark.gpu


def product_between_guards(a, b, out, pad, at, rows=1):
    """fp8_matmul's result, checked to be the same inside a wider buffer whose other values stay as they were.  The last
    row's padding is not there: the buffer ends with the result."""
    m, n, k = a.rows, b.rows, a.cols
    ld = n + pad
    flat = torch.full((rows * ld + at + (m - 1) * ld + n,), 7.0, dtype=TYPES[out], device=DEV)
    tail = torch.full((1 << 16,), 7.0, dtype=TYPES[out], device=DEV)      # (what the allocator puts next, most likely)
    view = flat[rows * ld + at:].as_strided((m, n), (ld, 1))
    code = vp.VP_OUT_BF16 if out == "bf16" else vp.VP_OUT_F32
    size = vp.vp_fp8_matmul_workspace(m, n, k, code)
    vp.vp_fp8_matmul(a, b, view, torch.empty(max(size, 16), dtype=torch.uint8, device=DEV))
    y = vp.fp8_matmul(a, b, out)
    assert torch.equal(view.nan_to_num(nan=3.0), y.nan_to_num(nan=3.0))
    view.fill_(7.0)
    assert (flat == 7).all() and (tail == 7).all()
    return y


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(4096, 4000, 4096), (8192, 1176, 1024), (8190, 4104, 2048), (300, 8100, 16384)])
@pytest.mark.parametrize("pad,at", [(0, 0), (8, 8), (200, 100), (5, 3)])
def test_widest_tiles_leave_the_neighbouring_columns(m, n, k, pad, at, out):
    """Columns that end inside a tile of 256, as whole 16-byte pieces."""
    a = vp.fp8_quantize(rand((m, k), 1, spread=0.7))
    b = vp.fp8_quantize(rand((n, k), 2, spread=0.7), 128)
    y = product_between_guards(a, b, out, pad, at)
    if (pad, at) == (5, 3):
        check_product(y[:200], vp.Fp8(a.q[:200], a.scale[:200], k, 1), b, k)
        check_product(y[-200:], vp.Fp8(a.q[-200:], a.scale[-200:], k, 1), b, k)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(130, 38488, 500), (38488, 130, 500), (255, 38400, 2000)])
def test_widest_tiles_of_fewer_rows_than_a_tile(m, n, k, out):
    """One operand has fewer rows than a tile, so that no load past its end lands in the matrix itself."""
    a = vp.fp8_quantize(rand((m, k), 1, spread=0.7))
    b = vp.fp8_quantize(rand((n, k), 2, spread=0.7), 128)
    check_product(vp.fp8_matmul(a, b, out), a, b, k)
