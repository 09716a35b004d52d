"""GPU tests of the products by the kernel that takes them: every cut, with scales of every kind, and results into rows
that are further apart than they are long, between values that no one may touch.

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


def widest(m, n, k, out):
    assert vp.vp_fp8_matmul_kernels(m, n, k, vp.VP_OUT_BF16 if out == "bf16" else vp.VP_OUT_F32)[0, 1] == 256


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(4096, 4000, 4096), (8192, 1176, 1024), (8190, 4104, 2048), (300, 8100, 16384)])
@pytest.mark.parametrize("pad,at", [(0, 0), (8, 8), (200, 100), (5, 3)])
def test_widest_tiles_leave_the_neighbouring_columns(m, n, k, pad, at, out):
    """Columns that end inside a tile of 256, as whole 16-byte pieces."""
    widest(m, n, k, out)
    a = vp.fp8_quantize(rand((m, k), 1, spread=0.7))
    b = vp.fp8_quantize(rand((n, k), 2, spread=0.7), 128)
    y = product_between_guards(a, b, out, pad, at)
    if (pad, at) == (5, 3):
        check_product(y[:200], vp.Fp8(a.q[:200], a.scale[:200], k, 1), b, k)
        check_product(y[-200:], vp.Fp8(a.q[-200:], a.scale[-200:], k, 1), b, k)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(130, 38488, 500), (38488, 136, 500), (255, 38400, 2000)])
def test_widest_tiles_of_fewer_rows_than_a_tile(m, n, k, out):
    """One operand has fewer rows than a tile, so that no load past its end lands in the matrix itself."""
    widest(m, n, k, out)
    a = vp.fp8_quantize(rand((m, k), 1, spread=0.7))
    b = vp.fp8_quantize(rand((n, k), 2, spread=0.7), 128)
    check_product(vp.fp8_matmul(a, b, out), a, b, k)


W, T, J = vp.VP_PRODUCT_WAVES, vp.VP_PRODUCT_TILES, vp.VP_PRODUCT_JOIN
#: Sizes, and the kernels that take them: every cut, the widest tiles with a rest of columns, few rows, and pieces.
CUTS = [((7, 201, 300), [(W, 16, 16, 1)]), ((2, 4099, 513), [(W, 16, 32, 1)]), ((130, 1001, 290), [(W, 32, 32, 1)]),
        ((513, 500, 130), [(W, 64, 32, 1)]), ((1200, 1301, 700), [(T, 64, 64, 1)]),
        ((6, 301, 6000), [(T, 64, 64, 12), (J, 0, 0, 12)]), ((66, 24628, 140), [(T, 128, 128, 1)]),
        ((65, 4099, 6000), [(T, 128, 128, 6), (J, 0, 0, 6)]), ((130, 38488, 513), [(T, 256, 256, 1)]),
        ((2100, 4099, 513), [(T, 256, 256, 1), (T, 128, 128, 1)]), ((1000, 4099, 8000), [(T, 256, 256, 3), (J, 0, 0, 3)])]


def scattered(rows, k, block, seed):
    """A matrix in 8 bits whose neighbouring scales differ by up to 2^60; with a scale for each row, one row has an infinity
    in its last block."""
    groups, blocks = R.up(rows, block) // block, R.up(k, 128) // 128
    e = torch.randint(-30, 31, (groups, blocks), generator=torch.Generator().manual_seed(seed)).to(DEV)
    x = rand((rows, k), seed, spread=0.0)
    x *= torch.exp2(e.float()).repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :k]
    if block == 1:
        x[rows // 2, k - 1] = float("inf")
    return vp.fp8_quantize(x, block)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("size,kernels", CUTS)
def test_every_cut(size, kernels, out):
    """Scales of every kind on both sides, rows that are not numbers, results between values that no one may touch."""
    m, n, k = size
    code = vp.VP_OUT_BF16 if out == "bf16" else vp.VP_OUT_F32
    assert [tuple(r) for r in vp.vp_fp8_matmul_kernels(m, n, k, code).tolist()] == kernels
    for ba, bb, pad, at in ((1, 1, 0, 0), (1, 128, 24, 16), (128, 1, 5, 3), (128, 128, 300, 7)):
        a, b = scattered(m, k, ba, m), scattered(n, k, bb, n + 1)
        y = product_between_guards(a, b, out, pad, at)
        nan = torch.zeros((m, n), dtype=torch.bool, device=DEV)
        if ba == 1:
            nan[m // 2] = True
            a.q[m // 2], a.scale[m // 2] = 0, 1
        if bb == 1:
            nan[:, n // 2] = True
            b.q[n // 2], b.scale[n // 2] = 0, 1
        assert torch.equal(torch.isnan(y), nan)
        check_product(torch.where(nan, torch.zeros_like(y), y), a, b, k)
