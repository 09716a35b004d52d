"""GPU tests of matrices in 8 bits at the ends of their range: values that f32 does not hold, scales of 1, 254 and 255.

What moves by powers of two is equal exactly; products have the tolerances of test_gpu_fp8.py.
"""
import pytest
import torch

import fp8_reference as R
import paper_2604_16893_amd as vp
from test_gpu_fp8 import DEV, check_product, same

pytestmark = pytest.mark.gpu


def held(rows, cols, scales, seed, block=1):
    """A matrix of random bytes (none a NaN), zero past cols, whose scales are drawn from `scales`."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    f = vp.Fp8.empty(rows, cols, block)
    u = torch.randint(0, 256, f.q.shape, generator=g, device=DEV).to(torch.uint8)
    u[(u & 127) == 127] = 0
    u[:, cols:] = 0
    f.q.view(torch.uint8).copy_(u)
    pick = torch.randint(0, len(scales), f.scale.shape, generator=g, device=DEV)
    f.scale.copy_(torch.tensor(scales, dtype=torch.uint8, device=DEV)[pick])
    return f


def test_transpose_of_the_largest_f32():
    """3.4e38 is 256 * 2^120 in 8 bits, 2^128, which no f32 holds; the transpose is of the value, not of an infinity."""
    x = torch.randn((130, 200), device=DEV)
    x[7, 11] = 3.4028234663852886e38
    x[8, 150] = -3.4028234663852886e38
    a = vp.fp8_quantize(x)
    assert int(a.scale.max()) == 247
    same(vp.fp8_transpose(a), R.values(a.q, a.scale, 200, 1).t(), 1)


@pytest.mark.parametrize("rows,cols", [(3, 5), (128, 128), (130, 257), (300, 1176)])
@pytest.mark.parametrize("scales", [(254,), (250, 251, 252, 253, 254), (1, 254), (1,), (1, 2, 3), (1, 60, 127, 200, 254),
                                    (245, 246, 247, 248, 249)])
def test_transpose_of_every_scale(rows, cols, scales):
    """Values up to 448 * 2^127 and down to 2^-135, beside each other too."""
    a = held(rows, cols, scales, rows + cols)
    t = vp.fp8_transpose(a)
    v = R.values(a.q, a.scale, cols, 1).t()
    q, s = R.quantize(v, 1)
    assert bool((t.scale == s).all()) and bool((t.q.double() == q).all())


@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_dequantize_of_every_scale(out):
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    for scales in ((254,), (1, 254), (1, 2, 3), (246, 247, 248)):
        a = held(130, 300, scales, 7)
        ref = R.values(a.q, a.scale, 300, 1)
        got = vp.fp8_dequantize(a, out)
        assert torch.equal(got, ref.to(torch.float32).to(dtype) if out == "f32" else ref.to(dtype))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(5, 300, 640), (130, 64, 6000), (200, 2106, 130), (130, 12604, 130), (130, 38488, 500)])
def test_product_whose_scale_is_not_a_number(m, n, k, out):
    """Scale 255 stands for NaN whatever the bytes beside it hold; the other rows do not see it."""
    a, b = held(m, k, (120, 121, 122), 1), held(n, k, (125, 126), 2, 128)
    a.scale[m // 2, (k - 1) // 128] = 255
    y = vp.fp8_matmul(a, b, out)
    assert torch.isnan(y[m // 2]).all()
    a.scale[m // 2, (k - 1) // 128] = 120
    z = vp.fp8_matmul(a, b, out)
    z[m // 2] = y[m // 2]
    assert torch.equal(torch.nan_to_num(y, nan=1.0), torch.nan_to_num(z, nan=1.0))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(5, 300, 640), (200, 2106, 130), (130, 12604, 130), (130, 38488, 500)])
def test_product_of_large_and_small_scales(m, n, k, out):
    """Scales of 2^118 against 2^-120: values just below 2^128, products of order one."""
    a, b = held(m, k, (243, 244, 245), 1), held(n, k, (7, 8), 2, 128)
    check_product(vp.fp8_matmul(a, b, out), a, b, k)


@pytest.mark.parametrize("m,n,k", [(5, 300, 640), (200, 2106, 1024), (66, 24628, 140), (130, 38488, 513)])
@pytest.mark.parametrize("small", [0.171875, 0.1875, 1.0])
def test_product_whose_large_terms_cancel(m, n, k, small):
    """One product of 256 in each run of 8 columns, its sign turned over from run to run, and seven of small^2 beside it
    (0.0295 is just below 2^-13 of 256).  f32 results hold the sum; bf16 ones may lose 7 * 2^-13 of each run's largest."""
    r = torch.arange(k, device=DEV)
    x = torch.where(r % 8 == 3, 16.0, small).repeat(m, 1)
    y = torch.where(r % 8 == 3, torch.where(r // 8 % 2 == 0, 16.0, -16.0), small).repeat(n, 1)
    a, b = vp.fp8_quantize(x), vp.fp8_quantize(y, 128)
    va, vb = R.values(a.q, a.scale, k, 1), R.values(b.q, b.scale, k, 128)
    assert torch.equal(va, x.double()) and torch.equal(vb, y.double())
    ref = (va[0] * vb[0]).sum()
    f32 = vp.fp8_matmul(a, b, "f32")
    check_product(f32, a, b, k)
    off = (vp.fp8_matmul(a, b).double() - ref).abs()
    most = 7 * 2.0 ** -13 * 256 * R.up(k, 8) / 8 + k ** 0.5 * 2.0 ** -23 * (va[0] * vb[0]).abs().sum()
    assert bool((off <= most * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()).all())
