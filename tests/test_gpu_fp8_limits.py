"""GPU tests of the 8-bit operators on sizes that one launch of a kernel does not take: 2^32 threads and more."""
import gc

import pytest
import torch

import fp8_reference as R
import paper_2604_16893_amd as vp
from test_gpu_fp8 import DEV, check_product, rand, same

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory():
    yield
    gc.collect()
    torch.cuda.empty_cache()


def line(n, first):
    """bf16 zeros, random from `first` on."""
    x = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    x[first:] = rand((n - first,), 1, torch.bfloat16)
    return x


@pytest.mark.parametrize("shape", ["row", "column"])
def test_more_tiles_than_a_launch(shape):
    """8.6 million tiles of 128 x 128, 512 threads each: values about the end of the first launch's and the last ones."""
    n, end = 1_100_000_003, (0xffffffff // 512) * 128
    x = line(n, end - 5000)
    if shape == "row":
        f = vp.fp8_quantize(x[None, :], 128)
    else:
        f = vp.fp8_quantize(x[:, None], rows=False, cols=True)
    assert f.shape == (1, n)
    first = end - 128 * 40
    q, s = R.quantize(x[None, first:], 1)
    assert torch.equal(f.q[:, first:].double(), q)
    last = -(-n // 128)
    assert torch.equal(f.scale[:, first // 128:last], s[:, :last - first // 128]) and (f.scale[:, last:] == 0).all()
    assert (f.q.view(torch.uint8)[:, :first] == 0).all() and (f.scale[:, :first // 128] == 1).all()


def test_more_rows_than_a_launch():
    """2^30 rows of one column: their conversions take two launches each; 150 GB."""
    if torch.cuda.mem_get_info()[0] < 180 << 30:
        pytest.skip("needs 180 GiB of device memory")
    n, end = (1 << 30) + 200, (0xffffffff // 256) * 64
    x = line(n, end - 100)[:, None]
    a = vp.fp8_quantize(x)
    part = vp.Fp8(a.q[end - 100:], a.scale[end - 100:], 1)
    same(part, x[end - 100:], 1)
    back = vp.fp8_dequantize(a)
    assert torch.equal(back[end - 100:].double(), R.values(part.q, part.scale, 1, 1)) and not back[:end - 100].any()
    del back
    b = vp.fp8_quantize(torch.tensor([[1.0], [-3.0], [0.5]], device=DEV), 128)
    y = vp.fp8_matmul(a, b)
    check_product(y[end - 100:], part, b, 1)
    assert not y[:end - 100].any()
