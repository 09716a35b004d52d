"""GPU tests of the norm's weight gradient over so many rows that the order of its sum shows.

Tolerance: a part of 64 rows, up to 64 parts in a row of a wave's or workgroup's, then at most 16 steps of the join over
workgroups: less than 2^7 additions in a row of one accumulator, 2^-24 each of S = sum |dy n|, and the roundings of dy n:
2^-17 S, the bound of test_gpu_norm.py.  Equal terms make an accumulator's roundings all go one way.
"""
import gc

import pytest
import torch

import paper_2604_16893_amd as vp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("values", ["equal", "positive", "signed"])
@pytest.mark.parametrize("rows,cols,dtype", [(1 << 22, 64, "bf16"), ((1 << 22) + 77, 65, "f32"), (1 << 20, 700, "bf16"),
                                             (1 << 21, 1280, "bf16"), ((1 << 18) + 3, 4100, "bf16"), (1 << 18, 9000, "bf16"),
                                             (1 << 18, 2048, "f32")])
def test_weight_gradient_of_many_rows(rows, cols, dtype, values):
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    dy = torch.empty((rows, cols), dtype=t, device=DEV)
    if values == "equal":
        dy.fill_(0.1)
    else:
        dy.uniform_(0.0 if values == "positive" else -1.0, 1.0, generator=g)
    h, rstd = torch.ones_like(dy), torch.full((rows,), 0.9993, device=DEV)
    w = torch.ones(cols, dtype=t, device=DEV)
    _, dw = vp.rms_norm_backward(dy, h, w, rstd)
    ref, size = (torch.zeros(cols, dtype=torch.float64, device=DEV) for _ in range(2))
    for r in range(0, rows, 1 << 16):
        part = dy[r:r + (1 << 16)].double() * rstd[0].double()
        ref += part.sum(0)
        size += part.abs().sum(0)
    assert bool(((dw.double() - ref).abs() <= 2.0 ** -17 * size).all())
    del dy, h, part
    gc.collect()
    torch.cuda.empty_cache()
