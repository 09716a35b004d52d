"""The 8-bit operators and torch.autograd: no graph is recorded, so a call that would lose a gradient is refused, and a
torch.autograd.Function around them gives the gradients."""
import pytest
import torch

import fp8_reference as R
import paper_2604_16893_amd as vp


@pytest.mark.parametrize("call", [
    lambda x, w: vp.fp8_quantize(x),
    lambda x, w: vp.vp_fp8_quantize(x, None, None),
    lambda x, w: vp.rms_norm(x, w),
    lambda x, w: vp.rms_norm(x.detach(), w),
    lambda x, w: vp.rms_norm(x.detach(), w.detach(), x),
    lambda x, w: vp.vp_rms_norm(x, w, out=x),
])
def test_gradients_are_not_lost_in_silence(call):
    x, w = torch.zeros((4, 200), requires_grad=True), torch.ones(200, requires_grad=True)
    with pytest.raises(vp.VPError, match="gradient"):
        call(x, w)
    with torch.no_grad(), pytest.raises(vp.VPError, match="CUDA"):     # (the next check: these are not on a GPU)
        call(x, w)


class NormedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gain, weight):
        n, h, rstd = vp.rms_norm(x, gain, out="fp8")
        w, w_t = vp.fp8_quantize(weight, 128, cols=True)
        ctx.save_for_backward(h, gain, rstd)
        ctx.held = n, w_t
        return vp.fp8_matmul(n, w)

    @staticmethod
    def backward(ctx, grad):
        h, gain, rstd = ctx.saved_tensors
        n, w_t = ctx.held
        g, g_t = vp.fp8_quantize(grad, cols=True)
        dx, dgain = vp.rms_norm_backward(vp.fp8_matmul(g, w_t), h, gain, rstd)
        return dx, dgain.to(gain.dtype), vp.fp8_matmul(g_t, vp.fp8_transpose(n), "f32")


@pytest.mark.gpu
def test_a_function_gives_the_gradients():
    """Against 64 bits without quantisation: two 8-bit factors behind each result, a rounding of 0.026 of it as a whole for
    each, and the transposes' third: below 0.026 * sqrt(3) < 0.05."""
    g = torch.Generator(device="cuda:0")
    g.manual_seed(5)
    x = torch.randn(300, 640, generator=g, device="cuda:0").bfloat16().requires_grad_()
    gain = (1 + 0.1 * torch.randn(640, generator=g, device="cuda:0")).bfloat16().requires_grad_()
    weight = (torch.randn(384, 640, generator=g, device="cuda:0") / 25).requires_grad_()
    grad = torch.randn(300, 384, generator=g, device="cuda:0").bfloat16()
    with pytest.raises(vp.VPError, match="gradient"):
        vp.rms_norm(x, gain)
    y = NormedLinear.apply(x, gain, weight)
    y.backward(grad)
    ref, h, rstd = R.rms_norm(x.detach(), None, gain.detach(), 1e-6)
    dn = grad.double() @ weight.detach().double()
    dx, dgain = R.rms_norm_backward(dn, h, gain.detach(), rstd, None)
    for got, want in ((y.detach(), ref @ weight.detach().double().t()), (x.grad, dx), (gain.grad, dgain),
                      (weight.grad, grad.double().t() @ ref)):
        assert ((got.double() - want).norm() / want.norm()).item() < 0.05
