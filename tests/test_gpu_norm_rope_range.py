"""disc_norm_rope and its gradient over the whole range of sizes that is accepted, and with eps = 0."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc
from held_reference import norm_rope64
from model_ops_reference import UNIT

pytestmark = pytest.mark.gpu
DEV = "cuda"
# size of the values, eps; bf16 (f16 does not reach there) but for the last two
SIZES = [(3e-18, 0.0), (1e-15, 0.0), (1e-12, 0.0), (1e-15, 1e-6), (1.0, 0.0), (1e10, 1e-6), (1e14, 1e-6), (1e15, 1e-6), (1e17, 1e-6)]
CASES = [(torch.bfloat16, s, e) for s, e in SIZES] + [(torch.float16, 1e-4, 0.0), (torch.float16, 1e4, 1e-6)]


def frequencies(rot):
    return torch.exp(torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) * (-math.log(10000.0) / rot)).float()


def inputs(n, heads, d, dtype, size, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn((n, heads, d), generator=g, device=DEV, dtype=torch.float64) * size).to(dtype)
    pos = torch.randint(0, 5000, (n,), generator=g, device=DEV, dtype=torch.int32)
    w = 1 + 0.2 * torch.randn(d, generator=g, device=DEV)
    dy = torch.randn((n, heads, d), generator=g, device=DEV, dtype=torch.float64)
    return x, pos, w, dy


@pytest.mark.parametrize("dtype,size,eps", CASES)
@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (64, 32, True), (72, 72, False)])
def test_forward(d, rot, inter, dtype, size, eps):
    x, pos, w, _ = inputs(37, 5, d, dtype, size, 1)
    freq = frequencies(rot)
    got = disc.disc_norm_rope(x, None, pos, freq, q_weight=w, eps=eps, interleaved=inter)[0].double()
    want, most = norm_rope64(x.double(), w.double(), pos, freq, eps=eps, interleaved=inter)
    # the factors of tol_forward, which are relative, and one rounding; the absolute step belongs to f16 alone
    tol = UNIT[dtype] * want.abs() + 2.0 ** -16 * most + (2.0 ** -25 if dtype is torch.float16 else 0.0)
    err = (got - want).abs()
    assert torch.all(err <= tol), float((err / tol).max())


@pytest.mark.parametrize("dtype,size,eps", CASES)
@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (64, 32, True), (72, 72, False)])
def test_gradient(d, rot, inter, dtype, size, eps):
    x, pos, w, dy = inputs(37, 5, d, dtype, size, 2)
    # gradients of a size at which dx = dy / size is one of the type's values
    dy = (dy * (size if dtype is torch.float16 and size < 1 else 1.0)).to(dtype)
    freq = frequencies(rot)
    dx, _, dw, _ = disc.disc_norm_rope_grad(x, None, pos, freq, dy, None, q_weight=w, eps=eps, interleaved=inter)
    a, b = x.double().requires_grad_(), w.double().requires_grad_()
    want, want_w = torch.autograd.grad(norm_rope64(a, b, pos, freq, eps=eps, interleaved=inter)[0], [a, b], dy.double())
    # with xh = x r, c = |w| G and G a bound of the rotated-back gradient: dx = r (w g - xh mean(w g xh)), each factor off by less than 2^-16
    # of itself and the mean by 2^-17 more, so 2^-13 of r (c + |xh| mean(c |xh|)); one rounding
    most = norm_rope64(dy.double(), None, pos, freq, norm=False, interleaved=inter)[1]
    r = 1 / torch.sqrt(x.double().square().mean(dim=-1, keepdim=True) + eps)
    xh, c = x.double().abs() * r, most * w.double().abs()
    tol = 2.0 ** -13 * r * (c + xh * (c * xh).mean(dim=-1, keepdim=True)) + UNIT[dtype] * want.abs() + (2.0 ** -25 if dtype is torch.float16 else 0.0)
    err = (dx.double() - want).abs()
    assert torch.all(err <= tol), float((err / tol).max())
    # 185 terms g xh, each as above, summed in fp32
    err, tol = (dw.double() - want_w).abs(), (most * xh).sum(dim=(0, 1)) * (2.0 ** -14 + 185 * 2.0 ** -24)
    assert torch.all(err <= tol), float((err / tol).max())
