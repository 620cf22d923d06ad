"""Gradients of head norms that nobody asks for are not formed."""
import pytest
import torch

import paper_2504_09135_b200 as disc
from paper_2504_09135_b200 import model_ops

pytestmark = pytest.mark.gpu
DEV = "cuda"


def inputs(n=20, hq=4, hkv=2, d=64):
    g = torch.Generator(device=DEV).manual_seed(8)
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    w = [1 + 0.2 * torch.randn(d, generator=g, device=DEV) for _ in range(2)]
    freq = torch.exp(torch.arange(d // 2, device=DEV) * (-0.2))
    return q, k, v, w[0], w[1], torch.arange(n, dtype=torch.int32, device=DEV), freq


WANTED = [(1, 1, 1, 1), (1, 1, 0, 0), (1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (1, 0, 0, 1), (0, 0, 1, 1)]


@pytest.mark.parametrize("wanted", WANTED)
def test_only_what_is_asked_for_is_formed(wanted, monkeypatch):
    q, k, _, qw, kw, pos, freq = inputs()
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    want = disc.disc_norm_rope_grad(q, k, pos, freq, dq, dk, q_weight=qw, k_weight=kw)
    formed = []
    real = model_ops.disc_norm_rope_grad

    def spy(*args, **named):
        formed.append(real(*args, **named))
        return formed[-1]

    monkeypatch.setattr(model_ops, "disc_norm_rope_grad", spy)
    leaves = [t.detach().clone().requires_grad_(bool(a)) for t, a in zip((q, k, qw, kw), wanted)]
    y = disc.disc_norm_rope(leaves[0], leaves[1], pos, freq, q_weight=leaves[2], k_weight=leaves[3])
    torch.autograd.backward(y, (dq, dk))
    for leaf, a, g in zip(leaves, wanted, want):
        assert torch.equal(leaf.grad, g) if a else leaf.grad is None
    (got,) = formed
    assert (got[0] is not None) == bool(wanted[0] or wanted[2]) and (got[1] is not None) == bool(wanted[1] or wanted[3])
    assert (got[2] is not None) == bool(wanted[2]) and (got[3] is not None) == bool(wanted[3])


def test_sums_of_the_weights_one_by_one():
    q, k, _, qw, kw, pos, freq = inputs()
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    args = (q, k, pos, freq, dq, dk)
    want = disc.disc_norm_rope_grad(*args, q_weight=qw, k_weight=kw)
    for a in (False, True):
        for b in (False, True):
            got = disc.disc_norm_rope_grad(*args, q_weight=qw, k_weight=kw, q_weight_grad=a, k_weight_grad=b)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            assert torch.equal(got[2], want[2]) if a else got[2] is None
            assert torch.equal(got[3], want[3]) if b else got[3] is None
