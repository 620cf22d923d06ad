"""Tensors with a tangent (forward-mode differentiation) are refused: the results would have none."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def inputs(n=20, hq=4, hkv=2, d=64):
    g = torch.Generator(device=DEV).manual_seed(8)
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    w = [1 + 0.2 * torch.randn(d, generator=g, device=DEV) for _ in range(2)]
    freq = torch.exp(torch.arange(d // 2, device=DEV) * (-0.2))
    return q, k, v, w[0], w[1], torch.arange(n, dtype=torch.int32, device=DEV), freq


def test_tangents_are_refused():
    q, k, v, qw, kw, pos, freq = inputs()
    cache = disc.DiscCache.empty(1, 20, 16, 2, 64, 20, 1)
    disc.disc_cache_extend(cache)
    plan = disc.disc_attend_plan(cache, 4)
    logits = torch.randn((20, 50), device=DEV)
    cu = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    with forward_ad.dual_level():
        def dual(t):
            return forward_ad.make_dual(t, torch.ones_like(t))

        for call in (lambda: disc.disc_norm_rope(dual(q), k, pos, freq), lambda: disc.disc_norm_rope(q, dual(k), pos, freq),
                     lambda: disc.disc_norm_rope(q, k, pos, dual(freq)), lambda: disc.disc_norm_rope(q, k, pos, freq, q_weight=dual(qw)),
                     lambda: disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=dual(kw)),
                     lambda: disc.disc_norm_rope_grad(q, None, pos, freq, dual(q), None),
                     lambda: disc.disc_norm_rope_write(cache, 0, q, k, dual(v), freq), lambda: disc.disc_norm_rope_write(cache, 0, q, k, v, freq, q_weight=dual(qw)),
                     lambda: disc.disc_cache_write(cache, 0, dual(k), v), lambda: disc.disc_attend_cached(cache, 0, dual(q), plan),
                     lambda: disc.disc_attend_prompt(q, dual(k), v, cu, max_len=20), lambda: disc.disc_logprobs(dual(logits), pos)):
            with pytest.raises(TypeError, match="tangent"):
                call()
        # tensors without one are taken as ever
        a = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw)
    assert torch.equal(a[0], disc.disc_norm_rope(q, k, pos, freq, q_weight=qw)[0])
