"""Buffers given as `out` are known to autograd as written in place."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def inputs(n=20, hq=4, hkv=2, d=64):
    g = torch.Generator(device=DEV).manual_seed(8)
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).bfloat16() for h in (hq, hkv, hkv))
    w = [1 + 0.2 * torch.randn(d, generator=g, device=DEV) for _ in range(2)]
    freq = torch.exp(torch.arange(d // 2, device=DEV) * (-0.2))
    return q, k, v, w[0], w[1], torch.arange(n, dtype=torch.int32, device=DEV), freq


def saved(t):
    """The output of an operation whose gradient needs t as it was."""
    w = torch.ones_like(t, requires_grad=True)
    return (w * t).sum()


def test_buffers_that_a_graph_has_saved_are_known_to_be_written():
    q, k, v, qw, kw, pos, freq = inputs()
    cache = disc.DiscCache.empty(1, 4, 16, 2, 64, 20, 1, held="i8")
    cu = torch.arange(21, dtype=torch.int32, device=DEV)
    logits = torch.randn((20, 50), device=DEV)
    r = disc.disc_logprobs(logits, pos)
    plain = disc.DiscCache.empty(1, 20, 16, 2, 64, 20, 1)
    disc.disc_cache_extend(plain)
    plan = disc.disc_attend_plan(plain, 4)
    out, lse = torch.empty_like(q), torch.empty((20, 4), device=DEV)
    cu1 = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    calls = [((q, k), lambda: disc.disc_norm_rope(q, k, pos, freq, out=(q, k))),
             ((q,), lambda: disc.disc_norm_rope_write(cache, 0, q, k, v, freq, out=q)),
             ((k, v), lambda: disc.disc_cache_read(cache, 0, cu, 20, out=(k, v))),
             ((out, lse), lambda: disc.disc_attend_prompt(q, k, v, cu1, max_len=20, out=out, lse=lse)),
             ((out, lse), lambda: disc.disc_attend_cached(plain, 0, q, plan, out=out, lse=lse)),
             ((r["logp"], r["entropy"], r["lse"]), lambda: disc.disc_logprobs(logits, pos, out=r)),
             ((logits,), lambda: disc.disc_logprobs_grad(logits, pos, r["lse"], None, torch.ones(20, device=DEV), out=logits))]
    for buffers, call in calls:
        losses = [saved(t) for t in buffers]
        call()
        for loss in losses:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
    # inputs are not
    losses = [saved(t) for t in (q, k, qw)]
    disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, out=(torch.empty_like(q), torch.empty_like(k)))
    for loss in losses:
        loss.backward()


def test_buffers_of_inference_mode():
    with torch.inference_mode():
        q, k, _, qw, kw, pos, freq = inputs()
        want = disc.disc_norm_rope(q, k, pos, freq)
        disc.disc_norm_rope(q, k, pos, freq, out=(q, k))
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
