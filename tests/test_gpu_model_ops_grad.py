"""Calls on tensors that require a gradient: the log-probabilities have one, the others refuse."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,inv_t", [(3, 50, 1.0), (5, 4001, 0.7), (2, 128256, 30.0)])
def test_log_probabilities_and_entropy_have_a_gradient(dtype, n, V, inv_t):
    z = (torch.randn((n, V), device=DEV) * 2).to(dtype).requires_grad_()
    t = torch.randint(0, V, (n,), dtype=torch.int32, device=DEV)
    plain = disc.disc_logprobs(z.detach(), t, top=3, inv_temperature=inv_t)
    r = disc.disc_logprobs(z, t, top=3, inv_temperature=inv_t)
    for k in plain:
        assert torch.equal(r[k], plain[k])
    assert r["logp"].requires_grad and r["entropy"].requires_grad
    assert not any(r[k].requires_grad for k in ("lse", "top_ids", "top_logp", "status"))
    a, b = torch.randn(n, device=DEV), torch.randn(n, device=DEV)
    g, = torch.autograd.grad((a * r["logp"] + b * r["entropy"]).sum(), z)
    assert torch.equal(g, disc.disc_logprobs_grad(z.detach(), t, plain["lse"], plain["entropy"], a, b, inv_temperature=inv_t))
    r = disc.disc_logprobs(z, t, inv_temperature=inv_t)
    g, = torch.autograd.grad((a * r["logp"]).sum(), z)
    assert torch.equal(g, disc.disc_logprobs_grad(z.detach(), t, plain["lse"], plain["entropy"], a, inv_temperature=inv_t))
    r = disc.disc_logprobs(z, inv_temperature=inv_t)
    assert r["logp"] is None
    g, = torch.autograd.grad(r["entropy"].sum(), z)
    assert torch.equal(g, disc.disc_logprobs_grad(z.detach(), None, plain["lse"], plain["entropy"], None, torch.ones(n, device=DEV), inv_temperature=inv_t))


def test_a_gradient_through_a_projection_and_on_another_stream():
    n, d, V = 6, 16, 500
    h, w = torch.randn((n, d), device=DEV), torch.randn((d, V), device=DEV).requires_grad_()
    t = torch.randint(0, V, (n,), dtype=torch.int32, device=DEV)
    disc.disc_logprobs(h @ w, t)["logp"].sum().backward()
    got, w.grad = w.grad, None
    torch.log_softmax(h @ w, dim=1).gather(1, t.long()[:, None]).sum().backward()
    assert torch.all((got - w.grad).abs() <= 2.0 ** -14 * (h.abs().T @ torch.ones((n, V), device=DEV)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        w2 = w.detach().clone().requires_grad_()
        disc.disc_logprobs(h @ w2, t)["logp"].sum().backward()
    torch.cuda.synchronize()
    assert torch.equal(w2.grad, got)


def test_without_a_gradient_asked_for_nothing_is_recorded():
    z = torch.randn((3, 50), device=DEV, requires_grad=True)
    with torch.no_grad():
        assert not disc.disc_logprobs(z)["lse"].requires_grad
    out = disc.disc_logprobs(z.detach())
    with pytest.raises(TypeError):
        disc.disc_logprobs(z, out=out)                  # given buffers have no history


def test_what_has_no_gradient_refuses():
    q = torch.randn((8, 2, 64), device=DEV).bfloat16()
    g = q.clone().requires_grad_()
    cu = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    for args in ((g, q, q), (q, g, q), (q, q, g)):
        with pytest.raises(TypeError):
            disc.disc_attend_prompt(*args, cu, max_len=8)
    cache = disc.DiscCache.empty(1, 16, 16, 2, 64, 8, 2)
    disc.disc_cache_extend(cache)
    for args in ((g, q), (q, g)):
        with pytest.raises(TypeError):
            disc.disc_cache_write(cache, 0, *args)
    disc.disc_cache_write(cache, 0, q, q)
    plan = disc.disc_attend_plan(cache, 2)
    with pytest.raises(TypeError):
        disc.disc_attend_cached(cache, 0, g, plan)
    with torch.no_grad():
        disc.disc_attend_prompt(g, g, g, cu, max_len=8)
        disc.disc_cache_write(cache, 0, g, g)
        disc.disc_attend_cached(cache, 0, g, plan)
    z = torch.randn((8, 50), device=DEV, requires_grad=True)
    lse = torch.zeros(8, device=DEV)
    with pytest.raises(TypeError):
        disc.disc_logprobs_grad(z, torch.zeros(8, dtype=torch.int32, device=DEV), lse, None, lse)
