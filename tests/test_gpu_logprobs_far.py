"""Log-probabilities and gradients of rows whose log-sum-exp is large: masks of a finite value, low temperatures.  fp32 holds such a
log-sum-exp only to some 2^-24 of its size, but log-probabilities, probabilities and gradients hang on differences of logits."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def reference(z, inv_t):
    """log p, p and entropy in 64 bits, from differences to the row's maximum."""
    d = (z.double() - z.double().amax(dim=1, keepdim=True)) * float(torch.tensor(inv_t, dtype=torch.float32))
    lp = d - torch.logsumexp(d, dim=1, keepdim=True)
    p = lp.exp()
    return lp, p, -(p * torch.where(p > 0, lp, 0.0)).sum(dim=1)


def base(V):
    """What fp32 sums of V terms in 256 threads and 2^x to 2^-22 allow, whatever the size of the logits."""
    return 2.0 ** -20 + (V / 256 + 40) * 2.0 ** -24


def check(z, t, inv_t, top):
    """A log-probability is log2(e)/T times a difference of logits (three roundings of 2^-24, twice) plus the logarithm of the sum."""
    n, V = z.shape
    r = disc.disc_logprobs(z, t, top=top, inv_temperature=inv_t)
    lp, p, H = reference(z, inv_t)
    assert torch.all(r["status"] == 0)
    want = lp.gather(1, t.long()[:, None])[:, 0]
    assert torch.all((r["logp"].double() - want).abs() <= base(V) + 2.0 ** -21 * want.abs())
    assert torch.all(r["logp"] <= 0)
    assert torch.all((r["entropy"].double() - H).abs() <= base(V) * (2 + 2 * math.log(V + 1)))
    want = lp.gather(1, r["top_ids"].long())
    assert torch.all((r["top_logp"].double() - want).abs() <= base(V) + 2.0 ** -21 * want.abs())
    a, b = torch.randn(n, device=DEV), torch.randn(n, device=DEV)
    one = torch.zeros_like(lp)
    one.scatter_(1, t.long()[:, None], 1.0)
    for db in (None, b):
        a64 = a.double()[:, None]
        b64 = torch.zeros_like(a64) if db is None else db.double()[:, None]
        step = torch.where(p > 0, lp, 0.0)
        want = ((one - p) * a64 - p * (step + H[:, None]) * b64) * inv_t
        # of a probability: its own log's error; of the entropy's part the errors of log p and H
        rel = base(V) + 2.0 ** -21 * step.abs()
        tol = inv_t * p * (rel * (a64.abs() + b64.abs() * (step.abs() + H[:, None])) + b64.abs() * (rel + base(V) * (2 + 2 * math.log(V + 1))))
        tol = tol + UNIT[z.dtype] * want.abs() + 2.0 ** -23 * inv_t * a64.abs() * one + 1e-30
        g = disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], a, db, inv_temperature=inv_t)
        err = (g.double() - want).abs()
        assert torch.all(err <= tol), float((err - tol).max())
        same = z.clone()                                # in place
        disc.disc_logprobs_grad(same, t, r["lse"], r["entropy"], a, db, inv_temperature=inv_t, out=same)
        assert torch.equal(same, g)
    return r


SIZES = [(3, 7), (5, 300), (4, 1000), (3, 3000), (2, 32001), (200, 20000), (1, 128256)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("value", [-1e9, "lowest", -2e4, 1e6])
def test_rows_of_one_large_value(dtype, n, V, value):
    z = torch.full((n, V), torch.finfo(dtype).min if value == "lowest" else value, dtype=dtype, device=DEV)
    t = torch.randint(0, V, (n,), dtype=torch.int32, device=DEV)
    r = check(z, t, 1.0, min(4, V))
    assert torch.all((r["logp"] + math.log(V)).abs() <= base(V) + 2.0 ** -21 * math.log(V))
    g = disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], torch.ones(n, device=DEV))
    assert torch.all(g.double().sum(dim=1).abs() <= 2 * (UNIT[dtype] + base(V)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", SIZES)
def test_masks_of_a_finite_value_beside_logits(dtype, n, V):
    z = (torch.randn((n, V), device=DEV) * 3).to(dtype)
    z[:, ::2] = -1e9
    z[n // 2] = -1e9                                    # nothing left of one row
    t = (torch.randint(0, V // 2, (n,), device=DEV) * 2 + 1).to(torch.int32)
    check(z, t, 1.0, min(3, V))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("inv_t", [1000.0, 40.0])
def test_low_temperatures(dtype, n, V, inv_t):
    """Logits near 30 that differ by hundredths: at T = 1/1000 their log-sum-exp is some 3e4."""
    z = (30 + torch.randn((n, V), device=DEV) * 0.02).to(dtype)
    z[0] = (torch.randn(V, device=DEV) * 3).to(dtype)
    t = torch.randint(0, V, (n,), dtype=torch.int32, device=DEV)
    check(z, t, inv_t, min(5, V))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 5000, 40000])
def test_rows_without_a_finite_sum_have_no_finite_gradient(dtype, V):
    z = torch.randn((4, V), device=DEV).to(dtype)
    z[0, V // 2] = math.inf
    z[1, V // 3] = math.nan
    z[2] = -math.inf
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    r = disc.disc_logprobs(z, t)
    for b in (None, torch.ones(4, device=DEV)):
        g = disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], torch.ones(4, device=DEV), b)
        assert not torch.isfinite(g[:2]).any()
        assert torch.all(g[2] == 0) and torch.isfinite(g[3]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,cut", [(200, 77), (9000, 4000), (40001, 8)])
@pytest.mark.parametrize("inv_t", [1.0, 40.0])
def test_a_row_in_two_parts_with_the_whole_rows_log_sum_exp(dtype, V, cut, inv_t):
    """Each part's gradient is its part of the whole row's: the log-sum-exp that is given counts, not the part's own.  It is held to
    2^-24 of its size, as is its product with log2(e)."""
    z = (torch.randn((6, V), device=DEV) * 4).to(dtype)
    t = torch.full((6,), -1, dtype=torch.int32, device=DEV)
    r = disc.disc_logprobs(z, inv_temperature=inv_t)
    lp, p, H = reference(z, inv_t)
    b = torch.randn(6, device=DEV)
    for part, q, l in ((z[:, :cut], p[:, :cut], lp[:, :cut]), (z[:, cut:], p[:, cut:], lp[:, cut:])):
        step = torch.where(q > 0, l, 0.0)
        want = -q * (step + H[:, None]) * b.double()[:, None] * inv_t
        got = disc.disc_logprobs_grad(part, t, r["lse"], r["entropy"], None, b, inv_temperature=inv_t)
        rel = base(V) + 2.0 ** -21 * step.abs() + 2.0 ** -22 * r["lse"].double().abs()[:, None]
        tol = inv_t * q * b.double().abs()[:, None] * (rel * (step.abs() + H[:, None] + 1) + base(V) * (2 + 2 * math.log(V + 1))) + UNIT[dtype] * want.abs() + 1e-30
        assert torch.all((got.double() - want).abs() <= tol)
