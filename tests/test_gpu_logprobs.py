"""disc_logprobs and disc_logprobs_grad against the definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _logits(n, V, dtype, seed, ld=None, offset=0, scale=3.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ld = V if ld is None else ld
    flat = torch.full((offset + n * ld,), math.nan, dtype=dtype, device=DEV)      # what is not a logit must not be looked at
    z = flat[offset:].view(n, ld)[:, :V]
    z.copy_(torch.randn((n, V), generator=gen, device=DEV) * scale)
    return z


def _order(row):
    """Ids by value, larger first, -0 = +0, lower id first, NaN last."""
    x = row.float().cpu().numpy().astype(np.float64)
    key = np.where(np.isnan(x), -np.inf, x + 0.0)
    return np.lexsort((np.arange(x.size), -key, np.isnan(x)))


def _check(z, targets, top, inv_t, r):
    """Sums in fp32: a thread adds at most V / 256 + 40 terms, each step 2^-24; 2^x is good to 2^-22; arguments are rounded relative
    to the row's span."""
    n, V = z.shape
    y = z.double() * inv_t
    lp = torch.log_softmax(y, dim=1)
    p = lp.exp()
    H = -(p * torch.where(p > 0, lp, 0.0)).sum(dim=1)
    lse = torch.logsumexp(y, dim=1)
    span = torch.where(torch.isinf(y), 0.0, y).abs().amax(dim=1)
    tol = 2.0 ** -21 + (V / 256 + 40) * 2.0 ** -24 + 2.0 ** -22 * span
    assert torch.all((r["lse"].double() - lse).abs() <= tol)
    assert torch.all((r["entropy"].double() - H).abs() <= tol * (2 + 2 * math.log(V + 1)))
    if targets is not None:
        t = targets.long()
        want = torch.where(t >= 0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
        err = (r["logp"].double() - want).abs()
        err[torch.isinf(want) & (r["logp"] == -math.inf)] = 0
        assert torch.all(err <= 2 * tol)
    for i in range(n if top else 0):
        ids = r["top_ids"][i].cpu().numpy()
        order = _order(z[i])[:top]
        assert np.array_equal(ids[:order.size], order), i
        assert np.all(ids[order.size:] == -1)
        got = r["top_logp"][i, :order.size].double()
        want = lp[i, torch.as_tensor(order.copy(), device=DEV)]
        same = torch.isinf(want) & (got == want)
        assert torch.all(((got - want).abs() <= 2 * tol[i]) | same)
        assert torch.all(r["top_logp"][i, order.size:] == -math.inf)
    assert torch.all(r["status"] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,ld,offset,top", [
    (1, 1, 1, 0, 1), (3, 2, 2, 0, 5), (5, 7, 9, 1, 3), (4, 64, 64, 0, 64), (2, 255, 255, 3, 20), (300, 256, 256, 0, 5), (7, 1000, 1003, 5, 64),
    (1, 8192, 8192, 0, 20), (2, 50257, 50257, 0, 20), (1, 128256, 128256, 0, 64), (3, 128256, 128257, 1, 1), (160, 32000, 32000, 0, 20), (9, 32001, 32008, 7, 0)])
def test_against_the_definition(dtype, n, V, ld, offset, top):
    z = _logits(n, V, dtype, n + V, ld, offset)
    t = torch.randint(-1, V, (n,), dtype=torch.int32, device=DEV)
    t[0] = V - 1
    for inv_t in (1.0, 0.7):
        _check(z, t, top, inv_t, disc.disc_logprobs(z, t, top=top, inv_temperature=inv_t))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 32000, 128256])
def test_rows_that_are_hard_for_the_selection(dtype, V):
    rows = [torch.zeros(V), torch.linspace(-5, 5, V), torch.linspace(5, -5, V), torch.randint(0, 3, (V,)).float(), torch.randint(0, 40, (V,)).float() / 8]
    stripes = torch.randn(V) * 0.1                     # every large value in the columns of few threads
    stripes[torch.arange(V) // 8 % 256 == 3] += 20
    rows.append(stripes)
    some = torch.full((V,), -math.inf)                 # all masked but a few
    some[[1, 17, V - 1]] = torch.tensor([0.5, -2.0, 0.5])
    rows.append(some)
    signs = torch.zeros(V)
    signs[::2] = -0.0
    rows.append(signs)
    z = torch.stack(rows).to(DEV, dtype)
    t = torch.zeros(len(rows), dtype=torch.int32, device=DEV)
    for part in (z, z[:1], z[3:5], z[6:7]):            # few rows: a row is shared by several blocks
        _check(part, t[:part.shape[0]], 20, 1.0, disc.disc_logprobs(part, t[:part.shape[0]], top=20))


def test_lowest_values_and_rows_without_mass_or_with_nan():
    V = 5000
    z = torch.randn((6, V), device=DEV)
    z[0] = -math.inf
    z[1, 7] = math.nan
    z[2, 9] = math.inf
    z[3] = torch.finfo(torch.float32).min / 2          # large masked values everywhere
    z[3, 11] = 0.0
    z[4] = math.nan
    z[5, 100:] = -math.inf
    t = torch.tensor([3, 3, 3, 11, 3, 4000], dtype=torch.int32, device=DEV)
    for rep in (z, z.bfloat16()):
        r = disc.disc_logprobs(rep, t, top=4)
        assert r["status"].tolist() == [disc.ROW_NOMASS, disc.ROW_NONFINITE, disc.ROW_NONFINITE, 0, disc.ROW_NONFINITE, 0]
        assert r["lse"][0] == -math.inf and r["logp"][0] == -math.inf and r["entropy"][0] == 0
        assert torch.all(r["top_logp"][0] == -math.inf) and r["top_ids"][0].tolist() == [0, 1, 2, 3]
        assert math.isnan(r["lse"][1]) and r["lse"][2] == math.inf
        assert r["logp"][3] == 0 and r["entropy"][3] == 0 and r["lse"][3] == 0
        assert r["top_ids"][4].tolist() == [0, 1, 2, 3] and r["top_ids"][2][0] == 9
        assert r["logp"][5] == -math.inf
        for i in range(6):
            assert r["top_ids"][i].tolist() == _order(rep[i])[:4].tolist()
        lse, H = disc.disc_logprobs(rep, t)["lse"], r["entropy"]
        g = disc.disc_logprobs_grad(rep, t, lse, H, torch.ones(6, device=DEV), torch.ones(6, device=DEV))
        assert torch.all(g[0] == 0) and torch.isfinite(g[3]).all() and torch.isfinite(g[5]).all()
        assert torch.all(g[5, 101:4000] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_the_lowest_value(dtype):
    """Masks of the type's lowest value: everywhere (an even distribution), and everywhere but at three tokens."""
    V, low = 3000, torch.finfo(dtype).min
    z = torch.full((3, V), low, dtype=dtype, device=DEV)
    z[1, [5, 2000, 2999]] = torch.tensor([1.0, 2.0, 0.5], dtype=dtype, device=DEV)
    z[2, 7] = torch.finfo(dtype).max
    t = torch.tensor([4, 2000, 7], dtype=torch.int32, device=DEV)
    r = disc.disc_logprobs(z, t, top=3)
    assert torch.all(r["status"] == 0)
    even = math.log(V)
    assert r["lse"][0] == low and abs(float(r["entropy"][0]) - even) < 1e-5
    _check(z[1:2], t[1:2], 3, 1.0, {k: x[1:2] for k, x in r.items()})
    assert r["logp"][2] == 0 and r["entropy"][2] == 0
    assert r["top_ids"].tolist() == [[0, 1, 2], [2000, 5, 2999], [7, 0, 1]]
    one = torch.ones(3, device=DEV)
    g = disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], one, None)
    # with lse rounded to fp32 the even row's probabilities are 1 each there; what counts is that the rows stay finite
    assert torch.isfinite(g).all() and g[2].abs().max() == 0
    p = torch.softmax(z[1].double(), dim=0)
    want = -p
    want[2000] += 1
    assert torch.all((g[1].double() - want).abs() <= UNIT[dtype] * want.abs() + 1e-6)


def test_targets_outside_the_vocabulary():
    z = torch.randn((3, 100), device=DEV)
    r = disc.disc_logprobs(z, torch.tensor([-1, 100, -2], dtype=torch.int32, device=DEV))
    assert r["logp"][0] == 0 and math.isnan(r["logp"][1]) and math.isnan(r["logp"][2])
    assert r["status"].tolist() == [0, disc.ROW_DEAD, disc.ROW_DEAD]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V,ld,offset", [(1, 1, 1, 0), (3, 7, 8, 1), (5, 1000, 1001, 3), (2, 32000, 32000, 0), (33, 4099, 4099, 0)])
def test_gradient_against_the_formula(dtype, n, V, ld, offset):
    z = _logits(n, V, dtype, 3 * n + V, ld, offset)
    gen = torch.Generator(device=DEV).manual_seed(V)
    t = torch.randint(0, V, (n,), generator=gen, dtype=torch.int32, device=DEV)
    t[n // 2] = -1
    a, b = torch.randn(n, generator=gen, device=DEV), torch.randn(n, generator=gen, device=DEV)
    inv_t = 0.8
    r = disc.disc_logprobs(z, t, inv_temperature=inv_t)
    lp = torch.log_softmax(z.double() * inv_t, dim=1)
    p = lp.exp()
    H = -(p * lp).sum(dim=1)
    one = torch.zeros_like(lp)
    one[torch.arange(n, device=DEV)[t >= 0], t[t >= 0].long()] = 1.0
    span = (z.double() * inv_t).abs().amax(dim=1)
    rel = (2.0 ** -20 + (V / 256 + 40) * 2.0 ** -24 + 2.0 ** -21 * span)[:, None]       # of a probability, and of lse and H
    for db in (b, None):
        a64 = torch.where(t >= 0, a, torch.zeros_like(a)).double()[:, None]
        b64 = torch.zeros_like(a64) if db is None else db.double()[:, None]
        want = ((one - p) * a64 - p * (lp + H[:, None]) * b64) * inv_t
        tol = inv_t * p * (rel * (a64.abs() + b64.abs() * (lp.abs() + H[:, None])) + b64.abs() * rel * (2 + 2 * math.log(V + 1)))
        tol = tol + UNIT[dtype] * want.abs() + 2.0 ** -23 * inv_t * a64.abs() * one + 1e-38
        got = disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], a, db, inv_temperature=inv_t)
        assert torch.all((got.double() - want).abs() <= tol)
        # in place, and into rows of another alignment
        other = _logits(n, V, dtype, 1, V + 3, 1)
        disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], a, db, inv_temperature=inv_t, out=other)
        assert torch.equal(other, got)
    z2 = z.clone()
    disc.disc_logprobs_grad(z2, t, r["lse"], r["entropy"], a, None, inv_temperature=inv_t, out=z2)
    assert torch.equal(z2, got)


def test_gradient_against_differences():
    """Central differences of the definition in 64 bits along random directions: the error of a difference of step h is
    h^2 / 6 times a third derivative, at most 40 |d|^3 here, plus what fp32 inputs allow."""
    n, V, h = 4, 97, 1e-4
    z = torch.randn((n, V), device=DEV) * 2
    t = torch.randint(0, V, (n,), dtype=torch.int32, device=DEV)
    a, b = torch.randn(n, device=DEV), torch.randn(n, device=DEV)

    def f(x):
        lp = torch.log_softmax(x, dim=1)
        return (a.double() * lp.gather(1, t.long()[:, None])[:, 0] - b.double() * (lp.exp() * lp).sum(dim=1)).sum()

    r = disc.disc_logprobs(z, t)
    g = disc.disc_logprobs_grad(z, t, r["lse"], r["entropy"], a, b).double()
    for k in range(8):
        d = torch.nn.functional.one_hot(torch.tensor([k * 11] * n, device=DEV), V).double() if k < 4 else torch.randn((n, V), device=DEV, dtype=torch.float64)
        diff = (f(z.double() + h * d) - f(z.double() - h * d)) / (2 * h)
        assert abs(float(diff - (g * d).sum())) <= 40 * h * h * float(d.abs().max()) ** 3 * n + 1e-5 * float(d.abs().sum())


def test_refusals():
    z = torch.randn((4, 100), device=DEV)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    with pytest.raises(disc.DiscError):
        disc.disc_logprobs(z.half(), t)
    with pytest.raises(disc.DiscError):
        disc.disc_logprobs(z, t, top=65)
    with pytest.raises(disc.DiscError):
        disc.disc_logprobs(z, t, inv_temperature=0.0)
    with pytest.raises(TypeError):
        disc.disc_logprobs(z, t[:3])
    with pytest.raises(TypeError):
        disc.disc_logprobs(z.t(), t)
    with pytest.raises(TypeError):
        disc.disc_logprobs(z, t.long())
    r = disc.disc_logprobs(z, t)
    with pytest.raises(disc.DiscError):
        disc.disc_logprobs_grad(z, None, r["lse"], r["entropy"], torch.ones(4, device=DEV))
    with pytest.raises(disc.DiscError):
        disc.disc_logprobs_grad(z, t, r["lse"], None, torch.ones(4, device=DEV), torch.ones(4, device=DEV))
    assert disc.disc_logprobs(z[:0], t[:0])["lse"].numel() == 0


def test_on_another_stream_and_the_same_twice():
    z = _logits(500, 20000, torch.bfloat16, 5)
    t = torch.randint(0, 20000, (500,), dtype=torch.int32, device=DEV)
    a = disc.disc_logprobs(z, t, top=7)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = disc.disc_logprobs(z, t, top=7)
    c = disc.disc_logprobs(z, t, top=7, stream=s)
    torch.cuda.synchronize()
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k])
