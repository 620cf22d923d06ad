"""A frequency that is not finite: position times frequency has no sine, and the pair's values are NaN, as in the definition."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (128, 128, True), (72, 40, False), (64, 64, True)])
def test_the_pair_is_nan_and_nothing_else_changes(d, rot, inter, bad):
    g = torch.Generator(device=DEV).manual_seed(4)
    q, k = (torch.randn((9, h, d), generator=g, device=DEV).bfloat16() for h in (4, 2))
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    pos = torch.arange(9, dtype=torch.int32, device=DEV) * 7         # the first is 0: 0 times infinity is NaN
    half = rot // 2
    freq = torch.exp(torch.arange(half, device=DEV) * (-0.1))
    how = dict(norm=False, interleaved=inter)
    want = disc.disc_norm_rope(q, k, pos, freq, **how) + disc.disc_norm_rope_grad(q, k, pos, freq, dq, dk, **how)[:2]
    i = half - 1                       # also the last pair, of another lane's half where there are more than 32
    for at in {0, i}:
        spoiled = freq.clone()
        spoiled[at] = bad
        got = disc.disc_norm_rope(q, k, pos, spoiled, **how) + disc.disc_norm_rope_grad(q, k, pos, spoiled, dq, dk, **how)[:2]
        pair = [2 * at, 2 * at + 1] if inter else [at, at + half]
        others = [c for c in range(d) if c not in pair]
        for a, b in zip(got, want):
            assert torch.isnan(a[..., pair]).all()
            assert torch.equal(a[..., others], b[..., others])
