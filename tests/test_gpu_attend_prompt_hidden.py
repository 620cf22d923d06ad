"""Non-finite keys and values at tokens that a query does not see do not reach it, wherever they lie in a block of 128 keys."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc
from model_ops_reference import assert_attend, attend64
from test_gpu_attend_prompt import cu_of, make

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128), (7, 1, 72), (40, 1, 8)])
@pytest.mark.parametrize("at", [[0], [1], [63, 64], [127], [128], [200], [255, 256], [298], [299], [5, 130, 290]])
def test_later_tokens(dtype, hq, hkv, d, at):
    n = 300
    q, k, v = make(n, hq, d, dtype, 1), make(n, hkv, d, dtype, 2), make(n, hkv, d, dtype, 3)
    clean, clean_lse = disc.disc_attend_prompt(q, k, v, cu_of([n]), max_len=n)
    bad = v.clone()
    for i, x in zip(at, (math.inf, math.nan, -math.inf)):
        bad[i] = x
    out, lse = disc.disc_attend_prompt(q, k, bad, cu_of([n]), max_len=n)
    assert torch.equal(lse, clean_lse)
    first = at[0]
    sees = [j + 1 for j in range(first)]
    assert_attend(out[:first], lse[:first], attend64(q[:first], k, v, 1 / math.sqrt(d), sees) if first else (out[:0].double(), lse[:0].double(), out[:0].double(), lse[:0].double()))
    assert not torch.isfinite(out[first]).any()
    # later queries see the first of them; p = 0 for it is possible, but not that nothing is left of it: 0 times infinity is no number
    assert not torch.isfinite(out[first:]).any()
    # the key as well
    bad_k = k.clone()
    bad_k[first:] = math.nan
    out, lse = disc.disc_attend_prompt(q, bad_k, bad, cu_of([n]), max_len=n)
    assert torch.equal(lse[:first], clean_lse[:first]) and torch.isnan(lse[first:]).all()
    if first:
        assert_attend(out[:first], lse[:first], attend64(q[:first], k, v, 1 / math.sqrt(d), sees))


@pytest.mark.parametrize("causal", [True, False])
def test_more_keys_than_queries_and_values_in_other_places(causal):
    """Queries that follow a context: query j sees lk - lq + j + 1 keys."""
    lq, lk, hq, hkv, d = 70, 333, 8, 2, 64
    qkv = make(lk, 20, d, torch.bfloat16, 4)                 # strides of a fused projection
    q, k, v = make(lq, hq, d, torch.bfloat16, 1), qkv[:, 4:6], qkv[:, 10:12]
    clean = v.clone()
    qkv[300, 10:12] = math.inf
    out, lse = disc.disc_attend_prompt(q, k, v, cu_of([lq]), cu_of([lk]), max_len=lq, causal=causal)
    see = lk - lq + 1 + torch.arange(lq)
    before = int((see <= 300).sum()) if causal else 0
    assert (before > 0) == causal
    if causal:
        assert_attend(out[:before], lse[:before], attend64(q[:before], k, clean, 1 / math.sqrt(d), see[:before].tolist()))
    assert not torch.isfinite(out[before:]).any()


def test_a_sequence_of_nothing_but_nan_ends():
    n, hq, hkv, d = 3000, 8, 2, 128
    q, k = make(n, hq, d, torch.bfloat16, 1), make(n, hkv, d, torch.bfloat16, 2)
    v = torch.full((n, hkv, d), math.nan, dtype=torch.bfloat16, device=DEV)
    out, _ = disc.disc_attend_prompt(q, k, v, cu_of([n]), max_len=n)
    v = make(n, hkv, d, torch.bfloat16, 3)
    v[1::2] = math.inf
    out2, _ = disc.disc_attend_prompt(q, k, v, cu_of([n]), max_len=n)
    v[:] = 1.0
    v[n // 2:] = math.nan
    out3, _ = disc.disc_attend_prompt(q, k, v, cu_of([n]), max_len=n)
    disc.disc_attend_check()
    assert torch.isnan(out).all() and torch.isfinite(out2[0]).all() and not torch.isfinite(out2[1:]).any()
    assert torch.all((out3[:n // 2].float() - 1).abs() <= 2.0 ** -8) and torch.isnan(out3[n // 2:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_values_beside_infinite_ones_that_are_seen(dtype):
    """Token 20 has an infinite value at place 5, token 40 at places 9 and 100, and token 41 a NaN at place 5: query 30 sees the first
    only, and all its values but the one at place 5 are finite."""
    n, hq, hkv, d = 200, 4, 2, 128
    q, k, v = make(n, hq, d, dtype, 1), make(n, hkv, d, dtype, 2), make(n, hkv, d, dtype, 3)
    bad = v.clone()
    bad[20, :, 5] = math.inf
    bad[40, :, 9] = -math.inf
    bad[40, :, 100] = math.inf
    bad[41, :, 5] = math.nan
    out, lse = disc.disc_attend_prompt(q, k, bad, cu_of([n]), max_len=n)
    rest = torch.ones(d, dtype=torch.bool, device=DEV)
    rest[[5, 9, 100]] = False
    o, l, to, tl = attend64(q, k, v, 1 / math.sqrt(d), list(range(1, n + 1)))
    assert torch.all((lse.double() - l).abs() <= tl)
    err = (out.double() - o).abs()
    assert torch.all(err[:20] <= to[:20])
    assert torch.all(err[:, :, rest] <= to[:, :, rest])
    assert torch.all(err[:40, :, 9] <= to[:40, :, 9]) and torch.all(err[:40, :, 100] <= to[:40, :, 100])
    assert not torch.isfinite(out[20:, :, 5]).any() and not torch.isfinite(out[40:, :, 9]).any() and not torch.isfinite(out[40:, :, 100]).any()
