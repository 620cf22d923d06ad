"""Groups of more than 16 query vectors with enough rows that a warp of the joining kernel takes two key heads of a row."""
import math

import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from test_gpu_attend_cached import build, check

pytestmark = pytest.mark.gpu
DEV = "cuda"


def groups(rows, group, page, seed):
    """Rows of few tokens; among them rows that end on a block, rows with nothing of their own, empty ones."""
    rng = np.random.default_rng(seed)
    n = -(-rows // group)
    shared = [int(x) for x in rng.integers(0, 5, n)]
    lens = []
    for r in range(rows):
        own = int(rng.choice([0, 1, 5, 15, 16, 17, 32, 40, 160]))
        lens.append(shared[r // group] * page + own)
    for g in range(0, n, 7):                                  # a group without common pages, one of its rows empty
        shared[g] = 0
        lens[g * group] = 0
    return lens, shared


@pytest.mark.parametrize("dtype,rows,group,hq,hkv,d,page", [
    (torch.bfloat16, 1300, 20, 9, 3, 64, 16), (torch.bfloat16, 1999, 13, 8, 2, 128, 32), (torch.float16, 1200, 20, 9, 3, 72, 16),
    (torch.bfloat16, 900, 6, 44, 4, 128, 16), (torch.float16, 800, 3, 105, 5, 40, 64)])
def test_two_key_heads_in_a_warp(dtype, rows, group, hq, hkv, d, page):
    lens, shared = groups(rows, group, page, rows)
    cache, table = build(lens, page, hkv, d, dtype, group=group, shared=shared, seed=rows)
    some = list(range(0, 2 * group)) + list(range(7 * group, 7 * group + 2)) + list(range(3, rows, 41)) + [rows - 1]
    check(cache, table, lens, hq, group, rows=some)


def test_non_finite_values_stay_with_their_row():
    rows, group, hq, hkv, d = 1300, 20, 9, 3, 64
    lens = [32 + 9] * rows
    cache, table = build(lens, 16, hkv, d, torch.bfloat16, group=group, shared=[2] * (rows // group))
    q = torch.randn((rows, hq, d), device=DEV).bfloat16()
    plan = disc.disc_attend_plan(cache, hq, group=group)
    clean, clean_lse = disc.disc_attend_cached(cache, 0, q, plan)
    cache.pool[0, 1, int(table[45, 2]), :, 4] = math.inf
    cache.pool[0, 0, int(table[700, 2]), 1, 2] = math.nan
    out, lse = disc.disc_attend_cached(cache, 0, q, plan)
    keep = torch.ones(rows, dtype=torch.bool, device=DEV)
    keep[[45, 700]] = False
    assert torch.equal(out[keep], clean[keep]) and torch.equal(lse[keep], clean_lse[keep])
    assert not torch.isfinite(out[45]).any()
    assert torch.isfinite(out[700, :3]).all() and not torch.isfinite(out[700, 3:6]).any() and torch.isfinite(out[700, 6:]).all()
