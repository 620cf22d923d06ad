"""disc_attend_plan / disc_attend_cached against attention in 64 bits over the rows' tokens."""
import math

import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from model_ops_reference import assert_attend, attend64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def build(lens, page, hkv, d, dtype, *, group=1, shared=None, layers=1, seed=0, spare=3, first_page=0, scale=1.0):
    """A cache whose rows have these lengths; `shared[q]` leading pages of the rows of group q are the same.  Every place that
    holds no token of a row is NaN."""
    rng = np.random.default_rng(seed)
    rows = len(lens)
    used = [-(-n // page) for n in lens]
    width = max(max(used), 1) + 1
    table = np.full((rows, width), -1, np.int32)
    n_pages = first_page + sum(used) + spare
    ids = list(first_page + rng.permutation(n_pages - first_page))
    for r in range(rows):
        s = 0
        if shared is not None and r % group:
            s = min(shared[r // group], used[r])
            table[r, :s] = table[r - r % group, :s]
        for j in range(s, used[r]):
            table[r, j] = ids.pop()
    gen = torch.Generator(device=DEV).manual_seed(seed)
    pool = torch.full((layers, 2, n_pages, hkv, page, d), math.nan, dtype=dtype, device=DEV)
    filled = np.zeros(n_pages, np.int64)
    for r in range(rows):
        for j in range(used[r]):
            filled[table[r, j]] = max(filled[table[r, j]], min(page, lens[r] - j * page))
    f = torch.as_tensor(filled, device=DEV)
    for l in range(layers):
        for i in range(2):
            for a in range(first_page, n_pages, 4096):
                x = torch.randn((min(4096, n_pages - a), hkv, page, d), generator=gen, device=DEV) * scale
                x.masked_fill_(torch.arange(page, device=DEV)[None, None, :, None] >= f[a:a + 4096, None, None, None], math.nan)
                pool[l, i, a:a + 4096] = x.to(dtype)
    ref = np.bincount(table[table >= 0].ravel(), minlength=n_pages).astype(np.int32)
    book = torch.as_tensor(np.concatenate([table.ravel(), np.asarray(lens, np.int32), ref])).to(DEV)
    return disc.DiscCache(pool, rows, width, book=book), table


def tokens(cache, table, r, n, layer):
    P = cache.page_size
    ids = torch.as_tensor(table[r, :-(-n // P)].astype(np.int64), device=DEV)
    kv = cache.pool[layer][:, ids]                                        # [2, pages, heads, P, d]
    return kv.permute(0, 1, 3, 2, 4).reshape(2, -1, cache.n_kv_heads, cache.head_dim)[:, :n]


def check(cache, table, lens, hq, group, *, layer=0, rows=None, q=None, seed=1, scale=None):
    d = cache.head_dim
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if q is None:
        q = torch.randn((len(lens), hq, d), generator=gen, device=DEV).to(cache.pool.dtype)
    scale = 1 / math.sqrt(d) if scale is None else scale
    plan = disc.disc_attend_plan(cache, hq, group=group)
    out, lse = disc.disc_attend_cached(cache, layer, q, plan, scale=scale)
    disc.disc_attend_check(plan=plan)
    again, lse2 = disc.disc_attend_cached(cache, layer, q, plan, scale=scale)       # the plan serves every layer, and the bits are the same
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    for r in range(len(lens)) if rows is None else rows:
        k, v = tokens(cache, table, r, lens[r], layer)
        assert_attend(out[r:r + 1], lse[r:r + 1], attend64(q[r:r + 1], k, v, scale, [lens[r]]))
    return out, lse


LENS = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128, 129, 200]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 2, 128), (3, 1, 40), (14, 2, 72), (16, 1, 128), (64, 1, 64), (40, 2, 8)])
def test_unrelated_rows(dtype, page, hq, hkv, d):
    cache, table = build(LENS, page, hkv, d, dtype, seed=page + hq)
    check(cache, table, LENS, hq, 1)


@pytest.mark.parametrize("dtype,page,hq,hkv,d,group", [
    (torch.bfloat16, 16, 4, 4, 64, 4), (torch.bfloat16, 16, 8, 2, 128, 16), (torch.float16, 32, 8, 2, 128, 7), (torch.bfloat16, 64, 6, 2, 80, 32),
    (torch.bfloat16, 16, 16, 1, 128, 8), (torch.float16, 128, 4, 1, 64, 33), (torch.bfloat16, 16, 64, 1, 128, 3), (torch.bfloat16, 16, 4, 4, 128, 100)])
def test_candidates_that_share_a_prompt(dtype, page, hq, hkv, d, group):
    rng = np.random.default_rng(group)
    queries = 5
    shared = [0, 1, 3, 9, 2]
    lens = []
    for s in shared:
        lens += [int(s * page + x) for x in rng.integers(0, 40, group)]
    lens[group] = shared[1] * page                         # a candidate with nothing of its own
    lens = lens[:len(lens) - group // 2]                   # the last query has fewer
    cache, table = build(lens, page, hkv, d, dtype, group=group, shared=shared, seed=group, layers=2)
    for layer in (0, 1):
        check(cache, table, lens, hq, group, layer=layer)
    # rows of one query that stand alone give the same to within the bounds
    check(cache, table, lens, hq, 1)


def test_empty_rows_among_candidates_and_an_empty_cache():
    lens = [0, 40, 0, 33, 0, 0, 0, 0]
    cache, table = build(lens, 16, 2, 64, torch.bfloat16, group=4, shared=[0, 0])
    check(cache, table, lens, 4, 4)
    cache, table = build([0, 0, 0], 16, 2, 64, torch.bfloat16)
    check(cache, table, [0, 0, 0], 4, 1)


@pytest.mark.parametrize("lens,hq,hkv", [([20011], 4, 4), ([9000, 1, 5003], 8, 1), ([131072 + 5], 8, 2)])
def test_long_rows_are_split_and_joined(lens, hq, hkv):
    cache, table = build(lens, 64, hkv, 128, torch.bfloat16, seed=3)
    check(cache, table, lens, hq, 1)
    check(cache, table, lens, hq, 1, scale=1.5)            # a few tokens carry most of the weight


def test_long_shared_prompts_are_split_too():
    shared, lens = [300], [300 * 16 + x for x in (1, 30, 0, 17, 16, 5)]
    cache, table = build(lens, 16, 1, 128, torch.bfloat16, group=6, shared=shared)
    check(cache, table, lens, 8, 6)


def test_many_rows():
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 300, 1500)]
    cache, table = build(lens, 16, 2, 64, torch.bfloat16)
    check(cache, table, lens, 8, 1, rows=range(0, 1500, 37))


def test_a_candidate_with_non_finite_values_does_not_touch_the_others():
    group, page = 8, 16
    lens = [32 + 9] * group
    cache, table = build(lens, page, 2, 64, torch.bfloat16, group=group, shared=[2])
    q = torch.randn((group, 8, 64), device=DEV).bfloat16()
    plan = disc.disc_attend_plan(cache, 8, group=group)
    clean, _ = disc.disc_attend_cached(cache, 0, q, plan)
    cache.pool[0, 1, int(table[3, 2]), :, 4] = math.inf
    cache.pool[0, 0, int(table[5, 2]), :, 2] = math.nan
    out, lse = disc.disc_attend_cached(cache, 0, q, plan)
    for r in range(group):
        if r in (3, 5):
            assert not torch.isfinite(out[r]).all()
        else:
            assert torch.equal(out[r], clean[r])


def test_places_beyond_32_bit_offsets():
    """4.4e9 values of keys and values: the used pages lie in the last ones."""
    n = (1 << 31) // (2 * 128 * 128) + 70000
    lens = [700, 5]
    cache, table = build(lens, 128, 2, 128, torch.bfloat16, first_page=n)
    assert cache.pool.numel() > 1 << 32
    check(cache, table, lens, 4, 1)


def test_strided_queries_and_another_stream():
    lens = [100, 33]
    cache, table = build(lens, 16, 2, 64, torch.bfloat16)
    wide = torch.randn((2, 20, 72), device=DEV).bfloat16()
    q = wide[:, 3:11, :64]
    out, _ = check(cache, table, lens, 8, 1, q=q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        plan = disc.disc_attend_plan(cache, 8)
        b, _ = disc.disc_attend_cached(cache, 0, q, plan)
    torch.cuda.synchronize()
    assert torch.equal(out, b)


def test_refusals():
    cache, _ = build([5, 6], 16, 2, 64, torch.bfloat16)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_plan(cache, 3)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_plan(cache, 2 * 65)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_plan(cache, 4, group=0)
    plan = disc.disc_attend_plan(cache, 4)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_cached(cache, 0, q, plan, scale=0.0)
    with pytest.raises(TypeError):
        disc.disc_attend_cached(cache, 0, q.half(), plan)
    with pytest.raises(TypeError):
        disc.disc_attend_cached(cache, 0, q[:1], plan)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_cached(cache, 1, q, plan)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_cached(cache, 0, torch.zeros((2, 4, 68), dtype=torch.bfloat16, device=DEV)[:, :, 2:66], plan)
