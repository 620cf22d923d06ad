"""disc_attend_cached over a cache held in 8 bits against attention in 64 bits over the values that are held."""
import math

import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from held_reference import held_rows, tol_held
from model_ops_reference import UNIT, attend64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def vectors(n, heads, d, dtype, seed, spread):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g, device=DEV) * torch.exp(spread * torch.randn((n, heads, 1), generator=g, device=DEV))
    return x.to(dtype)


def build(prompts, own, K, *, held, dtype, d, hkv, page, seed=0, spread=0.5, layers=1):
    """K rows for each prompt; row q K + c has the prompt's tokens, in shared pages, and own[q K + c] tokens of its own."""
    rows = K * len(prompts)
    longest = max(prompts) + max(list(own) + [0])
    n_pages = sum(-(-n // page) for n in prompts) + sum(-(-n // page) + 1 for n in own) + 3
    cache = disc.DiscCache.empty(layers, n_pages, page, hkv, d, rows, -(-longest // page) + 2, dtype=dtype, held=held)
    cache.pool.fill_(0x80)                     # exponents of NaN wherever no token is
    heads = i32([q * K for q in range(len(prompts))])
    add = torch.zeros(rows, dtype=torch.int32, device=DEV)
    add[::K] = i32(list(prompts))
    assert int(disc.disc_cache_extend(cache, add).max()) == 0
    cu = i32(np.concatenate([[0], np.cumsum(prompts)]).tolist())
    n = sum(prompts)
    for layer in range(layers):
        disc.disc_cache_write(cache, layer, vectors(n, hkv, d, dtype, seed + 1 + layer, spread), vectors(n, hkv, d, dtype, seed + 11 + layer, spread), cu=cu, rows=heads)
    if K > 1:
        disc.disc_cache_fork(cache, heads.repeat_interleave(K))
    if max(list(own) + [0]):
        assert int(disc.disc_cache_extend(cache, i32(list(own))).max()) == 0
        cu = i32(np.concatenate([[0], np.cumsum(own)]).tolist())
        n = sum(own)
        for layer in range(layers):
            disc.disc_cache_write(cache, layer, vectors(n, hkv, d, dtype, seed + 21 + layer, spread), vectors(n, hkv, d, dtype, seed + 31 + layer, spread), cu=cu)
    return cache


def queries(cache, hq, seed=5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn((cache.n_rows, hq, cache.head_dim), generator=g, device=DEV).to(cache.dtype)


def check(cache, q, group, *, layer=0, rows=None, scale=None, skip=()):
    plan = disc.disc_attend_plan(cache, q.shape[1], group=group)
    out, lse = disc.disc_attend_cached(cache, layer, q, plan, scale=scale)
    disc.disc_attend_check(plan=plan)
    scale = 1 / math.sqrt(cache.head_dim) if scale is None else scale
    lens = cache.len.tolist()
    assert out.dtype == cache.dtype and out.shape == q.shape
    for r in rows if rows is not None else range(cache.n_rows):
        if r in skip:
            continue
        if lens[r] == 0:
            assert bool((out[r] == 0).all()) and bool((lse[r] == -math.inf).all())
            continue
        k, v = (torch.as_tensor(x, device=DEV) for x in held_rows(cache, layer, r, lens[r]))
        o, l, to, tl = attend64(q[r:r + 1], k, v, scale, [lens[r]])
        to = to + tol_held(k, v, q[r].double(), scale, UNIT[q.dtype])[None]
        err = (out[r:r + 1].double() - o).abs()
        assert torch.all(err <= to), (r, float((err - to).max()), float(err.max()))
        err = (lse[r:r + 1].double() - l).abs()
        assert torch.all(err <= tl), (r, float((err - tl).max()))
    return out, lse


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,hq,hkv,d,page", [
    ([1], 1, 1, 16, 16), ([16, 17, 15, 0, 1, 33], 4, 1, 64, 16), ([300, 1, 0, 129], 16, 2, 128, 32), ([2000, 3], 4, 4, 80, 64),
    ([65, 64, 63], 32, 2, 112, 128), ([700], 12, 1, 128, 16), ([5] * 40, 3, 1, 96, 16)])
def test_rows_alone(lens, hq, hkv, d, page, dtype, held):
    cache = build(lens, [0] * len(lens), 1, held=held, dtype=dtype, d=d, hkv=hkv, page=page)
    check(cache, queries(cache, hq), 1)


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("prompts,K,hq,hkv,d,page", [
    ([40, 100], 2, 8, 2, 128, 16), ([33, 1, 80], 4, 2, 1, 64, 16), ([500], 4, 8, 2, 128, 32), ([64, 65], 8, 2, 1, 80, 64), ([200, 16], 16, 2, 2, 64, 16)])
def test_rows_that_share(prompts, K, hq, hkv, d, page, dtype, held):
    own = [(3 * i) % 20 for i in range(K * len(prompts))]
    cache = build(prompts, own, K, held=held, dtype=dtype, d=d, hkv=hkv, page=page)
    check(cache, queries(cache, hq), K)


GROUPS = [([400, 90], 8, 16, 4, 128, 16), ([130], 32, 16, 4, 128, 32), ([1, 70, 300], 5, 16, 1, 64, 64), ([260], 3, 64, 1, 80, 16), ([800, 5], 40, 4, 1, 128, 16),
          ([64, 192], 6, 32, 2, 112, 128)]


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("prompts,K,hq,hkv,d,page", GROUPS)
def test_many_query_vectors(prompts, K, hq, hkv, d, page, dtype, held):
    own = [(7 * i) % 30 + (200 if i == 2 else 0) for i in range(K * len(prompts))]
    cache = build(prompts, own, K, held=held, dtype=dtype, d=d, hkv=hkv, page=page)
    rows = range(cache.n_rows) if cache.n_rows <= 30 else [0, 1, 2, 3, 17, cache.n_rows - 2, cache.n_rows - 1]
    check(cache, queries(cache, hq), K, rows=rows)


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("K,hq,hkv", [(1, 4, 1), (2, 16, 4), (6, 16, 2)])
def test_values_whose_sizes_differ_widely(K, hq, hkv, held):
    """Tokens' values from 2^-12 to 2^12 times the usual: the large ones must not push the others out of f16."""
    cache = build([150] * 2, [5] * 2 * K if K > 1 else [0, 0], K, held=held, dtype=torch.bfloat16, d=64, hkv=hkv, page=16, spread=4.0)
    check(cache, queries(cache, hq), K)


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("K,hq,hkv", [(1, 4, 1), (2, 16, 4), (8, 16, 2)])
def test_a_vector_that_is_not_finite_reaches_its_own_rows_alone(K, hq, hkv, held):
    cache = build([100] * 2, [9] * 2 * K if K > 1 else [0, 0], K, held=held, dtype=torch.bfloat16, d=64, hkv=hkv, page=16)
    q = queries(cache, hq)
    want, want_lse = check(cache, q, K)
    row = K - 1
    last = int(cache.len[row]) - 1
    for kv in range(2):
        pool = cache.pool.clone()
        page_id = int(cache.table[row, last // 16])
        pool[0, kv, page_id, 0, 16 * 64 + last % 16] = 0x80
        sick = disc.DiscCache(pool, cache.n_rows, cache.table_width, book=cache.book, held=held, page_size=16)
        plan = disc.disc_attend_plan(sick, hq, group=K)
        out, lse = disc.disc_attend_cached(sick, 0, q, plan)
        G = hq // hkv
        others = [r for r in range(cache.n_rows) if r != row]
        assert torch.isnan(out[row, :G]).all() and bool(torch.isnan(lse[row, :G]).all()) == (kv == 0)
        assert torch.equal(out[others], want[others]) and torch.equal(lse[others], want_lse[others])
        assert torch.equal(out[row, G:], want[row, G:])


def test_strides_scales_layers_and_queries_of_any_size():
    cache = build([90, 20, 200], [0] * 3, 1, held="e4m3", dtype=torch.bfloat16, d=128, hkv=2, page=16, layers=3)
    wide = torch.randn((3, 20, 128), device=DEV).bfloat16()
    check(cache, wide[:, 4:12], 1, layer=2, scale=0.3)
    check(cache, wide[:, :1].expand(3, 8, 128), 1, layer=1)
    for size in (1e-30, 1e-4, 300.0):
        check(cache, (wide[:, :8].float() * size).bfloat16(), 1, layer=1, scale=min(1.0, 1 / size))
    zero = torch.zeros((3, 8, 128), dtype=torch.bfloat16, device=DEV)
    check(cache, zero, 1)


def test_long_rows_are_split_the_same_way_every_time():
    cache = build([6000, 1, 3000], [0] * 3, 1, held="e4m3", dtype=torch.bfloat16, d=128, hkv=2, page=64)
    q = queries(cache, 8)
    out, lse = check(cache, q, 1, rows=[1, 2])
    for _ in range(3):
        again = disc.disc_attend_cached(cache, 0, q, disc.disc_attend_plan(cache, 8))
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("K,hq", [(1, 4), (16, 8)])
def test_captured(K, hq):
    cache = build([100, 50], [8] * 2 * K if K > 1 else [0, 0], K, held="i8", dtype=torch.float16, d=64, hkv=2, page=16)
    q = queries(cache, hq)
    want = check(cache, q, K, rows=[0, 1])
    plan = disc.disc_attend_plan(cache, hq, group=K)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        disc.disc_attend_plan(cache, hq, group=K, plan=plan)
        got = disc.disc_attend_cached(cache, 0, q, plan)
    for _ in range(2):
        got[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_plan_is_for_one_way_of_holding():
    a = build([20], [0], 1, held="e4m3", dtype=torch.bfloat16, d=64, hkv=1, page=16)
    b = build([20], [0], 1, held="i8", dtype=torch.bfloat16, d=64, hkv=1, page=16)
    q = queries(a, 2)
    plan = disc.disc_attend_plan(a, 2)
    with pytest.raises(TypeError):
        disc.disc_attend_cached(b, 0, q, plan)
    with pytest.raises(TypeError):
        disc.disc_attend_cached(a, 0, q.half(), plan)
