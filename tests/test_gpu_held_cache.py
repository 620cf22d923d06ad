"""A cache held in 8 bits: what is written, what is read back, what fork, extend and compact do with it."""
import math

import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from held_reference import hold64, norm_rope64, parts, place, tol_forward, values64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def cache_of(lens, *, held, dtype, d, hkv, page, layers=1, rows=None, extra=4):
    rows = rows or len(lens)
    n_pages = sum(-(-n // page) for n in lens) + extra
    cache = disc.DiscCache.empty(layers, n_pages, page, hkv, d, rows, max(-(-n // page) for n in lens) + 2, dtype=dtype, held=held)
    cache.pool.fill_(0x80)                       # exponents of NaN wherever no token is
    add = i32(list(lens) + [0] * (rows - len(lens)))
    assert int(disc.disc_cache_extend(cache, add).max()) == 0
    return cache


def vectors(n, heads, d, dtype, seed=0, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g, device=DEV) * torch.exp(spread * torch.randn((n, heads, 1), generator=g, device=DEV))
    return x.to(dtype)


def cu_of(lens):
    return i32(np.concatenate([[0], np.cumsum(lens)]).tolist())


SHAPES = [("e4m3", torch.bfloat16, 128, 2, 16), ("i8", torch.bfloat16, 64, 3, 32), ("e4m3", torch.float16, 80, 1, 64), ("i8", torch.float16, 112, 4, 128),
          ("e4m3", torch.bfloat16, 16, 5, 16), ("i8", torch.bfloat16, 96, 2, 16)]


@pytest.mark.parametrize("held,dtype,d,hkv,page", SHAPES)
def test_codes_and_values(held, dtype, d, hkv, page):
    lens = [1, page, page + 1, 0, 3 * page - 1, 7]
    cache = cache_of(lens, held=held, dtype=dtype, d=d, hkv=hkv, page=page, layers=2)
    n = sum(lens)
    fused = vectors(n, 3 * hkv, d, dtype, spread=4.0)
    k, v = fused[:, hkv:2 * hkv], fused[:, 2 * hkv:]
    before = cache.pool.clone()
    disc.disc_cache_write(cache, 1, k, v, cu=cu_of(lens))
    assert torch.equal(cache.pool[0], before[0])
    code, e = parts(cache)
    written = np.zeros(e.shape, bool)
    at = 0
    for r, m in enumerate(lens):
        for i in range(m):
            page_id, off = place(cache, r, i)
            for kv, x in enumerate((k, v)):
                want_c, want_e = hold64(x[at].double().cpu().numpy(), held)
                assert np.array_equal(code[1, kv, page_id, :, off], want_c) and np.array_equal(e[1, kv, page_id, :, off], want_e)
                written[1, kv, page_id, :, off] = True
            at += 1
    old = before.cpu().numpy()
    assert np.all(e[~written] == -128) and np.all(code[~written] == 0x80) and old.shape == cache.pool.shape
    # read back: exactly what the codes stand for, cut off at the type's largest value; f16 has infinities at this spread
    gk, gv = disc.disc_cache_read(cache, 1, cu_of(lens), n)
    big = float(torch.finfo(dtype).max)
    for got, x in ((gk, k), (gv, v)):
        want = np.clip(values64(*hold64(x.double().cpu().numpy(), held), held), -big, big)
        assert got.dtype == dtype and np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_borders_ties_and_values_that_are_not_finite(held, dtype):
    d, big = 16, torch.finfo(dtype).max
    tiny = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -24
    rows = [[0.0] * d, [448.0, 447.9, -432, 416, 17, 18, 19, -17] + [0.0] * 8, [449.0] + [1.0] * 15, [127.5, 63.5, 0.5, 1.5, -2.5] + [0.0] * 11,
            [127.0, 126.5, 0.5, 1.5, -0.5, -1.5] + [0.0] * 10, [big, -big, big / 2, 1.0] + [tiny] * 12, [tiny] * 8 + [-tiny, 0.0] * 4, [3 * tiny, -tiny] * 8,
            [math.nan] + [1.0] * 15, [1.0] * 15 + [math.inf], [-math.inf] * 16, [-0.0] * 16, [1.0, 1.0625, 1.125, 1.1875] * 4]
    x = torch.tensor(rows, dtype=torch.float64).to(dtype).to(DEV)[:, None, :]
    n = len(rows)
    cache = cache_of([n], held=held, dtype=dtype, d=d, hkv=1, page=16)
    disc.disc_cache_write(cache, 0, x, x.flip(0), cu=i32([0, n]))
    code, e = parts(cache)
    page_id = place(cache, 0, 0)[0]
    want_c, want_e = hold64(x[:, 0].double().cpu().numpy(), held)
    assert np.array_equal(e[0, 0, page_id, 0, :n], want_e)
    assert np.array_equal(code[0, 0, page_id, 0, :n], want_c)
    gk, gv = disc.disc_cache_read(cache, 0, i32([0, n]), n)
    want = np.clip(values64(want_c, want_e, held), -float(big), float(big))
    assert np.array_equal(gk[:, 0].double().cpu().numpy(), want, equal_nan=True) and np.array_equal(gv.flip(0)[:, 0].double().cpu().numpy(), want, equal_nan=True)
    assert np.all(np.isnan(want[8:11])) and np.all(want[[0, 11]] == 0)


@pytest.mark.parametrize("held", [None, "e4m3", "i8"])
def test_read_of_parts_of_rows(held):
    lens, page, d, hkv = [40, 5, 0, 77], 16, 64, 2
    cache = cache_of(lens, held=held, dtype=torch.bfloat16, d=d, hkv=hkv, page=page)
    k, v = vectors(sum(lens), hkv, d, torch.bfloat16, 1), vectors(sum(lens), hkv, d, torch.bfloat16, 2)
    disc.disc_cache_write(cache, 0, k, v, cu=cu_of(lens))
    full = disc.disc_cache_read(cache, 0, cu_of(lens), sum(lens))
    if held is None:
        assert torch.equal(full[0], k) and torch.equal(full[1], v)
    first = [0, 40, 45, 45]
    # row, from, how many; beyond the row's tokens and for rows that are none: zeros
    want = [(3, 16, 20), (0, 0, 40), (1, 3, 6), (2, 0, 2), (-1, 0, 3), (4, 0, 1), (3, 76, 1), (0, -2, 3), (3, 0, 0), (3, 1, 7)]
    n = sum(w[2] for w in want)
    out = tuple(torch.full((n + 9, hkv, d), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cu = cu_of([w[2] for w in want]) + 4
    got = disc.disc_cache_read(cache, 0, cu, n + 9, rows=i32([w[0] for w in want]), start=i32([w[1] for w in want]), out=out)
    for i in range(2):
        assert bool((got[i][:4] == 5).all() and (got[i][n + 4:] == 5).all())
        at = 4
        for r, s, m in want:
            for j in range(m):
                some = 0 <= r < 4 and 0 <= s + j < lens[r]
                assert torch.equal(got[i][at], full[i][first[r] + s + j] if some else torch.zeros_like(got[i][at])), (r, s, j)
                at += 1
    empty = disc.disc_cache_read(cache, 0, i32([0]), 0)
    assert empty[0].shape == (0, hkv, d)


@pytest.mark.parametrize("held,dtype,d,hkv,page", SHAPES[:4])
def test_fork_extend_and_compact_carry_the_vectors(held, dtype, d, hkv, page):
    K, lens = 3, [page + 5, 2 * page, 1]
    rows = K * len(lens)
    cache = disc.DiscCache.empty(2, 60, page, hkv, d, rows, 6, dtype=dtype, held=held)
    cache.pool.fill_(0x80)
    heads = i32([q * K for q in range(len(lens))])
    add = torch.zeros(rows, dtype=torch.int32, device=DEV)
    add[::K] = i32(lens)
    disc.disc_cache_extend(cache, add)
    said = []
    for layer in range(2):
        k, v = vectors(sum(lens), hkv, d, dtype, layer), vectors(sum(lens), hkv, d, dtype, 10 + layer)
        disc.disc_cache_write(cache, layer, k, v, cu=cu_of(lens), rows=heads)
        said.append((k, v))
    disc.disc_cache_fork(cache, heads.repeat_interleave(K))
    for step in range(2):
        disc.disc_cache_extend(cache)
        for layer in range(2):
            new = vectors(rows, hkv, d, dtype, 20 + 2 * step + layer), vectors(rows, hkv, d, dtype, 30 + 2 * step + layer)
            disc.disc_cache_write(cache, layer, *new)
            said.append(new)
    keep = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    keep[::K] = heads + i32([2, 0, 1])
    disc.disc_cache_fork(cache, keep)
    live = disc.disc_cache_compact(cache)
    total = [n + 2 for n in lens]
    assert int(live) == sum(-(-n // page) for n in total)
    for layer in range(2):
        got = disc.disc_cache_read(cache, layer, cu_of(total), sum(total), rows=heads)
        for kv in range(2):
            want, at = [], 0
            for q, n in enumerate(lens):
                chosen = q * K + [2, 0, 1][q]
                want += [said[layer][kv][at:at + n], said[2 + layer][kv][chosen:chosen + 1], said[4 + layer][kv][chosen:chosen + 1]]
                at += n
            want = torch.cat(want)
            exact = values64(*hold64(want.double().cpu().numpy(), held), held)
            assert np.array_equal(got[kv].double().cpu().numpy(), exact)


def frequencies(rot):
    return torch.exp(torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) * (-math.log(10000.0) / rot)).float()


@pytest.mark.parametrize("held", [None, "e4m3", "i8"])
@pytest.mark.parametrize("dtype,d,hq,hkv,page,inter", [(torch.bfloat16, 128, 16, 4, 16, False), (torch.float16, 64, 6, 3, 32, True), (torch.bfloat16, 80, 3, 1, 64, False)])
def test_norm_rope_write_is_the_two_calls(held, dtype, d, hq, hkv, page, inter):
    lens, new = [30, 1, 64, 0, 100], [3, 1, 17, 0, 1]
    old = [a - b for a, b in zip(lens, new)]
    a = cache_of(lens, held=held, dtype=dtype, d=d, hkv=hkv, page=page)
    b = cache_of(lens, held=held, dtype=dtype, d=d, hkv=hkv, page=page)
    n, freq = sum(new), frequencies(d // 16 * 8)
    q, k, v = vectors(n, hq + 2 * hkv, d, dtype, 5).split([hq, hkv, hkv], dim=1)
    qw, kw = torch.rand(d, device=DEV) + 0.5, torch.rand(d, device=DEV) + 0.5
    how = dict(q_weight=qw, k_weight=kw, interleaved=inter)
    pos = i32([o + j for o, m in zip(old, new) for j in range(m)])
    got = disc.disc_norm_rope_write(a, 0, q, k, v, freq, cu=cu_of(new), **how)
    q2, k2 = disc.disc_norm_rope(q, k, pos, freq, **how)
    disc.disc_cache_write(b, 0, k2, v, cu=cu_of(new))
    assert torch.equal(got, q2) and torch.equal(a.pool.view(torch.uint8), b.pool.view(torch.uint8))
    y, size = norm_rope64(q.double(), qw.double(), pos, freq, interleaved=inter)
    assert torch.all((got.double() - y).abs() <= tol_forward(y, size, dtype))
    # given positions, rows in another order, rows with a status and no queries at all
    pos2, rows = pos + 1000, i32([4, 0, 2, 3, 1])
    order = [4, 0, 2, 3, 1]
    cu = cu_of([new[r] for r in order])
    status = torch.zeros(5, dtype=torch.uint8, device=DEV)
    status[2] = 32
    got = disc.disc_norm_rope_write(a, 0, q, k, v, freq, positions=pos2, cu=cu, rows=rows, status=status, out=None, **how)
    q2, k2 = disc.disc_norm_rope(q, k, pos2, freq, **how)
    disc.disc_cache_write(b, 0, k2, v, cu=cu, rows=rows, status=status)
    assert torch.equal(got, q2) and torch.equal(a.pool.view(torch.uint8), b.pool.view(torch.uint8))
    assert disc.disc_norm_rope_write(a, 0, None, k2, v, None, norm=False, cu=cu, rows=rows) is None
    disc.disc_cache_write(b, 0, k2, v, cu=cu, rows=rows)
    assert torch.equal(a.pool.view(torch.uint8), b.pool.view(torch.uint8))


def test_one_token_a_row_and_tokens_without_a_place():
    cache = disc.DiscCache.empty(1, 8, 16, 2, 64, 4, 2, held="e4m3")
    disc.disc_cache_extend(cache, i32([5, 0, 16, 1]))
    before = cache.pool.clone()
    q, k, v = vectors(4, 6, 64, torch.bfloat16).split([2, 2, 2], dim=1)
    freq = frequencies(64)
    status = torch.tensor([0, 0, 1, 0], dtype=torch.uint8, device=DEV)
    got = disc.disc_norm_rope_write(cache, 0, q, k, v, freq, status=status)
    want = disc.disc_norm_rope(q, None, i32([4, 0, 15, 0]), freq)[0]     # row 1 has no token: position 0
    assert torch.equal(got, want)
    changed = (cache.pool != before).flatten(3).any(dim=3).any(dim=2).any(dim=1).any(dim=0)
    assert int(cache.table[2, 0]) not in changed.nonzero().flatten().tolist()
    # packed tokens that belong to no sequence, and a sequence that is no row
    before = cache.pool.clone()
    got = disc.disc_norm_rope_write(cache, 0, q, k, v, freq, cu=i32([1, 2, 3]), rows=i32([3, 9]))
    want = disc.disc_norm_rope(q, None, i32([0, 0, 0, 0]), freq)[0]
    assert torch.equal(got, want)
    assert int((cache.pool != before).flatten(3).any(dim=3).any(dim=2).any(dim=1).any(dim=0).sum()) <= 1


def test_caches_and_calls_that_are_refused():
    with pytest.raises(TypeError):
        disc.DiscCache.empty(1, 4, 16, 2, 64, 2, 2, held="e5m2")
    with pytest.raises(disc.DiscError):
        disc.DiscCache.empty(1, 4, 16, 2, 72, 2, 2, held="e4m3") and disc.disc_cache_extend(disc.DiscCache.empty(1, 4, 16, 2, 72, 2, 2, held="e4m3"))
    with pytest.raises(TypeError):
        disc.DiscCache(torch.zeros((1, 2, 4, 2, 16 * 65), dtype=torch.int8, device=DEV), 2, 2, held="i8", page_size=16)
    with pytest.raises(TypeError):
        disc.DiscCache(torch.zeros((1, 2, 4, 2, 16 * 65), dtype=torch.uint8, device=DEV), 2, 2, held="i8")
    with pytest.raises(TypeError):
        disc.DiscCache(torch.zeros((1, 2, 4, 2, 16, 64), dtype=torch.bfloat16, device=DEV), 2, 2, dtype=torch.float16)
    with pytest.raises(disc.DiscError):
        disc.DiscCache.empty(1, 4, 16, 2, 64, 2, 2, held="e4m3", dtype=torch.float32)
    cache = disc.DiscCache.empty(1, 4, 16, 2, 64, 2, 2, held="e4m3")
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(TypeError):
        disc.disc_cache_write(cache, 0, x.half(), x.half())
    with pytest.raises(disc.DiscError):
        disc.disc_cache_write(cache, 1, x, x)
    with pytest.raises(disc.DiscError):
        disc.disc_norm_rope_write(cache, 1, None, x, x)
    with pytest.raises(TypeError):
        disc.disc_norm_rope_write(cache, 0, x[:1], x, x)
    with pytest.raises(TypeError):
        disc.disc_norm_rope_write(cache, 0, x.detach().requires_grad_(), x, x)
    with pytest.raises(disc.DiscError):
        disc.disc_cache_read(cache, 0, i32([0, 0, 0, 0]), 4)
    with pytest.raises(disc.DiscError):
        disc.disc_cache_read(cache, -1, i32([0, 1]), 1)
    with pytest.raises(TypeError):
        disc.disc_cache_read(cache, 0, i32([0, 1]), 1, out=(x, x))
