"""Head norms and caches in 8 bits where offsets pass 32 bits, on other streams, replayed, and with several users at once."""
import math

import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from held_reference import hold64, norm_rope64, tol_forward, values64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def frequencies(rot):
    return torch.exp(torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) * (-math.log(10000.0) / rot)).float()


@pytest.mark.parametrize("group", [1, 6])
def test_pages_beyond_four_gigabytes(group):
    """A plane of 5 GB whose low pages are taken: 40,000 pages of 8 heads x 128 tokens x 129 bytes."""
    cache = disc.DiscCache.empty(1, 40000, 128, 8, 128, 6, 4, held="e4m3")
    cache.ref[:39980] = 1
    lens = [300, 0, 129, 5, 128, 1] if group == 1 else [260] + [0] * 5
    assert int(disc.disc_cache_extend(cache, i32(lens)).max()) == 0 and int(cache.table[0, 0]) == 39980
    n = sum(lens)
    cu = i32(np.concatenate([[0], np.cumsum(lens)]).tolist())
    x = torch.randn((n, 16, 128), device=DEV).bfloat16()
    k, v = x[:, :8], x[:, 8:]
    disc.disc_cache_write(cache, 0, k, v, cu=cu)
    if group > 1:
        disc.disc_cache_fork(cache, i32([0] * 6))
        disc.disc_cache_extend(cache)
        new = torch.randn((6, 16, 128), device=DEV).bfloat16()
        disc.disc_norm_rope_write(cache, 0, None, new[:, :8], new[:, 8:], None, norm=False)
        lens = [261] * 6
        cu = i32(np.concatenate([[0], np.cumsum(lens)]).tolist())
        k, v = (torch.cat([torch.cat([old, fresh[r:r + 1]]) for r in range(6)]) for old, fresh in ((k, new[:, :8]), (v, new[:, 8:])))
    gk, gv = disc.disc_cache_read(cache, 0, cu, sum(lens))
    hk, hv = (torch.as_tensor(values64(*hold64(t.double().cpu().numpy(), "e4m3"), "e4m3"), device=DEV) for t in (k, v))
    assert torch.equal(gk.double(), hk) and torch.equal(gv.double(), hv)
    q = torch.randn((6, 32, 128), device=DEV).bfloat16()
    out, _ = disc.disc_attend_cached(cache, 0, q, disc.disc_attend_plan(cache, 32, group=group))
    at = 0
    for r, m in enumerate(lens):
        for h in (0, 31):
            if m == 0:
                assert bool((out[r, h] == 0).all())
                continue
            p = torch.softmax(hk[at:at + m, h // 4] @ q[r, h].double() / 128 ** 0.5, dim=0)
            want, size = p @ hv[at:at + m, h // 4], p @ hv[at:at + m, h // 4].abs()
            # probabilities and outputs rounded to bf16, scores to 2^-17 of sizes up to some ten
            assert torch.all((out[r, h].double() - want).abs() <= 2.0 ** -8 * (size + want.abs()) + 2.0 ** -12 * size)
        at += m


def test_vectors_beyond_four_gigabytes():
    n, heads, d = 430_000, 40, 128
    q = torch.randn((n, 1, d), device=DEV).bfloat16().expand(n, heads, d).contiguous()
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    freq = frequencies(d)
    out, _ = disc.disc_norm_rope(q, None, pos, freq, out=None)
    for rows in (slice(0, 3), slice(n // 2, n // 2 + 3), slice(n - 3, n)):
        y, size = norm_rope64(q[rows].double(), None, pos[rows], freq)
        assert torch.all((out[rows].double() - y).abs() <= tol_forward(y, size, q.dtype))
    dq = disc.disc_norm_rope_grad(q, None, pos, freq, out, None)[0]
    small = disc.disc_norm_rope_grad(q[-3:], None, pos[-3:], freq, out[-3:], None)[0]
    assert torch.equal(dq[-3:], small)


@pytest.mark.parametrize("held", ["e4m3", "i8"])
def test_other_streams_and_two_caches_at_once(held):
    sides = [torch.cuda.Stream() for _ in range(2)]
    caches = [disc.DiscCache.empty(1, 60, 16, 2, 64, 8, 10, held=held) for _ in range(2)]
    x = [torch.randn((8 * 40, 12, 64), device=DEV).bfloat16() for _ in range(2)]
    freq, lens = frequencies(64), [40] * 8
    cu = i32(np.arange(9).tolist()) * 40
    for c in caches:
        disc.disc_cache_extend(c, i32(lens[:4] + [0] * 4))
    torch.cuda.synchronize()
    cu = i32([0, 40, 80, 120, 160])
    got = []
    for c, t, side in zip(caches, x, sides):
        q, k, v = t[:160].split([8, 2, 2], dim=1)
        qn = disc.disc_norm_rope_write(c, 0, q, k, v, freq, cu=cu, rows=i32([0, 1, 2, 3]), stream=side)
        gk, gv = disc.disc_cache_read(c, 0, cu, 160, stream=side)
        plan = disc.disc_attend_plan(c, 8, stream=side)
        with torch.cuda.stream(side):
            last = torch.zeros((8, 8, 64), dtype=torch.bfloat16, device=DEV)
            last[:4] = qn[39::40]
        out, lse = disc.disc_attend_cached(c, 0, last, plan, stream=side)
        got.append((qn, gk, gv, out, lse))
    torch.cuda.synchronize()
    for c, t, g in zip(caches, x, got):
        q, k, v = t[:160].split([8, 2, 2], dim=1)
        again = disc.DiscCache(torch.zeros_like(c.pool), 8, 10, book=c.book, held=held, page_size=16)
        qn = disc.disc_norm_rope_write(again, 0, q, k, v, freq, cu=cu)
        assert torch.equal(again.pool, c.pool) and torch.equal(qn, g[0])
        gk, gv = disc.disc_cache_read(again, 0, cu, 160)
        last = torch.zeros((8, 8, 64), dtype=torch.bfloat16, device=DEV)
        last[:4] = qn[39::40]
        out, lse = disc.disc_attend_cached(again, 0, last, disc.disc_attend_plan(again, 8))
        for a, b in zip((gk, gv, out, lse), g[1:]):
            assert torch.equal(a, b)


def test_a_graph_of_a_chunk_replayed_on_new_inputs():
    cache = disc.DiscCache.empty(1, 40, 16, 2, 64, 3, 8, held="i8", dtype=torch.float16)
    disc.disc_cache_extend(cache, i32([30, 5, 64]))
    x = torch.randn((99, 8, 64), device=DEV).half()
    q, k, v = x.split([4, 2, 2], dim=1)
    cu, freq, w = i32([0, 30, 35, 99]), frequencies(32), torch.rand(64, device=DEV) + 0.5

    def run():
        a = disc.disc_norm_rope_write(cache, 0, q, k, v, freq, cu=cu, q_weight=w, k_weight=w)
        return (a, *disc.disc_cache_read(cache, 0, cu, 99))

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in range(2):
        x.copy_(torch.randn(x.shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got_now = [t.clone() for t in got]
        cache.pool.zero_()
        for a, b in zip(got_now, run()):
            assert torch.equal(a, b)
