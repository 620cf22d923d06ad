"""The calls of many positions enqueued one after the other, without a wait, on books that every call changes: the kernels begin while
the ones before them still run.  The same calls with a wait after each give the same bits."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def life(rows, group, hq, hkv, d, pages, width, wait, *, steps=40):
    rng = np.random.default_rng(rows)
    gen = torch.Generator(device=DEV).manual_seed(rows)

    def dev(x):
        return torch.as_tensor(np.ascontiguousarray(x)).to(DEV)

    plans = []
    for t in range(steps):
        first = np.arange(rows) // group * group
        parent = np.where(rng.random(rows) < 0.1, first, np.arange(rows))
        if t % 10 == 9:
            parent = np.where(rng.random(rows) < 0.3, -1, first + rng.integers(0, group, rows)).clip(max=rows - 1)
        # at least one token each: a row that stays as it is must not be written to
        plans.append((dev(rng.integers(1, 9, rows).astype(np.int32)), dev(parent.astype(np.int32)), dev((rng.random(rows) < 0.02).astype(np.uint8))))
    q = torch.randn((steps, rows, hq, d), generator=gen, device=DEV).bfloat16()
    kv = torch.randn((steps, rows, 2 * hkv, d), generator=gen, device=DEV).bfloat16()
    cache = disc.DiscCache.empty(1, pages, 16, hkv, d, rows, width)
    disc.disc_cache_extend(cache, dev(np.where(np.arange(rows) % group == 0, 100, 0).astype(np.int32)))
    disc.disc_cache_fork(cache, dev((np.arange(rows) // group * group).astype(np.int32)))
    add, none = torch.empty(rows, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    parent, freed = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, dtype=torch.uint8, device=DEV)
    status = torch.empty(rows, dtype=torch.uint8, device=DEV)
    got = []
    torch.cuda.synchronize()

    def step():
        if wait:
            torch.cuda.synchronize()

    for t in range(steps):
        # the same few buffers for what changes from position to position
        add.copy_(plans[t][0]); step()
        disc.disc_cache_extend(cache, add, status=status); step()
        disc.disc_cache_write(cache, 0, kv[t, :, :hkv], kv[t, :, hkv:], status=status); step()
        disc.disc_cache_extend(cache, none, status=freed); step()
        disc.disc_cache_free(cache, freed); step()                    # nothing: the call before has just cleared it
        plan = disc.disc_attend_plan(cache, hq, group=group); step()
        got.append(disc.disc_attend_cached(cache, 0, q[t], plan)); step()
        freed.copy_(plans[t][2]); step()
        disc.disc_cache_free(cache, freed); step()
        disc.disc_cache_free(cache, status); step()                   # rows that found no page
        parent.copy_(plans[t][1]); step()
        disc.disc_cache_fork(cache, parent); step()
        disc.disc_cache_extend(cache, status=status); step()
        plan = disc.disc_attend_plan(cache, hq, group=group); step()
        got.append(disc.disc_attend_cached(cache, 0, q[t], plan)); step()
        if t % 7 == 6:
            got.append((disc.disc_cache_compact(cache),)); step()
    torch.cuda.synchronize()
    disc.disc_attend_check(plan=plan)
    return [x for g in got for x in g] + [cache.book, cache.pool.view(torch.int16)]


@pytest.mark.parametrize("rows,group,hq,hkv,d,pages,width", [
    (24, 1, 4, 2, 64, 300, 16), (24, 8, 8, 2, 64, 200, 16), (900, 1, 8, 2, 64, 9000, 16), (900, 4, 4, 2, 128, 7000, 16), (960, 32, 8, 2, 128, 9000, 16),
    (2000, 20, 12, 3, 64, 12000, 16)])
def test_enqueued_calls_give_what_calls_with_waits_give(rows, group, hq, hkv, d, pages, width):
    want = life(rows, group, hq, hkv, d, pages, width, True)
    for _ in range(3):
        for i, (a, b) in enumerate(zip(life(rows, group, hq, hkv, d, pages, width, False), want)):
            assert torch.equal(a, b), i
