"""Plans that do not fit: of a cache of other sizes, not made yet."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def filled(rows=6, page=16, hkv=2, d=64, width=3, n_pages=20, dtype=torch.bfloat16):
    pool = torch.randn((1, 2, n_pages, hkv, page, d), device=DEV).to(dtype)
    cache = disc.DiscCache(pool, rows, width)
    disc.disc_cache_extend(cache, torch.full((rows,), 30, dtype=torch.int32, device=DEV))
    return cache


@pytest.mark.parametrize("group", [1, 6])
@pytest.mark.parametrize("other", [dict(rows=7), dict(page=32), dict(hkv=4), dict(d=72), dict(width=4), dict(n_pages=21), dict(dtype=torch.float16)])
def test_a_plan_of_another_cache_is_refused(group, other):
    a, b = filled(), filled(**other)
    plan = disc.disc_attend_plan(b, 24, group=group)
    q = torch.randn((a.n_rows, 24, a.head_dim), device=DEV).bfloat16()
    with pytest.raises(TypeError):
        disc.disc_attend_cached(a, 0, q, plan)
    with pytest.raises(TypeError):
        disc.disc_attend_plan(a, 24, group=group, plan=plan)
    c = filled()                                       # the same sizes: any of them may use it, made anew
    mine = disc.disc_attend_plan(a, 24, group=group)
    disc.disc_attend_plan(c, 24, group=group, plan=mine)
    out, _ = disc.disc_attend_cached(c, 0, q, mine)
    assert torch.equal(out, disc.disc_attend_cached(c, 0, q, disc.disc_attend_plan(c, 24, group=group))[0])


@pytest.mark.parametrize("group", [1, 6])
def test_a_plan_that_was_never_made_is_refused(group):
    cache = filled()
    plan = disc.AttendPlan(cache, 24, group)
    q = torch.randn((6, 24, 64), device=DEV).bfloat16()
    with pytest.raises(TypeError):
        disc.disc_attend_cached(cache, 0, q, plan)
    disc.disc_attend_check(plan=plan)
    assert disc.disc_attend_plan(cache, 24, group=group, plan=plan) is plan
    disc.disc_attend_cached(cache, 0, q, plan)


@pytest.mark.parametrize("group,hq", [(1, 4), (6, 4), (6, 24), (1, 64)])
def test_a_plan_older_than_the_books_reads_nothing_outside_the_pool(group, hq):
    """Rows that have let go of their pages since the plan was made: their results mean nothing, and the others are as they were."""
    cache = filled()
    q = torch.randn((6, hq, 64), device=DEV).bfloat16()
    plan = disc.disc_attend_plan(cache, hq, group=group)
    want, _ = disc.disc_attend_cached(cache, 0, q, plan)
    freed = torch.tensor([1, 0, 0, 1, 0, 1], dtype=torch.uint8, device=DEV)
    disc.disc_cache_free(cache, freed)
    old, _ = disc.disc_attend_cached(cache, 0, q, plan)
    new, lse = disc.disc_attend_cached(cache, 0, q, disc.disc_attend_plan(cache, hq, group=group))
    torch.cuda.synchronize()
    disc.disc_attend_check(plan=plan)
    kept = freed == 0
    assert torch.equal(old[kept], want[kept])
    assert torch.all(new[~kept] == 0) and torch.isinf(lse[~kept]).all()
