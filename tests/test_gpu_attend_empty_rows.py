"""Groups with rows that have no tokens: the others still share their pages."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from test_gpu_attend_cached import build, check

pytestmark = pytest.mark.gpu
DEV = "cuda"


def items(cache, hq, group):
    """How many items the plan has: where the last lane's would begin (after the error word's 256 bytes, one number per lane)."""
    plan = disc.disc_attend_plan(cache, hq, group=group)
    lanes = 296 // cache.n_kv_heads
    return int(plan.buf[256:256 + 4 * (lanes + 1)].view(torch.int32)[-1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group,hq,hkv,d,page", [(8, 2, 1, 64, 16), (5, 6, 2, 128, 32), (16, 1, 1, 72, 16), (32, 4, 1, 64, 16), (32, 8, 2, 128, 32), (7, 33, 1, 72, 16), (20, 64, 2, 128, 16)])
@pytest.mark.parametrize("none", [[0], [3], [0, 1, 4], "last", "all but two"])
def test_freed_candidates(dtype, group, hq, hkv, d, page, none):
    full = 2000 // page
    lens = [full * page + 1 + x % 30 for x in range(group)] + [full * page + 3] * group
    cache, table = build(lens, page, hkv, d, dtype, group=group, shared=[full, full], seed=group)
    before = items(cache, hq, group)
    gone = [group - 1] if none == "last" else [r for r in range(group) if r not in (2, 4)] if none == "all but two" else none
    freed = np.zeros(2 * group, np.uint8)
    freed[gone] = 1
    disc.disc_cache_free(cache, torch.as_tensor(freed).to(DEV))
    for r in gone:
        lens[r] = 0
    out, lse = check(cache, table, lens, hq, group, rows=[0, 1, 2, 3, 4, group - 1, group, 2 * group - 1])
    assert torch.all(out[gone] == 0) and torch.isinf(lse[gone]).all()
    # without sharing each of the rows would have its own over the prompt; lanes' shares are whole fours of blocks, which moves the
    # number by some per cent
    assert items(cache, hq, group) <= 1.1 * before + 2


def test_groups_of_empty_rows_among_others():
    group = 32
    lens = [0] * group + [500] * group + [0] * group + [0] * (group - 1) + [700]
    for hq in (8, 64):                                     # 64: a group is worked on in parts
        cache, table = build(lens, 16, 1, 64, torch.bfloat16, group=group, shared=[0, 31, 0, 0], seed=1)
        check(cache, table, lens, hq, group, rows=[0, 31, 32, 40, 63, 64, 126, 127])
