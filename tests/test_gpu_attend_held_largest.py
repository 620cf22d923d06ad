"""f16 values at the end of the type's range, whose e4m3 codes are rounded up beyond it: attention gives them as reading back does, as the largest
finite value and not as infinity."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("hq,group", [(1, 1), (16, 1), (4, 2), (4, 8)])
def test_means_of_the_largest_values(hq, group, held):
    d, page, lens = 64, 16, [1, 40, 9000, 16, 17, 300, 2, 33]
    cache = disc.DiscCache.empty(1, 700, page, 1, d, len(lens), 600, held=held, dtype=torch.float16)
    assert int(disc.disc_cache_extend(cache, torch.tensor(lens, dtype=torch.int32, device=DEV)).max()) == 0
    n = sum(lens)
    cu = torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)
    g = torch.Generator(device=DEV).manual_seed(2)
    k = torch.randn((n, 1, d), generator=g, device=DEV).half()
    q = torch.randn((len(lens), hq, d), generator=g, device=DEV).half()
    x = torch.where(torch.arange(d, device=DEV) % 2 == 0, 65504.0, -65504.0).half()
    disc.disc_cache_write(cache, 0, k, x.expand(n, 1, d).contiguous(), cu=cu)
    back = disc.disc_cache_read(cache, 0, cu, n)[1]
    plan = disc.disc_attend_plan(cache, hq, group=group)
    out, _ = disc.disc_attend_cached(cache, 0, q, plan)
    disc.disc_attend_check(plan=plan)
    want = back[0, 0].float()
    assert bool((want.abs() > 65000).all()) and bool((back == back[0, 0]).all())
    # probabilities rounded to f16, whose sum is that of the rounded ones up to 2^-11; sums in fp32; one rounding
    assert bool((out.float().abs() <= 65504).all())
    assert bool(((out.float() / want - 1).abs() <= 2 * 2.0 ** -11 + 2.0 ** -14).all())
