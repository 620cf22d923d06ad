"""One token that outweighs the others by more than f16 can tell apart, which are so many that together they count; and values at the ends of
the range that vectors have."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq", [1, 16])
def test_many_small_probabilities_beside_a_large_one(hq, dtype, held):
    """All rows hold the same pages, as many rows as blocks of threads run at a time, so that a warp has a quarter of a row's 2^19 tokens.
    Scores: 18 for one token, 0 for the others, whose probabilities are then 2^-25.97 of the first's, and 2^-6.97 together."""
    n, d, page, rows = 1 << 19, 16, 128, 444
    big = 77777
    one = disc.DiscCache.empty(1, n // page, page, 1, d, 1, n // page, dtype=dtype, held=held)
    assert int(disc.disc_cache_extend(one, torch.tensor([n], dtype=torch.int32, device=DEV)).max()) == 0
    k, v = torch.zeros((n, 1, d), dtype=dtype, device=DEV), torch.zeros((n, 1, d), dtype=dtype, device=DEV)
    k[big, 0, 0] = 18.0                # 288 2^-4 in e4m3, 72 2^-2 in i8: held exactly
    v[:, 0, :8] = 1.0
    v[big, 0, :8], v[big, 0, 8:] = 0.0, 1.0
    disc.disc_cache_write(one, 0, k, v, cu=torch.tensor([0, n], dtype=torch.int32, device=DEV))
    book = torch.cat([one.table.expand(rows, -1).reshape(-1), one.len.expand(rows), one.ref * rows]).contiguous()
    cache = disc.DiscCache(one.pool, rows, n // page, book=book, held=held, dtype=dtype, page_size=page)
    q = torch.zeros((rows, hq, d), dtype=dtype, device=DEV)
    q[:, :, 0] = 1.0
    plan = disc.disc_attend_plan(cache, hq)
    out, lse = disc.disc_attend_cached(cache, 0, q, plan, scale=1.0)
    disc.disc_attend_check(plan=plan)
    rest = (n - 1) * math.exp(-18.0)
    small, large = rest / (1 + rest), 1 / (1 + rest)
    # What is below half of f16's smallest step, 2^-25, is lost, of factors that are relative to 2^7 at most: for a warp's 2^17 tokens 2^17 2^-32.
    # Sums of 2^13 products of 16 in fp32, truncated: 2^-10 of small.  A thread adds 2^13 pairs of probabilities to its sum, each off by 2^-24 of
    # it: 2^-11.  Joining and exponentials 2^-18; and one rounding.
    unit = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    rel = 2.0 ** -10 + 2.0 ** -11 + 2.0 ** -18 + unit
    err = (out[..., :8].double() - small).abs().max()
    assert float(err) <= 2.0 ** -15 + small * rel, (float(err), small)
    assert float((out[..., 8:].double() - large).abs().max()) <= 2.0 ** -15 + rel
    assert float((lse.double() - (18.0 + math.log1p(rest))).abs().max()) <= 2.0 ** -11 + 2.0 ** -15


@pytest.mark.parametrize("held", ["e4m3", "i8"])
@pytest.mark.parametrize("hq,group", [(1, 1), (16, 1), (4, 8)])
def test_values_of_the_smallest_and_largest_sizes(hq, group, held):
    """bf16 values of 2^-118 and of 2^100 come out as they are where all tokens hold the same one, in rows that are split and that are not."""
    d, page, lens = 64, 16, [1, 40, 9000, 16, 17, 300, 2, 33]
    cache = disc.DiscCache.empty(2, 700, page, 1, d, len(lens), 600, held=held)
    assert int(disc.disc_cache_extend(cache, torch.tensor(lens, dtype=torch.int32, device=DEV)).max()) == 0
    n = sum(lens)
    cu = torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)
    g = torch.Generator(device=DEV).manual_seed(2)
    k = torch.randn((n, 1, d), generator=g, device=DEV).bfloat16()
    q = torch.randn((len(lens), hq, d), generator=g, device=DEV).bfloat16()
    for layer, size in enumerate((2.0 ** -118, 2.0 ** 100)):
        # 1 to 1.75 times a power of two: codes of both forms hold them exactly
        x = (1 + (torch.arange(d, device=DEV) % 4) / 4) * size
        disc.disc_cache_write(cache, layer, k, x.bfloat16().expand(n, 1, d).contiguous(), cu=cu)
        plan = disc.disc_attend_plan(cache, hq, group=group)
        out, lse = disc.disc_attend_cached(cache, layer, q, plan)
        disc.disc_attend_check(plan=plan)
        # probabilities rounded to f16 or bf16, whose sum is that of the rounded ones only up to 2^-8; sums in fp32; one rounding
        assert bool(((out.double() / x.double() - 1).abs() <= 2 * 2.0 ** -8 + 2.0 ** -10).all()), float((out.double() / x.double() - 1).abs().max())
