"""Vectors with unusual strides: broadcast over tokens or heads, and axes of one entry, whose stride means nothing."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("side", [False, True])
@pytest.mark.parametrize("hq,hkv,group", [(4, 2, 1), (4, 2, 6), (12, 2, 6), (40, 1, 6)])
def test_queries_broadcast_over_rows_or_heads(hq, hkv, group, side):
    cache = disc.DiscCache(torch.randn((1, 2, 20, hkv, 16, 64), device=DEV).bfloat16(), 6, 3)
    disc.disc_cache_extend(cache, torch.full((6,), 30, dtype=torch.int32, device=DEV))
    plan = disc.disc_attend_plan(cache, hq, group=group)
    stream = torch.cuda.Stream() if side else None
    for shape in ((1, hq, 64), (6, 1, 64), (1, 1, 64)):
        q = torch.randn(shape, device=DEV).bfloat16().expand(6, hq, 64)
        want, _ = disc.disc_attend_cached(cache, 0, q.contiguous(), plan)
        torch.cuda.synchronize()
        got, _ = disc.disc_attend_cached(cache, 0, q, plan, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_prompts_broadcast_over_heads_or_tokens():
    cu = torch.tensor([0, 5, 40], dtype=torch.int32, device=DEV)
    q = torch.randn((40, 8, 64), device=DEV).bfloat16()
    k = torch.randn((40, 1, 64), device=DEV).bfloat16().expand(40, 4, 64)
    v = torch.randn((1, 4, 64), device=DEV).bfloat16().expand(40, 4, 64)
    for args in ((q, k, k), (q, k, v), (q[:1].expand(40, 8, 64), k, v), (q[:, :1].expand(40, 8, 64), k.contiguous(), v)):
        got = disc.disc_attend_prompt(*args, cu, max_len=35)
        want = disc.disc_attend_prompt(*(x.contiguous() for x in args), cu, max_len=35)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    none = torch.empty((0, 8, 64), dtype=torch.bfloat16, device=DEV)
    out, _ = disc.disc_attend_prompt(none, none, none, torch.zeros(2, dtype=torch.int32, device=DEV), max_len=0)
    assert out.shape == none.shape


@pytest.mark.parametrize("tokens,heads,strides", [(4, 1, (64, 3, 1)), (1, 2, (5, 64, 1)), (1, 1, (1, 7, 1))])
def test_writing_with_axes_of_one_entry(tokens, heads, strides):
    cache = disc.DiscCache.empty(1, 8, 16, heads, 64, tokens, 2)
    disc.disc_cache_extend(cache)
    k = torch.randn(1000, device=DEV).bfloat16().as_strided((tokens, heads, 64), strides)
    disc.disc_cache_write(cache, 0, k, k)
    for r in range(tokens):
        assert torch.equal(cache.pool[0, :, int(cache.table[r, 0]), :, 0], k[r].expand(2, heads, 64))
