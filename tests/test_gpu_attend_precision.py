"""Cached attention with up to 8 query vectors per group: the probabilities lose nothing to the inputs' type."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc
from test_gpu_attend_cached import build, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def run(cache, hq, group, q):
    return disc.disc_attend_cached(cache, 0, q, disc.disc_attend_plan(cache, hq, group=group))[0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d,group", [(8, 1, 64, 1), (8, 2, 128, 1), (3, 3, 40, 1), (4, 2, 128, 4), (5, 5, 72, 8), (2, 1, 64, 3)])
def test_the_outputs_rounding_is_what_is_left(dtype, hq, hkv, d, group):
    """Before its rounding the output is off by a score's error e in fp32 (2^-23 d sum|q k| scale + 2^-21 |s|), twice, and what two
    values of the type leave of a probability (u^2; f16: 2^-24 at least, below its smallest number), times sum p|v|.  Rounding keeps the
    order, so the output lies between the roundings of the two ends of that."""
    lens = [700, 3, 64, 1500, 33, 1, 260, 17, 700, 701, 702, 703]
    cache, table = build(lens, 16, hkv, d, dtype, group=group, shared=[2 if group > 1 else 0] * 12, seed=hq)
    gen = torch.Generator(device=DEV).manual_seed(7)
    q = torch.randn((len(lens), hq, d), generator=gen, device=DEV).to(dtype)
    out = run(cache, hq, group, q)
    u = UNIT[dtype]
    for r, n in enumerate(lens):
        k, v = (x.double().repeat_interleave(hq // hkv, dim=1) for x in tokens(cache, table, r, n, 0))
        qr = q[r].double()
        s = torch.einsum("hd,nhd->hn", qr, k) / math.sqrt(d)
        e = (2.0 ** -23 * d / math.sqrt(d) * torch.einsum("hd,nhd->hn", qr.abs(), k.abs()) + 2.0 ** -21 * s.abs()).amax(dim=1)
        p = torch.softmax(s, dim=1)
        want = torch.einsum("hn,nhd->hd", p, v)
        spread = torch.einsum("hn,nhd->hd", p, v.abs())
        off = (2 * e[:, None] + u * u + 2.0 ** -18) * spread + 2.0 ** -30
        if dtype is torch.float16:
            off = off + 2.0 ** -24 * v.abs().sum(dim=0)
        assert torch.all((out[r] >= (want - off).to(dtype)) & (out[r] <= (want + off).to(dtype))), r


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_an_infinite_value_stays_one(dtype):
    """A probability that the type holds exactly leaves a remainder of 0, and 0 times infinity is not part of the sum."""
    for lens in ([1], [2, 5, 40]):
        cache, table = build(lens, 16, 1, 64, dtype)
        cache.pool[0, 1, int(table[0, 0]), 0, 0, :32] = math.inf
        cache.pool[0, 1, int(table[0, 0]), 0, 0, 5] = -math.inf
        cache.pool[0, 1, int(table[0, 0]), 0, 0, 9] = math.nan
        q = torch.randn((len(lens), 4, 64), device=DEV).to(dtype)
        out = run(cache, 4, 1, q)
        assert torch.isposinf(out[0, :, :5]).all() and torch.isneginf(out[0, :, 5]).all() and torch.isnan(out[0, :, 9]).all() and torch.isposinf(out[0, :, 10:32]).all()
        assert torch.isfinite(out[0, :, 32:]).all() and torch.isfinite(out[1:]).all()
