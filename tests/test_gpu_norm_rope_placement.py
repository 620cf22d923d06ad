"""Where disc_norm_rope_write puts what it forms: the whole pool against the two calls that it stands for, and the places that change."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def two_caches(lens, held, dtype, d, hkv, page):
    made = []
    for _ in range(2):
        cache = disc.DiscCache.empty(1, 24, page, hkv, d, len(lens), 6, dtype=dtype, held=held)
        cache.pool.view(torch.uint8).fill_(0x11)
        assert int(disc.disc_cache_extend(cache, i32(lens)).max()) == 0
        made.append(cache)
    return made


def places(cache, where):
    """Of the pool [1][2][pages][heads]..., which bytes belong to the tokens `where` = [(row, token)]."""
    mark = torch.zeros_like(cache.pool.view(torch.uint8), dtype=torch.bool)
    P, d = cache.page_size, cache.head_dim
    for row, token in where:
        page, off = int(cache.table[row, token // P]), token % P
        part = mark[0, :, page]
        if cache.held:
            part[:, :, off * d:(off + 1) * d] = True
            part[:, :, P * d + off] = True
        else:
            part[:, :, off] = True
    return mark


@pytest.mark.parametrize("held", [None, "e4m3", "i8"])
@pytest.mark.parametrize("dtype,d,hq,hkv,page", [(torch.bfloat16, 128, 8, 4, 16), (torch.float16, 64, 2, 1, 32), (torch.bfloat16, 80, 3, 3, 16), (torch.bfloat16, 16, 1, 2, 64)])
@pytest.mark.parametrize("what", ["one each", "with a status", "packed, a gap and a row that is none"])
def test_the_pool_is_that_of_the_two_calls(what, dtype, d, hq, hkv, page, held):
    lens = [5, 0, page, 1, 2 * page + 1]
    a, b = two_caches(lens, held, dtype, d, hkv, page)
    before = a.pool.view(torch.uint8).clone()
    g = torch.Generator(device=DEV).manual_seed(6)
    n = 5
    q, k, v = torch.randn((n, hq + 2 * hkv, d), generator=g, device=DEV).to(dtype).split([hq, hkv, hkv], dim=1)
    w = torch.rand(d, generator=g, device=DEV) + 0.5
    freq = torch.exp(torch.arange(d // 16 * 4, device=DEV) * (-0.3))
    status = cu = rows = None
    last = [(r, m - 1) for r, m in enumerate(lens) if m]
    pos = [max(m - 1, 0) for m in lens]
    if what == "with a status":
        status = torch.tensor([0, 0, 1, 0, 0], dtype=torch.uint8, device=DEV)
        last = [x for x in last if x[0] != 2]
    elif what != "one each":
        # tokens 0 and 4 belong to nobody; 1 to row 3; 2 and 3 are two sequences, one of a row that there is not
        cu, rows, last, pos = i32([1, 2, 3, 4]), i32([3, 9, 4]), [(3, 0), (4, 2 * page)], [0, 0, 0, 2 * page, 0]
    got = disc.disc_norm_rope_write(a, 0, q, k, v, freq, k_weight=w, cu=cu, rows=rows, status=status)
    q2, k2 = disc.disc_norm_rope(q, k, i32(pos), freq, k_weight=w)
    disc.disc_cache_write(b, 0, k2, v, cu=cu, rows=rows, status=status)
    assert torch.equal(got, q2)
    now = a.pool.view(torch.uint8)
    assert torch.equal(now, b.pool.view(torch.uint8))
    mark = places(a, last)
    assert torch.equal(now[~mark], before[~mark])
    assert bool((now != before)[mark].float().mean() > 0.9)          # 0x11 may be one of the codes
    # and the values are the tokens': read back, within half a step of what was given (e4m3: a 16th; i8: a 126th of the vector's largest)
    starts = i32([t for _, t in last])
    kr, vr = disc.disc_cache_read(a, 0, i32(list(range(len(last) + 1))), len(last), rows=i32([r for r, _ in last]), start=starts)
    token = [r for r, _ in last] if cu is None else [1, 3]
    for x, y in ((kr, k2), (vr, v)):
        want = y[token].double()
        off = {None: 0.0, "e4m3": 2.0 ** -4, "i8": 0.0}[held] * want.abs() + {None: 0.0, "e4m3": 2.0 ** -16, "i8": 1 / 126}[held] * want.abs().amax(dim=-1, keepdim=True)
        assert torch.all((x.double() - want).abs() <= off * 1.0001)
