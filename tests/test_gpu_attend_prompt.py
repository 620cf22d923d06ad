"""disc_attend_prompt against attention in 64 bits, sequence by sequence."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc
from model_ops_reference import assert_attend, attend64

pytestmark = pytest.mark.gpu
DEV = "cuda"


def cu_of(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device=DEV)


def make(n, heads, d, dtype, seed, scale=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn((n, heads, d), generator=gen, device=DEV) * scale).to(dtype)


def check(q, k, v, lq, lk, *, causal=True, scale=None, max_len=None, only=None):
    d = q.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    same = lk is lq
    out, lse = disc.disc_attend_prompt(q, k, v, cu_of(lq), None if same else cu_of(lk), max_len=max(lq) if max_len is None else max_len,
                                       scale=scale, causal=causal)
    disc.disc_attend_check()
    a = b = 0
    for i, (n, m) in enumerate(zip(lq, lk)):
        if only is None or i in only:
            sees = [max(0, min(m, j + m - n + 1)) if causal else m for j in range(n)]
            assert_attend(out[a:a + n], lse[a:a + n], attend64(q[a:a + n], k[b:b + m], v[b:b + m], scale, sees))
        a, b = a + n, b + m
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (4, 1, 128), (8, 2, 128), (6, 2, 72), (7, 1, 40), (16, 1, 64), (5, 5, 8), (128, 1, 128), (80, 1, 64), (3, 3, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(dtype, hq, hkv, d, causal):
    lens = [1, 2, 0, 17, 127, 128, 129, 300, 3]
    n = sum(lens)
    check(make(n, hq, d, dtype, 1), make(n, hkv, d, dtype, 2), make(n, hkv, d, dtype, 3), lens, lens, causal=causal)


@pytest.mark.parametrize("lens,hq,hkv,d", [([1], 1, 1, 128), ([1, 1, 1], 16, 4, 64), ([257, 255, 256, 512], 1, 1, 64), ([1500], 4, 2, 128), ([2049, 700], 4, 4, 64)])
def test_lengths_around_the_tiles(lens, hq, hkv, d):
    n = sum(lens)
    check(make(n, hq, d, torch.bfloat16, 4), make(n, hkv, d, torch.bfloat16, 5), make(n, hkv, d, torch.bfloat16, 6), lens, lens)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2)])
def test_other_numbers_of_keys_than_queries(causal, hq, hkv):
    lq, lk = [5, 300, 1, 130, 40, 7, 200], [200, 20, 513, 130, 0, 6, 329]      # rows that see nothing among them
    check(make(sum(lq), hq, 64, torch.bfloat16, 7), make(sum(lk), hkv, 64, torch.bfloat16, 8), make(sum(lk), hkv, 64, torch.bfloat16, 9), lq, lk, causal=causal)


def test_no_keys_at_all():
    q = make(9, 2, 64, torch.bfloat16, 1)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    out, lse = disc.disc_attend_prompt(q, none, none, cu_of([4, 5]), cu_of([0, 0]), max_len=5)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)
    out, lse = disc.disc_attend_prompt(none, q, q, cu_of([0]), cu_of([9]), max_len=0)
    assert out.shape == (0, 2, 64)


def test_scores_that_grow_and_large_ones():
    """Keys in order of their scores: the running maximum moves in every block; and scores of some hundreds."""
    lens = [1000]
    q = torch.ones((1000, 2, 64), device=DEV).bfloat16()
    ramp = torch.linspace(-30, 30, 1000, device=DEV)[:, None, None].expand(1000, 2, 64).bfloat16().contiguous()
    v = make(1000, 2, 64, torch.bfloat16, 3)
    check(q, ramp, v, lens, lens)
    check(q, -ramp, v, lens, lens)
    check(make(1000, 2, 64, torch.bfloat16, 5, 12.0), make(1000, 2, 64, torch.bfloat16, 6, 3.0), v, lens, lens)
    check(q, torch.zeros_like(v), v, lens, lens)           # all scores equal


def test_fused_projection_slices_and_other_orders():
    lens = [200, 90]
    n = sum(lens)
    qkv = make(n, 8 + 2 * 2, 128, torch.bfloat16, 1)
    check(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], lens, lens)
    wide = make(n, 12, 136, torch.bfloat16, 2)[:, :, 8:]   # rows of 272 bytes
    check(wide[:, :8], wide[:, 8:10], wide[:, 10:], lens, lens)


def test_another_sequence_with_non_finite_keys_and_values_is_not_seen():
    lens = [70, 130, 50]
    n = sum(lens)
    q, k, v = make(n, 4, 64, torch.bfloat16, 1), make(n, 2, 64, torch.bfloat16, 2), make(n, 2, 64, torch.bfloat16, 3)
    clean, _ = check(q, k, v, lens, lens)
    k[70:200] = math.nan
    v[70:200] = math.inf
    out, _ = check(q, k, v, lens, lens, only=(0, 2))
    assert torch.equal(out[:70], clean[:70]) and torch.equal(out[200:], clean[200:])


def test_long_sequence_against_some_rows():
    n, hq, hkv, d = 9000, 4, 1, 128
    q, k, v = make(n, hq, d, torch.bfloat16, 1), make(n, hkv, d, torch.bfloat16, 2), make(n, hkv, d, torch.bfloat16, 3)
    out, lse = disc.disc_attend_prompt(q, k, v, cu_of([n]), max_len=n)
    pick = torch.tensor([0, 1, 127, 128, 4095, 4096, 7777, n - 1], device=DEV)
    assert_attend(out[pick], lse[pick], attend64(q[pick], k, v, 1 / math.sqrt(d), (pick + 1).tolist()))


def test_same_bits_twice_and_on_another_stream():
    lens = [777, 64, 1300]
    n = sum(lens)
    q, k, v = make(n, 8, 128, torch.float16, 1), make(n, 2, 128, torch.float16, 2), make(n, 2, 128, torch.float16, 3)
    cu = cu_of(lens)
    a = disc.disc_attend_prompt(q, k, v, cu, max_len=1300)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = disc.disc_attend_prompt(q, k, v, cu, max_len=1300)
    c = disc.disc_attend_prompt(q, k, v, cu, max_len=5000, stream=s)       # a loose bound on the lengths
    torch.cuda.synchronize()
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z)


def test_refusals():
    q = make(10, 4, 64, torch.bfloat16, 1)
    cu = cu_of([10])
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(q.float(), q.float(), q.float(), cu, max_len=10)
    with pytest.raises(TypeError):
        disc.disc_attend_prompt(q, q.half(), q, cu, max_len=10)
    with pytest.raises(TypeError):
        disc.disc_attend_prompt(q, q, q[:9], cu, max_len=10)
    with pytest.raises(TypeError):
        disc.disc_attend_prompt(q.transpose(1, 2), q, q, cu, max_len=10)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(q, q[:, :3].contiguous(), q[:, :3].contiguous(), cu, max_len=10)       # 4 heads over 3
    big = make(10, 4, 136, torch.bfloat16, 1)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(big, big, big, cu, max_len=10)
    odd = make(10, 4, 68, torch.bfloat16, 1)[:, :, :64]
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(odd, odd, odd, cu, max_len=10)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(q, q, q, cu, max_len=10, scale=-1.0)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(q, q[:5], q[:5], cu, max_len=10)           # other numbers of keys need their own offsets
    many = make(10, 129, 64, torch.bfloat16, 1)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_prompt(many, q[:, :1].contiguous(), q[:, :1].contiguous(), cu, max_len=10)
