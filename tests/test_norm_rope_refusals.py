"""Argument checks of the norm, rotation and 8-bit cache entry points that come before anything touches a device: they run here
without one.  The pointers are never followed."""
import ctypes as C
import struct

import pytest

from paper_2504_09135_b200 import binding
from paper_2504_09135_b200.binding import DISC_HELD_E4M3, DISC_HELD_I8, _Cache

ARG, UNSUPPORTED = -1, -7
P = 1 << 20
FIELDS = ["q", "k", "v", "q_out", "k_out", "q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "q_out_token", "q_out_head", "k_out_token",
          "k_out_head", "positions", "inv_freq", "q_weight", "k_weight", "n_tokens", "cu", "rows", "status", "dtype", "n_q_heads", "n_kv_heads", "head_dim",
          "rot", "interleaved", "norm", "weight_dtype", "eps", "n_seqs"]


def call(**over):
    f = dict(q=P, k=P, v=P, q_out=2 * P, k_out=3 * P, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64, q_out_token=256, q_out_head=64,
             k_out_token=128, k_out_head=64, positions=P, inv_freq=P, q_weight=P, k_weight=P, n_tokens=4, cu=0, rows=0, status=0, dtype=1, n_q_heads=4,
             n_kv_heads=2, head_dim=64, rot=64, interleaved=0, norm=1, weight_dtype=0, eps=1e-6, n_seqs=4)
    assert set(over) <= set(f)
    f.update(over)
    return struct.pack("5Q10q4Qq3Q8ifi", *(f[k] for k in FIELDS))


def cache(**over):
    f = dict(pool=P, table=P, len=P, ref=P, scratch=P, scratch_bytes=1 << 40, n_layers=2, n_pages=10, n_kv_heads=2, page_size=16, head_dim=64,
             n_rows=4, table_width=5, dtype=1 | DISC_HELD_E4M3)
    f.update(over)
    return _Cache(*[f[k] for k, _ in _Cache._fields_])


BAD = [(dict(q=0), ARG), (dict(k=0), ARG), (dict(q=P + 8), ARG), (dict(q_out=0), ARG), (dict(positions=0), ARG), (dict(inv_freq=0), ARG),
       (dict(rot=-8), ARG), (dict(rot=72), ARG), (dict(rot=60), UNSUPPORTED), (dict(n_tokens=-1), ARG), (dict(n_tokens=(1 << 30) + 1), ARG),
       (dict(n_q_heads=-1), ARG), (dict(n_kv_heads=1 << 17), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG),
       (dict(dtype=0), UNSUPPORTED), (dict(dtype=1 | DISC_HELD_I8), UNSUPPORTED), (dict(head_dim=60, rot=8), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
       (dict(weight_dtype=2), UNSUPPORTED), (dict(q_weight=P + 4), ARG), (dict(q_token=100), UNSUPPORTED), (dict(k_head=4), UNSUPPORTED),
       (dict(q_out_token=4), UNSUPPORTED)]


@pytest.mark.parametrize("over,want", BAD + [(dict(k_out=0), ARG), (dict(n_q_heads=0, n_kv_heads=0), ARG), (dict(head_dim=0), ARG)])
def test_norm_rope(over, want):
    assert binding.lib().disc_norm_rope(call(**over), 0) == want


def test_norm_rope_with_nothing_to_do():
    L = binding.lib()
    assert L.disc_norm_rope(call(n_tokens=0, q=0, positions=0), 0) == 0
    assert L.disc_norm_rope(None, 0) == ARG


@pytest.mark.parametrize("over,want", BAD + [(dict(k_out=0), ARG)])
def test_norm_rope_grad(over, want):
    assert binding.lib().disc_norm_rope_grad(call(**over), P, P, P, P, P, 1 << 40, 0) == want


def test_norm_rope_grad_buffers():
    L = binding.lib()
    need = L.disc_norm_rope_scratch_bytes(4, 2, 64, 4)
    assert need > 0
    g = L.disc_norm_rope_grad
    assert g(call(), 0, P, P, P, P, need, 0) == ARG and g(call(), P, P + 8, P, P, P, need, 0) == ARG
    assert g(call(), P, P, P, P, 0, need, 0) == ARG and g(call(), P, P, P, P, P, need - 1, 0) == ARG and g(call(), P, P, P, P, P + 2, need, 0) == ARG
    assert g(call(norm=0), P, P, P, 0, P, need, 0) == ARG
    assert g(None, P, P, P, P, P, need, 0) == ARG
    for bad in ((0, 0, 64, 4), (-1, 2, 64, 4), (4, 2, 0, 4), (4, 2, 136, 4), (4, 2, 64, -1)):
        assert L.disc_norm_rope_scratch_bytes(*bad) == ARG
    # enough for every way of cutting the same vectors
    for hq in (1, 3, 8, 40):
        for n in (1, 7, 500, 100000):
            assert 0 < L.disc_norm_rope_scratch_bytes(hq, 0, 64, n) <= L.disc_norm_rope_scratch_bytes(hq, hq, 64, n) + 64 * 4


@pytest.mark.parametrize("over,want", BAD + [(dict(v=0), ARG), (dict(n_seqs=3), ARG), (dict(n_seqs=-1), ARG), (dict(n_tokens=5, n_seqs=5), ARG),
                                             (dict(n_kv_heads=1), ARG), (dict(head_dim=48, rot=48), ARG), (dict(dtype=2), ARG)])
def test_norm_rope_write(over, want):
    if over == dict(positions=0):
        return                               # the places in the rows are taken
    c = cache()
    got = binding.lib().disc_norm_rope_write(C.addressof(c), 0, call(**over), 0)
    # what does not fit the cache is an argument error before it is an unsupported one
    assert got == want or (got == ARG and set(over) & {"dtype", "head_dim"})


def test_norm_rope_write_caches():
    L = binding.lib()
    for over, want in ((dict(pool=0), ARG), (dict(table=0), ARG), (dict(len=0), ARG), (dict(dtype=1 | 0x30), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED)):
        c = cache(**over)
        assert L.disc_norm_rope_write(C.addressof(c), 0, call(), 0) == want
    c = cache()
    p = C.addressof(c)
    assert L.disc_norm_rope_write(p, 2, call(), 0) == ARG and L.disc_norm_rope_write(p, -1, call(), 0) == ARG and L.disc_norm_rope_write(0, 0, call(), 0) == ARG
    assert L.disc_norm_rope_write(p, 0, call(n_tokens=0, n_seqs=0), 0) == 0 and L.disc_norm_rope_write(p, 0, None, 0) == ARG


@pytest.mark.parametrize("held", [DISC_HELD_E4M3, DISC_HELD_I8])
def test_held_caches(held):
    L = binding.lib()
    for over, want in ((dict(head_dim=72), UNSUPPORTED), (dict(head_dim=8), UNSUPPORTED), (dict(dtype=held), UNSUPPORTED), (dict(dtype=3 | held), UNSUPPORTED),
                       (dict(dtype=1 | 0x30), UNSUPPORTED), (dict(dtype=1 | 0x40), UNSUPPORTED), (dict(dtype=-15), UNSUPPORTED), (dict(pool=P + 8), ARG)):
        c = cache(**{"dtype": 1 | held, **over})
        p = C.addressof(c)
        assert L.disc_cache_fork(p, P, 0) == want and L.disc_cache_extend(p, 0, P, 0) == want and L.disc_cache_compact(p, P, 0) == want
        assert L.disc_cache_write(p, 0, P, 128, 64, P, 128, 64, 4, 0, 4, 0, 0, 0) == want
        assert L.disc_cache_read(p, 0, P, 4, 0, 0, 4, P, P, 0) == want
        assert L.disc_attend_plan_bytes(p, 4, 1) in (want, ARG) or over.get("pool")
    c = cache(dtype=2 | held)
    p = C.addressof(c)
    assert L.disc_attend_plan_bytes(p, 4, 1) > 0
    assert L.disc_cache_write(p, 0, P + 2, 128, 64, P, 128, 64, 4, 0, 4, 0, 0, 0) == ARG and L.disc_cache_write(p, 0, P, 100, 64, P, 128, 64, 4, 0, 4, 0, 0, 0) == UNSUPPORTED

    def read(layer=0, cu=P, seqs=4, rows=0, n=4, k=P, v=P):
        return L.disc_cache_read(p, layer, cu, seqs, rows, 0, n, k, v, 0)

    assert read(layer=2) == ARG and read(layer=-1) == ARG and read(cu=0) == ARG and read(seqs=5) == ARG and read(seqs=-1) == ARG and read(n=-1) == ARG
    assert read(k=0) == ARG and read(v=P + 16) == ARG and read(n=0, cu=0) == 0 and read(seqs=0, cu=0) == 0
