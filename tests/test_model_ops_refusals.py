"""Argument checks of the model-side entry points that come before anything touches a device: they run here without one.
The pointers are never followed."""
import ctypes as C

import pytest

from paper_2504_09135_b200 import binding
from paper_2504_09135_b200.binding import _Cache

ARG, UNSUPPORTED = -1, -7
P = 1 << 20                        # an aligned non-null pointer


def cache(**over):
    f = dict(pool=P, table=P, len=P, ref=P, scratch=P, scratch_bytes=1 << 40, n_layers=2, n_pages=10, n_kv_heads=2, page_size=16, head_dim=64,
             n_rows=4, table_width=5, dtype=1)
    f.update(over)
    return _Cache(*[f[k] for k, _ in _Cache._fields_])


@pytest.mark.parametrize("over,want", [
    (dict(pool=0), ARG), (dict(ref=0), ARG), (dict(scratch=0), ARG), (dict(scratch_bytes=0), ARG), (dict(n_rows=0), ARG), (dict(n_pages=-1), ARG),
    (dict(dtype=0), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
    (dict(page_size=24), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED), (dict(pool=P + 8), ARG),
    (dict(n_rows=1 << 20, table_width=1 << 12), UNSUPPORTED)])
def test_caches_that_are_refused(over, want):
    L, c = binding.lib(), cache(**over)
    p = C.addressof(c)
    assert L.disc_cache_fork(p, P, 0) == want
    assert L.disc_cache_free(p, P, 0) == want
    assert L.disc_cache_extend(p, 0, P, 0) == want
    assert L.disc_cache_compact(p, P, 0) == want
    assert L.disc_cache_write(p, 0, P, 128, 64, P, 128, 64, 4, 0, 4, 0, 0, 0) == want


def test_cache_calls_that_are_refused():
    L, c = binding.lib(), cache()
    p = C.addressof(c)
    for fn, args in ((L.disc_cache_fork, (p, 0, 0)), (L.disc_cache_free, (p, 0, 0)), (L.disc_cache_extend, (p, 0, 0, 0)), (L.disc_cache_compact, (p, 0, 0))):
        assert fn(*args) == ARG
        assert fn(0, *args[1:]) == ARG

    def write(layer=0, k=P, kt=128, kh=64, tokens=4, cu=0, seqs=4, rows=0):
        return L.disc_cache_write(p, layer, k, kt, kh, P, 128, 64, tokens, cu, seqs, rows, 0, 0)

    assert write(layer=2) == ARG and write(layer=-1) == ARG and write(k=0) == ARG and write(k=P + 2) == ARG
    assert write(tokens=3) == ARG and write(tokens=-1) == ARG and write(seqs=5, tokens=5) == ARG
    assert write(kt=100) == UNSUPPORTED and write(kh=4) == UNSUPPORTED
    assert write(tokens=0, seqs=0) == 0


def test_attention_calls_that_are_refused():
    L, c = binding.lib(), cache()
    p = C.addressof(c)
    assert L.disc_attend_plan_bytes(p, 3, 1) == ARG and L.disc_attend_plan_bytes(p, 4, 0) == ARG and L.disc_attend_plan_bytes(0, 4, 1) == ARG
    assert L.disc_attend_plan_bytes(p, 2 * 65, 1) == UNSUPPORTED
    need = L.disc_attend_plan_bytes(p, 4, 2)
    assert need > 0
    assert L.disc_attend_plan(p, 4, 2, P, need - 1, 0) == ARG and L.disc_attend_plan(p, 4, 2, P + 16, need, 0) == ARG and L.disc_attend_plan(p, 4, 2, 0, need, 0) == ARG

    def cached(layer=0, q=P, row=256, head=64, scale=0.1, plan=P, nbytes=need, out=P):
        return L.disc_attend_cached(p, layer, q, row, head, 4, 2, scale, plan, nbytes, out, 0, 0)

    assert cached(layer=2) == ARG and cached(q=0) == ARG and cached(out=0) == ARG and cached(q=P + 8) == ARG and cached(nbytes=need - 1) == ARG
    assert cached(scale=0.0) == ARG and cached(scale=float("nan")) == ARG and cached(scale=float("inf")) == ARG
    assert cached(row=252) == UNSUPPORTED and cached(head=60) == UNSUPPORTED

    def prompt(q=P, k=P, qt=256, qh=64, dtype=1, hq=4, hkv=2, d=64, nq=10, nk=10, cu=P, seqs=1, mx=10, scale=0.1, out=P, err=P):
        return L.disc_attend_prompt(q, qt, qh, k, 128, 64, P, 128, 64, dtype, hq, hkv, d, nq, nk, cu, 0, seqs, mx, 1, scale, out, 0, err, 0)

    assert prompt(q=0) == ARG and prompt(k=0) == ARG and prompt(cu=0) == ARG and prompt(out=0) == ARG and prompt(err=0) == ARG and prompt(q=P + 4) == ARG
    assert prompt(hq=3) == ARG and prompt(hkv=0) == ARG and prompt(nq=-1) == ARG and prompt(nk=9) == ARG and prompt(scale=0.0) == ARG
    assert prompt(dtype=0) == UNSUPPORTED and prompt(d=68) == UNSUPPORTED and prompt(d=136) == UNSUPPORTED and prompt(hq=258) == UNSUPPORTED
    assert prompt(qt=250) == UNSUPPORTED and prompt(qh=0) == UNSUPPORTED
    assert prompt(nq=0, nk=0) == 0 and prompt(seqs=0) == 0


def test_log_probability_calls_that_are_refused():
    L = binding.lib()

    def lp(z=P, dtype=1, ld=100, n=4, v=100, t=1.0, tgt=P, top=3, logp=P, ids=P, status=P):
        return L.disc_logprobs(z, dtype, ld, n, v, t, tgt, top, logp, 0, 0, ids, 0, status, 0)

    assert lp(z=0) == ARG and lp(ld=99) == ARG and lp(n=-1) == ARG and lp(v=0) == ARG and lp(t=0.0) == ARG and lp(t=float("nan")) == ARG
    assert lp(logp=0) == ARG and lp(ids=0) == ARG and lp(status=0) == ARG and lp(z=P + 1) == ARG and lp(top=-1) == ARG
    assert lp(dtype=2) == UNSUPPORTED and lp(top=65) == UNSUPPORTED and lp(n=1 << 28) == UNSUPPORTED
    assert lp(n=0) == 0

    def grad(z=P, dtype=1, ld=100, n=4, v=100, t=1.0, tgt=P, lse=P, h=P, a=P, b=P, out=2 * P, old=100):
        return L.disc_logprobs_grad(z, dtype, ld, n, v, t, tgt, lse, h, a, b, out, old, 0)

    assert grad(z=0) == ARG and grad(out=0) == ARG and grad(lse=0) == ARG and grad(tgt=0) == ARG and grad(h=0) == ARG and grad(old=99) == ARG
    assert grad(out=P, old=104) == ARG and grad(t=-1.0) == ARG and grad(dtype=2) == UNSUPPORTED
    assert grad(n=0) == 0
