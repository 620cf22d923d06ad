"""Outputs that lie on another input are refused before anything touches a device; the pointers are never followed."""
import ctypes as C

import pytest

from paper_2504_09135_b200 import binding
from test_norm_rope_refusals import ARG, P, cache, call


@pytest.mark.parametrize("over", [dict(q_out=3 * P, k_out=2 * P, q=2 * P, k=3 * P), dict(q_out=2 * P, k=2 * P), dict(k_out=3 * P, q=3 * P), dict(q_out=2 * P, k_out=2 * P),
                                  dict(q_out=P, q_out_token=512), dict(k_out=5 * P, k=5 * P, k_out_head=128)])
def test_norm_rope(over):
    f = dict(q=P, k=5 * P, q_out=2 * P, k_out=3 * P)
    f.update(over)
    assert binding.lib().disc_norm_rope(call(**f), 0) == ARG


@pytest.mark.parametrize("over", [dict(q_out=5 * P), dict(q_out=6 * P), dict(q_out=P, q_out_head=128)])
def test_norm_rope_write(over):
    c = cache()
    f = dict(q=P, k=5 * P, v=6 * P, q_out=2 * P)
    f.update(over)
    assert binding.lib().disc_norm_rope_write(C.addressof(c), 0, call(**f), 0) == ARG


def test_cache_read():
    c = cache()
    assert binding.lib().disc_cache_read(C.addressof(c), 0, P, 4, 0, 0, 4, 2 * P, 2 * P, 0) == ARG
