"""Tensors that are not on the current device are refused: kernels are launched there, and would follow their pointers.  One device is
enough to see it: the binding is told that another one is current."""
import pytest
import torch

import paper_2504_09135_b200 as disc
from paper_2504_09135_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_tensors_of_another_device_are_refused(monkeypatch):
    z = torch.randn((4, 100), device=DEV)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    q = torch.randn((4, 4, 64), device=DEV).bfloat16()
    cu = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    cache = disc.DiscCache.empty(1, 8, 16, 4, 64, 4, 2)
    flags = torch.zeros(4, dtype=torch.uint8, device=DEV)
    calls = [lambda: disc.disc_logprobs(z, t), lambda: disc.disc_logprobs_grad(z, t, z[:, 0].contiguous(), None, z[:, 1].contiguous()),
             lambda: disc.disc_attend_prompt(q, q, q, cu, max_len=4), lambda: disc.disc_cache_extend(cache), lambda: disc.disc_cache_write(cache, 0, q, q),
             lambda: disc.disc_cache_fork(cache, t), lambda: disc.disc_cache_free(cache, flags), lambda: disc.disc_cache_compact(cache),
             lambda: disc.disc_attend_plan(cache, 4), lambda: disc.disc_attend_cached(cache, 0, q, plan)]
    disc.disc_cache_extend(cache)
    plan = disc.disc_attend_plan(cache, 4)
    for call in calls[:5]:
        call()
    monkeypatch.setattr(binding, "_several", True)
    for call in calls[:5]:
        call()
    monkeypatch.setattr(binding, "_raw_device", lambda: 1)
    for call in calls:
        with pytest.raises(TypeError, match="current device"):
            call()
