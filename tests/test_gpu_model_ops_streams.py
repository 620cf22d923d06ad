"""Calls on a stream that is not the current one: what they make belongs to that stream."""
import pytest
import torch

import paper_2504_09135_b200 as disc

pytestmark = pytest.mark.gpu


def _logprobs(side):
    z = torch.randn(4096, 64, device="cuda")
    return lambda: disc.disc_logprobs(z, stream=side)["lse"]


def _grad(side):
    z = torch.randn(64, 64, device="cuda")
    t = torch.zeros(64, dtype=torch.int32, device="cuda")
    d = torch.ones(64, device="cuda")
    o = disc.disc_logprobs(z, t)
    return lambda: disc.disc_logprobs_grad(z, t, o["lse"], o["entropy"], d, stream=side)


def _prompt(side):
    q = torch.randn(32, 4, 64, device="cuda").bfloat16()
    cu = torch.tensor([0, 32], dtype=torch.int32, device="cuda")
    return lambda: disc.disc_attend_prompt(q, q, q, cu, max_len=32, stream=side)[0]


def _cached(side):
    cache = disc.DiscCache.empty(1, 8, 16, 4, 128, 8, 1)
    k = torch.randn(8, 4, 128, device="cuda").bfloat16()
    disc.disc_cache_extend(cache)
    disc.disc_cache_write(cache, 0, k, k)
    plan = disc.disc_attend_plan(cache, 8)
    q = torch.randn(8, 8, 128, device="cuda").bfloat16()
    return lambda: disc.disc_attend_cached(cache, 0, q, plan, stream=side)[0]


@pytest.mark.parametrize("make", [_logprobs, _grad, _prompt, _cached])
def test_outputs_do_not_take_memory_in_use_on_the_current_stream(make):
    side = torch.cuda.Stream()
    call = make(side)
    torch.cuda.synchronize()
    want = call()
    torch.cuda.synchronize()
    # 16 KB that the current stream still has to read when they are given back: the size of the outputs
    held = [torch.ones(4096, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)
    kept = [x.clone() for x in held]
    del held
    got = call()
    side.synchronize()
    early = not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert early, "the side stream was to finish first"
    assert all(bool((x == 1).all()) for x in kept)
    assert torch.equal(got, want)
