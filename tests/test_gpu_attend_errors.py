"""The words that say that a bounded wait of an attention kernel ran out.  They are set here by the host, as a kernel would."""
import pytest
import torch

import paper_2504_09135_b200 as disc
from workloads import make_set, scaled
from workloads.attention_lm import AttentionLM

pytestmark = pytest.mark.gpu
DEV = "cuda"


def set_word(plan):
    plan.error.fill_(1)


@pytest.mark.parametrize("group", [1, 32])
def test_the_word_of_a_plan_outlives_the_next_plan_and_is_cleared_by_the_check(group):
    cache = disc.DiscCache.empty(1, 64, 16, 2, 64, 32, 2)
    disc.disc_cache_extend(cache)
    plan = disc.disc_attend_plan(cache, 8, group=group)
    disc.disc_attend_check(plan=plan)
    set_word(plan)
    assert disc.disc_attend_plan(cache, 8, group=group) is plan
    q = torch.randn((32, 8, 64), device=DEV).bfloat16()
    disc.disc_attend_cached(cache, 0, q, plan)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_check(plan=plan)
    disc.disc_attend_check(plan=plan)
    other = disc.disc_attend_plan(cache, 4, group=group)
    disc.disc_attend_check(plan=other)


def test_the_word_of_prompts_is_cleared_by_the_check():
    q = torch.randn((8, 2, 64), device=DEV).bfloat16()
    cu = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    disc.disc_attend_prompt(q, q, q, cu, max_len=8)
    disc.disc_attend_check()
    disc.model_ops.attend_error_word(q.device).fill_(1)
    with pytest.raises(disc.DiscError):
        disc.disc_attend_check()
    disc.disc_attend_check()


class Failing(AttentionLM):
    """The model, with a wait that runs out at position `at`."""
    at = None

    def step(self, tokens, cache, plan, status=None):
        self.position += 1
        if self.position == self.at:
            set_word(plan)
        return super().step(tokens, cache, plan, status)


@pytest.mark.parametrize("at", [None, 1, 3])
def test_a_decode_reports_a_wait_that_ran_out_at_any_position(at):
    w = scaled("genret", n_draws=5000)
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    assert G.l_max > 3
    B, K = 2, 4
    lens = [5, 20]
    lm = Failing(w.V, 1, 8, 2, 32)
    lm.position, lm.at = 0, at
    cache = lm.new_cache(B * K, 60, n_pages=60)
    prompts = torch.zeros(sum(lens), dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, 5, 25], dtype=torch.int32, device=DEV)
    r = disc.DiscDecoder(G, B, K).decode_cached(lm, cache, prompts, cu, max(lens), seed=1)
    assert lm.position >= 3
    assert int(r["attend_error"]) == (at is not None)
    G.close()
