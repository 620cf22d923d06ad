"""decode_cached with prompts of no tokens: their candidates are reported, the other queries' are as they were."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from test_gpu_cached_decode import plain_hidden
from workloads import make_set, scaled
from workloads.attention_lm import AttentionLM

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("lens", [[7, 0, 20, 16], [9, 33, 0], [0, 12, 5], [0, 0, 17, 0, 0]])
def test_empty_prompts(lens):
    w = scaled("genret", n_draws=5000)
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    B, K = len(lens), 4
    prompts = torch.as_tensor(np.random.default_rng(1).integers(0, w.V, sum(lens)).astype(np.int32), device=DEV)
    cu = torch.as_tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEV)
    lm = AttentionLM(w.V, 2, 8, 2, 64, seed=3)
    cache = lm.new_cache(B * K, max(lens) + G.l_max, n_pages=40 * B)
    dec = disc.DiscDecoder(G, B, K)
    seen = []
    r = dec.decode_cached(lm, cache, prompts, cu, max(lens), seed=5, on_step=lambda t, z, o: seen.append(z.clone()))
    none = np.array([n == 0 for n in lens])
    assert np.array_equal(r["cache_status"].view(B, K).cpu().numpy(), np.repeat(np.where(none, disc.ROW_DEAD, 0)[:, None], K, 1))
    seq, steps = dec.seq.cpu().numpy(), dec.state.depth.cpu().numpy()
    for row in range(0, B * K, 3):
        b = row // K
        if not none[b]:
            # the bound of the decode's own test: two runs that round activations to bf16
            whole = torch.cat([prompts[cu[b]:cu[b + 1]], torch.as_tensor(seq[row, :steps[row] - 1].astype(np.int32), device=DEV)])
            z = lm.logits(plain_hidden(lm, whole))[lens[b] - 1:].float()
            for t in range(steps[row]):
                assert (seen[t][row].float() - z[t]).abs().max() < 0.12
    left = cache.len.view(B, K).cpu().numpy()
    idx = r["idx"].cpu().numpy()
    for b in range(B):
        assert left[b, 0] == (0 if none[b] else lens[b] + steps[b * K + idx[b]] - 1) and not left[b, 1:].any()
    G.close()


def test_no_prompt_tokens_at_all():
    w = scaled("tiny")
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    lm = AttentionLM(w.V, 1, 2, 1, 32)
    cache = lm.new_cache(8, 32, n_pages=20)
    cu = torch.zeros(3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        disc.DiscDecoder(G, 2, 4).decode_cached(lm, cache, torch.empty(0, dtype=torch.int32, device=DEV), cu, 0)
    G.close()


def test_a_model_whose_weights_require_gradients():
    """A decode has no backward pass: it is not recorded, whatever the caller's mode."""
    w = scaled("tiny")
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    runs = []
    for grad in (False, True):
        lm = AttentionLM(w.V, 1, 4, 2, 32)

        class Model:
            hq = lm.hq

            def prefill(self, *args):
                return AttentionLM.prefill.__wrapped__(lm, *args)

            def step(self, *args):
                return AttentionLM.step.__wrapped__(lm, *args)

            def logits(self, hidden):
                return lm.logits(hidden)

        for m in [lm.embed, lm.head] + [x for b in lm.blocks for x in b.values()]:
            m.requires_grad_(grad)
        cache = lm.new_cache(8, 64, n_pages=40)
        dec = disc.DiscDecoder(G, 2, 4)
        r = dec.decode_cached(Model(), cache, torch.arange(20, dtype=torch.int32, device=DEV), torch.tensor([0, 7, 20], dtype=torch.int32, device=DEV), 13, seed=3)
        runs.append((dec.seq.clone(), r["idx"]))
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    G.close()
