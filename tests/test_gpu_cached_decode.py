"""A decode with a model of attention layers over the paged cache, end to end, against the same model run in plain torch
on whole sequences without a cache."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from workloads import make_set, scaled
from workloads.attention_lm import AttentionLM

pytestmark = pytest.mark.gpu
DEV = "cuda"


def plain_hidden(lm, tokens):
    """Hidden vectors of one sequence: attention by the formula in fp32, rounded like the model's other activations."""
    n = tokens.numel()
    hide = torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1)

    def attend(layer, q, k, v):
        k, v = (x.float().repeat_interleave(lm.hq // lm.hkv, dim=1) for x in (k, v))
        s = torch.einsum("ihd,jhd->hij", q.float(), k) / lm.d ** 0.5
        p = torch.softmax(s.masked_fill(hide, -float("inf")), dim=-1)
        return torch.einsum("hij,jhd->ihd", p, v).to(q.dtype)

    return lm.run(tokens, torch.arange(n, device=DEV), attend)


@pytest.mark.parametrize("hq,hkv,d,B,K,name", [(4, 2, 64, 5, 8, "tiny"), (8, 2, 32, 6, 4, "tiny"), (8, 2, 64, 4, 16, "genret")])
def test_decode_over_the_cache(hq, hkv, d, B, K, name):
    w = scaled(name, n_draws=256 if name == "tiny" else 5000)
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    rng = np.random.default_rng(B + K)
    lens = [1, 15, 16, 40, 33, 100][:B]
    prompts = torch.as_tensor(rng.integers(0, w.V, sum(lens)).astype(np.int32), device=DEV)
    cu = torch.as_tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEV)
    lm = AttentionLM(w.V, 2, hq, hkv, d, seed=3)
    dec = disc.DiscDecoder(G, B, K)
    need = sum(-(-n // 16) + 2 * K for n in lens)
    cache = lm.new_cache(B * K, max(lens) + G.l_max, n_pages=need)
    seen = []
    r = dec.decode_cached(lm, cache, prompts, cu, max(lens), seed=5, on_step=lambda t, z, o: seen.append((z.clone(), o.token.clone(), o.logp.clone())))
    disc.disc_attend_check()
    torch.cuda.synchronize()
    assert torch.all(r["cache_status"] == 0) and torch.all(dec.state.done == 1)
    seq = dec.seq.cpu().numpy()
    members = {tuple(tok[off[i]:off[i + 1]]) for i in range(len(off) - 1)}
    steps = dec.state.depth.cpu().numpy()
    logp = torch.zeros(B * K, dtype=torch.float64, device=DEV)
    for z, t, lp in seen:
        logp += torch.where(t >= 0, lp, torch.zeros_like(lp)).double()
    # every candidate is a member, and the model saw the right history: its logits are those of a run without a cache.  Both round
    # the activations to bf16 (2^-9 each); a rounding that falls the other way early on moves logits of order one by some 2^-6.
    for row in range(B * K):
        b = row // K
        cand = seq[row, :steps[row]]
        assert tuple(cand) in members
        if row % K in (0, K - 1):
            whole = torch.cat([prompts[cu[b]:cu[b + 1]], torch.as_tensor(cand[:-1].astype(np.int32), device=DEV)])
            z = lm.logits(plain_hidden(lm, whole))[lens[b] - 1:].float()
            for t in range(steps[row]):
                err = (seen[t][0][row].float() - z[t]).abs().max()
                assert err < 0.12, (row, t, float(err))
    # scoring the candidates as whole sequences gives the log-probabilities that the decode added up
    packed = [torch.cat([prompts[cu[r // K]:cu[r // K + 1]], torch.as_tensor(seq[r, :steps[r]].astype(np.int32), device=DEV)]) for r in range(B * K)]
    pl = [p.numel() for p in packed]
    s = lm.score(torch.cat(packed), torch.as_tensor(np.concatenate([[0], np.cumsum(pl)]).astype(np.int32), device=DEV), max(pl), top=3)
    at = 0
    for row in range(B * K):
        n = lens[row // K]
        got = s["logp"][at + n - 1:at + pl[row] - 1].double().sum()
        assert abs(float(got - logp[row])) < 0.12 * steps[row]
        at += pl[row]
    assert torch.all(s["top_logp"][:, 0] >= s["top_logp"][:, 1])
    # what is left: the drawn candidates, their pages at the front of the pool
    idx = r["idx"].cpu().numpy()
    left = cache.len.cpu().numpy()
    want = np.zeros(B * K, np.int64)
    for b in range(B):
        want[b * K] = lens[b] + steps[b * K + idx[b]] - 1      # the last token drawn was never run
        assert tuple(r["tokens"][b, :steps[b * K + idx[b]]].tolist()) == tuple(seq[b * K + idx[b], :steps[b * K + idx[b]]])
    assert np.array_equal(left, want)
    live = int(r["live_pages"])
    assert live == int(sum(-(-int(n) // 16) for n in want)) and int(cache.ref[live:].sum()) == 0
    G.close()


def test_a_cache_without_room_is_reported():
    w = scaled("tiny")
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    B, K = 2, 4
    lm = AttentionLM(w.V, 1, 2, 1, 32)
    dec = disc.DiscDecoder(G, B, K)
    lens = [16, 20]
    prompts = torch.zeros(36, dtype=torch.int32, device=DEV)
    cu = torch.tensor([0, 16, 36], dtype=torch.int32, device=DEV)
    cache = lm.new_cache(B * K, 64, n_pages=5)
    r = dec.decode_cached(lm, cache, prompts, cu, 20, seed=1)
    st = r["cache_status"].cpu().numpy()
    assert st.any() and set(st.tolist()) <= {0, disc.ROW_NOPAGE}
    with pytest.raises(ValueError):
        dec.decode_cached(lm, lm.new_cache(3, 64, n_pages=5), prompts, cu, 20)
    G.close()


def test_decode_as_one_graph_gives_the_same():
    """Nothing on the path waits for the host: the whole decode is captured and replayed."""
    w = scaled("tiny")
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    B, K = 3, 8
    lm = AttentionLM(w.V, 2, 8, 2, 64)
    lens = [20, 7, 50]
    prompts = torch.as_tensor(np.random.default_rng(0).integers(0, w.V, sum(lens)).astype(np.int32), device=DEV)
    cu = torch.as_tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEV)
    cache = lm.new_cache(B * K, 60, n_pages=100)
    start = cache.book.clone()
    dec = disc.DiscDecoder(G, B, K)
    r = dec.decode_cached(lm, cache, prompts, cu, 50, seed=2)
    want = (dec.seq.clone(), r["idx"].clone(), dec.state.logw.clone(), cache.book.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    cache.book.copy_(start)
    with torch.cuda.graph(graph):
        r = dec.decode_cached(lm, cache, prompts, cu, 50, seed=2)
    for _ in range(2):
        cache.book.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (dec.seq, r["idx"], dec.state.logw, cache.book)):
            assert torch.equal(a, b)
    G.close()
