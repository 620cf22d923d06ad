"""A model with head norms and rotated positions decoding over caches in 16 and in 8 bits, against the same model in plain torch on whole
sequences."""
import numpy as np
import pytest
import torch

import paper_2504_09135_b200 as disc
from held_reference import hold64, norm_rope64, values64
from workloads import make_set, scaled
from workloads.attention_lm import AttentionLM

pytestmark = pytest.mark.gpu
DEV = "cuda"


def held_values(x, held):
    if held is None:
        return x.float()
    return torch.as_tensor(values64(*hold64(x.double().cpu().numpy(), held), held), device=DEV).float()


def plain_hidden(lm, tokens, held, first):
    """Hidden vectors of one sequence by the formulas in fp32, rounded like the model's other activations.  The tokens up to `first` attend
    to keys and values as they are, the others to what a cache holds of them."""
    n = tokens.numel()
    pos = torch.arange(n, device=DEV)
    hide = torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1)

    def attend(layer, q, k, v):
        t = lm.head_turn(layer)
        if lm.turns:
            q, k = (norm_rope64(x.double(), None if w is None else w.double(), pos, t["inv_freq"], norm=t["norm"])[0].to(x.dtype)
                    for x, w in ((q, t["q_weight"]), (k, t["k_weight"])))
        outs = []
        for keys, values in ((k.float(), v.float()), (held_values(k, held), held_values(v, held))):
            keys, values = (x.repeat_interleave(lm.hq // lm.hkv, dim=1) for x in (keys, values))
            s = torch.einsum("ihd,jhd->hij", q.float(), keys) / lm.d ** 0.5
            p = torch.softmax(s.masked_fill(hide, -float("inf")), dim=-1)
            outs.append(torch.einsum("hij,jhd->ihd", p, values))
        return torch.where((pos < first)[:, None, None], outs[0], outs[1]).to(q.dtype)

    return lm.run(tokens, pos, attend)


def model(V, **how):
    return AttentionLM(V, 2, 8, 2, 64, seed=3, **how)


@pytest.mark.parametrize("held", [None, "e4m3", "i8"])
@pytest.mark.parametrize("how", [dict(rotary=64, head_norm=True), dict(rotary=32), dict(head_norm=True), dict()])
def test_decode(how, held):
    w = scaled("tiny")
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    lens, K = [1, 33, 100], 8
    B = len(lens)
    prompts = torch.as_tensor(np.random.default_rng(1).integers(0, w.V, sum(lens)).astype(np.int32), device=DEV)
    cu = torch.as_tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEV)
    lm = model(w.V, **how)
    dec = disc.DiscDecoder(G, B, K)
    cache = lm.new_cache(B * K, max(lens) + G.l_max, n_pages=120, held=held)
    seen = []
    r = dec.decode_cached(lm, cache, prompts, cu, max(lens), seed=5, on_step=lambda t, z, o: seen.append(z.clone()))
    disc.disc_attend_check()
    torch.cuda.synchronize()
    assert torch.all(r["cache_status"] == 0) and int(r["attend_error"]) == 0
    seq, steps = dec.seq.cpu().numpy(), dec.state.depth.cpu().numpy()
    # both sides round the activations to bf16 (2^-9 each); a rounding that falls the other way early on moves logits of order one by some
    # 2^-6, and a code of 2^-4 in one of 64 values of a key moves a score by less than that
    for row in range(0, B * K, 5):
        b = row // K
        whole = torch.cat([prompts[cu[b]:cu[b + 1]], torch.as_tensor(seq[row, :steps[row] - 1].astype(np.int32), device=DEV)])
        z = lm.logits(plain_hidden(lm, whole, held, lens[b]))[lens[b] - 1:].float()
        for t in range(steps[row]):
            assert (seen[t][row].float() - z[t]).abs().max() < 0.12, (row, t)
    # the drawn candidates alone, read back from the pages that have moved together
    left = cache.len.cpu().numpy()
    rows = torch.arange(B, dtype=torch.int32, device=DEV) * K
    n = left[::K]
    k, v = disc.disc_cache_read(cache, 1, torch.as_tensor(np.concatenate([[0], np.cumsum(n)]).astype(np.int32), device=DEV), int(n.sum()), rows=rows)
    assert torch.isfinite(k.float()).all() and torch.isfinite(v.float()).all() and left.sum() == n.sum()
    G.close()


@pytest.mark.parametrize("held", [None, "e4m3", "i8"])
@pytest.mark.parametrize("how", [dict(rotary=64, head_norm=True), dict()])
def test_prompts_in_two_parts(how, held):
    V, first, more = 200, [20, 1, 64], [30, 17, 5]
    lm = model(V, **how)
    rng = np.random.default_rng(4)
    a, b = (torch.as_tensor(rng.integers(0, V, sum(x)).astype(np.int32), device=DEV) for x in (first, more))
    cu_a, cu_b = (torch.as_tensor(np.concatenate([[0], np.cumsum(x)]).astype(np.int32), device=DEV) for x in (first, more))
    cache = lm.new_cache(5, 120, n_pages=40, held=held)
    rows = torch.tensor([4, 0, 2], dtype=torch.int32, device=DEV)
    for part in (first, more):
        add = torch.zeros(5, dtype=torch.int32, device=DEV)
        add[rows.long()] = torch.as_tensor(part, dtype=torch.int32, device=DEV)
        status = disc.disc_cache_extend(cache, add)
        if part is first:
            lm.prefill(a, cu_a, max(first), cache, rows, status)
        else:
            got = lm.logits(lm.resume(b, cu_b, max(more), cache, rows, sum(first) + sum(more), status)).float()
    disc.disc_attend_check()
    for i in range(3):
        whole = torch.cat([a[cu_a[i]:cu_a[i + 1]], b[cu_b[i]:cu_b[i + 1]]])
        want = lm.logits(plain_hidden(lm, whole, held, first[i]))[first[i]:].float()
        assert (got[cu_b[i]:cu_b[i + 1]] - want).abs().max() < 0.12, i


@pytest.mark.parametrize("held", ["e4m3", "i8"])
def test_decode_as_one_graph_gives_the_same(held):
    w = scaled("tiny")
    tok, off = make_set(w)
    G = disc.disc_build_set(tok, off, w.V)
    B, K, lens = 3, 8, [20, 7, 50]
    lm = model(w.V, rotary=64, head_norm=True)
    prompts = torch.as_tensor(np.random.default_rng(0).integers(0, w.V, sum(lens)).astype(np.int32), device=DEV)
    cu = torch.as_tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEV)
    cache = lm.new_cache(B * K, 60, n_pages=100, held=held)
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
