"""Measured cases of the operators around the decoding step: attention over prompts, the paged
key-value cache, attention of one new token over that cache, and log-probabilities of given tokens.

`run` computes an operator either in its plain form (elementary torch operations in 32 bits) or, with
`own` set, through the package's public entry points.  Both take the same state from `prepare`.
`exact` gives the floating-point outputs from the definitions in 64 bits.

Cache layout everywhere: pool [layers][2][pages][kv heads][page size][head dim] (index 1: keys, values);
`book` is one int32 buffer with the page table [rows][table width], the lengths [rows] and the
reference counts [pages]; table entries past a row's last page are -1.
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ---- the cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # one short question typed by a user: what a single prompt costs in latency
        dict(name="prompt_short", kind="prompt", seqs=1, lo=17, hi=17, hq=16, hkv=16, d=64, type="bf16", layout=1),
        # a batch of 64 prompts of very different lengths, packed, half precision
        dict(name="prompt_ragged", kind="prompt", seqs=64, lo=1, hi=701, hq=16, hkv=4, d=64, type="f16", layout=2),
        # long documents in the prompt, width 2048 as 16 heads
        dict(name="prompt_long", kind="prompt", seqs=2, lo=8192, hi=8192, hq=16, hkv=4, d=128, type="bf16", layout=3),
        # one sequence, one new token: latency of a position
        dict(name="token_single", kind="token", queries=1, cands=1, lo=1500, hi=1500, tail=0, hq=16, hkv=4, d=128, page=16, type="bf16", layout=4),
        # 64 unrelated sequences of one to some thousand tokens
        dict(name="token_ragged", kind="token", queries=64, cands=1, lo=1, hi=8191, tail=0, hq=32, hkv=8, d=128, page=64, type="bf16", layout=5),
        # 128 queries with 32 candidates each: the candidates share the pages of their query's prompt
        dict(name="token_candidates", kind="token", queries=128, cands=32, lo=500, hi=1024, tail=16, hq=16, hkv=4, d=128, page=16, type="bf16", layout=6),
        # first position of a tiny decode: four candidates from each of four prompts
        dict(name="cache_fork_small", kind="fork", queries=4, cands=4, lo=20, hi=40, hkv=4, d=64, page=16, layers=2, type="bf16", spare=64, layout=7),
        # first position of a full decode: 32 candidates from each of 128 prompts, four layers
        dict(name="cache_fork_large", kind="fork", queries=128, cands=32, lo=200, hi=1024, hkv=4, d=128, page=16, layers=4, type="bf16", spare=20000, layout=8),
        # end of a decode: one candidate of each query is kept, the others' pages are freed, the live pages move together
        dict(name="cache_retire", kind="retire", queries=128, cands=16, lo=300, hi=1024, tail=16, hkv=4, d=128, page=16, layers=2, type="bf16", spare=20000, layout=9),
        # one row: the log-probability of a token and its alternatives, as an interactive caller asks for them
        dict(name="logprobs_single", kind="logprobs", n=1, v=128256, top=5, type="bf16", grad=False),
        # all candidates of a position scored with the 20 best alternatives
        dict(name="logprobs_large", kind="logprobs", n=4096, v=128256, top=20, type="bf16", grad=False),
        # the gradient of log-probabilities and entropies with respect to the logits, odd number of rows
        dict(name="logprobs_grad", kind="logprobs", n=2047, v=32000, top=0, type="bf16", grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "token", "fork", "retire", "logprobs", "logprobs"])
    layout = rng.randrange(1 << 30)
    if kind == "prompt":
        hi = _log_int(rng, 1, 8192)
        seqs = _log_int(rng, 1, max(1, min(64, (2 * 8192 * 8192) // (hi * hi))))
        hkv, g = rng.choice([(16, 1), (4, 4), (2, 8), (1, 16), (8, 2)])
        return dict(kind=kind, seqs=seqs, lo=rng.randint(1, hi), hi=hi, hq=hkv * g, hkv=hkv, d=rng.choice([64, 128]),
                    type=rng.choice(["bf16", "f16"]), layout=layout)
    if kind == "token":
        hkv, g = rng.choice([(8, 4), (4, 4), (2, 8), (16, 1)])
        d, page = rng.choice([64, 128]), rng.choice([16, 32, 64])
        cands = rng.choice([1, 1, 4, 8, 16, 32])
        hi = _log_int(rng, 1, 8191 if cands == 1 else 1024)
        # no more rows x tokens x heads than the largest listed case
        queries = _log_int(rng, 1, max(1, min(128, int(64 * 8191 * 8 // (hi * hkv * cands)) if cands == 1 else 128 * 32 // cands * 4 // hkv)))
        return dict(kind=kind, queries=queries, cands=cands, lo=rng.randint(1, hi), hi=hi, tail=0 if cands == 1 else rng.randint(1, 16), hq=hkv * g,
                    hkv=hkv, d=d, page=page, type=rng.choice(["bf16", "f16"]), layout=layout)
    if kind in ("fork", "retire"):
        hi = _log_int(rng, 16, 1024)
        case = dict(kind=kind, queries=_log_int(rng, 1, 128), cands=rng.choice([2, 4, 5, 8, 16]), lo=rng.randint(1, hi), hi=hi,
                    hkv=rng.choice([1, 2, 4]), d=rng.choice([64, 128]), page=rng.choice([16, 32]), layers=rng.randint(1, 3), type=rng.choice(["bf16", "f16"]),
                    spare=4096, layout=layout)
        if kind == "retire":
            case["tail"] = rng.randint(1, 16)
        return case
    grad = rng.random() < 0.4
    v = rng.choice([256, 32000, 128256, rng.randint(64, 128256)])
    return dict(kind=kind, n=_log_int(rng, 1, max(1, min(4096, 4096 * 32000 // v if grad else 4096 * 128256 // v))), v=v, top=0 if grad else rng.randint(0, 20),
                type=rng.choice(["bf16", "f32"]) if v < 100000 else "bf16", grad=grad)


# ---- layouts: decided by the case alone ---------------------------------------------------------------
def _lens(case):
    r = np.random.RandomState(case["layout"] % (1 << 31))
    n = case.get("seqs") or case["queries"]
    lens = r.randint(case["lo"], case["hi"] + 1, n)
    lens[r.randint(n)] = case["hi"]
    return lens.astype(np.int64), r


def _tables(case):
    """Page tables as a decode leaves them, over a pool whose pages lie scattered.

    token / retire: row q * cands + c is candidate c of query q after `tail` (or fewer) tokens of its own; the full pages of
    the prompt are shared, the page where the prompt ends is each candidate's own copy.
    fork: the first row of each query holds its prompt, the other rows are empty."""
    lens, r = _lens(case)
    B, K, P = len(lens), case["cands"], case["page"]
    rows = B * K
    own_lens = np.zeros(rows, np.int64)
    if case["kind"] == "fork":
        total = np.zeros(rows, np.int64)
        total[::K] = lens
    elif K == 1:
        total = lens.copy()
    else:
        own_lens = r.randint(1, case["tail"] + 1, rows)
        total = np.repeat(lens, K) + own_lens
    used = (total + P - 1) // P
    width = int(max(used.max(), (case["hi"] + case.get("tail", 0) + P) // P)) + 1
    shared = np.repeat(lens // P, K) if K > 1 and case["kind"] != "fork" else np.zeros(rows, np.int64)
    private = used - shared
    n_shared = int(shared[::K].sum())
    need = n_shared + int(private.sum())
    pages = need + case.get("spare", 64)
    ids = r.permutation(pages).astype(np.int32)
    table = np.full((rows, width), -1, np.int32)
    at = np.arange(width)[None, :]
    sb = np.concatenate([[0], np.cumsum(shared[::K])])[:-1].repeat(K)
    pb = n_shared + np.concatenate([[0], np.cumsum(private)])[:-1]
    in_shared = at < shared[:, None]
    in_own = (at >= shared[:, None]) & (at < used[:, None])
    table[in_shared] = ids[(sb[:, None] + at)[in_shared]]
    table[in_own] = ids[(pb[:, None] + at - shared[:, None])[in_own]]
    ref = np.bincount(table[table >= 0].ravel(), minlength=pages).astype(np.int32)
    parent = np.full(rows, -1, np.int32)
    if case["kind"] == "fork":
        parent = (np.arange(rows) // K * K).astype(np.int32)
    elif case["kind"] == "retire":
        parent[::K] = np.arange(B) * K + r.randint(0, K, B)
    return dict(table=table, len=total.astype(np.int32), ref=ref, pages=pages, width=width, rows=rows, parent=parent)


# ---- inputs --------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, dt = case["kind"], _TYPES[case["type"]]
    if kind == "prompt":
        lens = _lens(case)[0]
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        T, d = int(cu[-1]), case["d"]
        # one fused projection output, sliced into queries, keys and values as a model does
        qkv = _normal(gen, (T, case["hq"] + 2 * case["hkv"], d), dt)
        q, k, v = qkv.split([case["hq"], case["hkv"], case["hkv"]], dim=1)
        return dict(kind=kind, q=q, k=k, v=v, cu=torch.as_tensor(cu).cuda(), max_len=int(lens.max()), scale=1.0 / math.sqrt(d))
    if kind == "logprobs":
        n, V = case["n"], case["v"]
        logits = torch.empty((n, V), dtype=dt, device="cuda")
        for a in range(0, n, 512):       # a language model's logits: wide, with some tokens far above the rest
            part = _normal(gen, (min(512, n - a), V), torch.float32, 2.0)
            logits[a:a + 512] = part.to(dt)
        st = dict(kind=kind, grad=case["grad"], logits=logits, top=case["top"], inv_t=1.0,
                  targets=torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32))
        if case["grad"]:
            z = logits.float()
            st["lse"] = torch.logsumexp(z, dim=1)
            p = torch.exp(z - st["lse"][:, None])
            st["entropy"] = st["lse"] - (p * z).sum(dim=1)
            st["d_logp"] = _normal(gen, (n,), torch.float32, 1.0 / n)
            st["d_entropy"] = _normal(gen, (n,), torch.float32, 0.01 / n)
        return st
    t = _tables(case)
    layers = case.get("layers", 1)
    pool = torch.empty((layers, 2, t["pages"], case["hkv"], case["page"], case["d"]), dtype=dt, device="cuda")
    for plane in pool.view(layers * 2, *pool.shape[2:]):
        plane.copy_(_normal(gen, plane.shape, dt))
    book = torch.as_tensor(np.concatenate([t["table"].ravel(), t["len"], t["ref"]])).cuda()
    st = dict(kind=kind, pool=pool, book=book, start=book.clone(), rows=t["rows"], width=t["width"], group=case["cands"],
              max_len=int(t["len"].max()), parent=torch.as_tensor(t["parent"]).cuda())
    if kind == "token":
        st["q"] = _normal(gen, (t["rows"], case["hq"], case["d"]), dt)
        st["scale"] = 1.0 / math.sqrt(case["d"])
    if kind == "fork":
        st["k"] = _normal(gen, (t["rows"], case["hkv"], case["d"]), dt)
        st["v"] = _normal(gen, (t["rows"], case["hkv"], case["d"]), dt)
    return st


def work(case):
    kind, size = case["kind"], _SIZE[case["type"]]
    if kind == "prompt":
        lens = _lens(case)[0]
        T = int(lens.sum())
        return dict(bytes=T * case["d"] * (2 * case["hq"] + 2 * case["hkv"]) * size + T * case["hq"] * 4,
                    flops=4 * case["d"] * case["hq"] * int((lens * (lens + 1) // 2).sum()))
    if kind == "logprobs":
        n, V = case["n"], case["v"]
        if case["grad"]:
            return dict(bytes=2 * n * V * size + n * 20, flops=8 * n * V)
        return dict(bytes=n * V * size + n * (20 + 8 * case["top"]), flops=6 * n * V)
    t = _tables(case)
    token = 2 * case["hkv"] * case["d"] * size       # bytes of one token's keys and values in one layer
    if kind == "token":
        P, lens = case["page"], t["len"].astype(np.int64)
        # a page that several rows share is read once
        first = np.unique(t["table"][t["table"] >= 0], return_index=True)[1]
        filled = np.clip(lens[:, None] - np.arange(t["width"])[None, :] * P, 0, P)[t["table"] >= 0]
        return dict(bytes=int(filled[first].sum()) * token + t["rows"] * case["hq"] * (2 * case["d"] * size + 4) + int((t["table"] >= 0).sum()) * 4,
                    flops=4 * case["d"] * case["hq"] * int(lens.sum()))
    if kind == "fork":
        K, fill = case["cands"], t["len"][::case["cands"]] % case["page"]
        copied = int(fill.sum())
        return dict(bytes=(copied + copied * (K - 1)) * token * case["layers"] + 2 * t["rows"] * token + 8 * int((t["table"] >= 0).sum()) * K, flops=0)
    keep = t["table"][t["parent"][t["parent"] >= 0]]
    live = np.unique(keep[keep >= 0])
    moved = int((live >= len(live)).sum())
    return dict(bytes=2 * moved * case["page"] * token * case["layers"] + 8 * int((t["table"] >= 0).sum()) + 8 * t["pages"], flops=0)


# ---- plain forms -----------------------------------------------------------------------------------------
def _softmax_parts(s, ok):
    """exp(s - max) over the allowed places, its sum, and the log of the sum of exponentials; -inf where nothing is allowed."""
    s = torch.where(ok, s, torch.full_like(s, -math.inf))
    m = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, torch.zeros_like(m)))
    total = p.sum(dim=-1, keepdim=True)
    return p, total, (m + torch.log(total)).squeeze(-1)


def _plain_prompt(st):
    q, k, v, cu = st["q"], st["k"], st["v"], st["cu"].long()
    T, hq, d = q.shape
    hkv, L, n = k.shape[1], st["max_len"], cu.numel() - 1
    pos = torch.arange(L, device=q.device)
    lens = cu[1:] - cu[:-1]
    at = (cu[:-1, None] + pos[None, :]).clamp_(max=T - 1)
    qp = q[at].float().view(n, L, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    kp = k[at].float().permute(0, 2, 3, 1)
    s = torch.matmul(qp, kp).view(n, hkv, hq // hkv, L, L) * st["scale"]
    ok = (pos[None, None, :] <= pos[None, :, None]) & (pos[None, None, :] < lens[:, None, None])
    p, total, lse = _softmax_parts(s, ok[:, None, None])
    del s
    o = torch.matmul(p.view(n, hkv, -1, L), v[at].float().permute(0, 2, 1, 3)).view(n, hkv, hq // hkv, L, d) / total
    tok = torch.arange(T, device=q.device)
    seq = torch.searchsorted(cu, tok, right=True) - 1
    out = o.permute(0, 3, 1, 2, 4).reshape(n, L, hq, d)[seq, tok - cu[seq]]
    return dict(out=out.to(q.dtype), lse=lse.permute(0, 3, 1, 2).reshape(n, L, hq)[seq, tok - cu[seq]])


def _views(st):
    book, rows, width = st["book"], st["rows"], st["width"]
    return book[:rows * width].view(rows, width), book[rows * width:rows * width + rows], book[rows * width + rows:]


def _plain_token(st):
    table, lens, _ = _views(st)
    kp, vp, q = st["pool"][0, 0], st["pool"][0, 1], st["q"]
    P, hkv = kp.shape[2], kp.shape[1]
    R, hq, d = q.shape
    pos = torch.arange(st["max_len"], device=q.device)
    page = table.long()[:, pos // P].clamp_(min=0)
    k = kp[page, :, (pos % P)[None, :]].float()
    s = torch.matmul(q.float().view(R, hkv, hq // hkv, d), k.permute(0, 2, 3, 1)) * st["scale"]
    del k
    p, total, lse = _softmax_parts(s, (pos[None, :] < lens[:, None])[:, None, None, :])
    v = vp[page, :, (pos % P)[None, :]].float()
    o = torch.matmul(p, v.permute(0, 2, 1, 3)) / torch.where(total > 0, total, torch.ones_like(total))
    return dict(out=o.view(R, hq, d).to(q.dtype), lse=lse.reshape(R, hq))


def _plain_take_parents(st):
    """Row r becomes what row parent[r] was; -1 empties it."""
    table, lens, ref = _views(st)
    parent = st["parent"].long()
    some = parent >= 0
    new = torch.where(some[:, None], table[parent.clamp(min=0)], torch.full_like(table, -1))
    for_ref = torch.zeros(ref.numel() + 1, dtype=torch.int32, device=ref.device)
    for_ref.index_add_(0, new.reshape(-1).long().where(new.reshape(-1) >= 0, torch.tensor(ref.numel(), device=ref.device)), torch.ones(new.numel(), dtype=torch.int32, device=ref.device))
    new_lens = torch.where(some, lens[parent.clamp(min=0)], torch.zeros_like(lens))
    table.copy_(new)
    lens.copy_(new_lens)
    ref.copy_(for_ref[:-1])


def _plain_extend(st):
    """Room for one more token in every row: new pages, and private copies of shared last pages."""
    table, lens, ref = _views(st)
    pool = st["pool"]
    P, n_pages, rows = pool.shape[4], pool.shape[2], st["rows"]
    dev = ref.device
    row = torch.arange(rows, device=dev)
    fill = lens.long() % P
    last = (lens.long() // P).clamp(max=st["width"] - 1)
    page = table[row, last].long()
    partial = fill > 0
    spot = page.where(partial, torch.tensor(n_pages, device=dev))
    count = torch.zeros(n_pages + 1, dtype=torch.int32, device=dev).index_add_(0, spot, torch.ones(rows, dtype=torch.int32, device=dev))
    keeper = torch.full((n_pages + 1,), rows, dtype=torch.int64, device=dev).scatter_reduce_(0, spot, row, "amin")
    refs = torch.cat([ref, ref.new_zeros(1)])[spot]
    keeps = (count[spot] == refs) & (keeper[spot] == row)
    copy = partial & (refs > 1) & ~keeps
    need = (copy | ~partial).long()
    free = ref == 0
    ids = torch.full((n_pages + rows,), -1, dtype=torch.int64, device=dev)
    ids.scatter_(0, torch.where(free, torch.cumsum(free, 0) - 1, torch.tensor(n_pages + rows - 1, device=dev)), torch.arange(n_pages, device=dev))
    upto = torch.cumsum(need, 0)
    fits = (need == 0) | (upto <= free.sum())
    takes = fits & (need > 0)
    got = ids[(upto - 1).clamp(min=0)]
    chosen = takes & copy
    src, dst = page[chosen], got[chosen]
    keep_old = (torch.arange(P, device=dev)[None, :] >= fill[chosen][:, None])[None, None, :, None, :, None]
    pool[:, :, dst] = torch.where(keep_old, pool[:, :, dst], pool[:, :, src])
    ref.index_add_(0, src, torch.full((src.numel(),), -1, dtype=torch.int32, device=dev))
    ref.index_add_(0, got[takes], torch.ones(int(takes.sum()), dtype=torch.int32, device=dev))
    table[row, last] = torch.where(takes, got.int(), table[row, last])
    lens.add_(fits.int())
    return torch.where(fits, 0, 32).to(torch.uint8)


def _plain_write(st):
    table, lens, _ = _views(st)
    P = st["pool"].shape[4]
    row = torch.arange(st["rows"], device=lens.device)
    at = lens.long() - 1
    page = table[row, at // P].long()
    st["pool"][0, 0][page, :, at % P] = st["k"]
    st["pool"][0, 1][page, :, at % P] = st["v"]


def _plain_compact(st):
    table, lens, ref = _views(st)
    pool = st["pool"]
    live = ref > 0
    n = int(live.sum())
    ids = torch.arange(ref.numel(), device=ref.device)
    src, dst = ids[n:][live[n:]], ids[:n][~live[:n]]
    pool[:, :, dst] = pool[:, :, src]
    to = ids.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    ref[dst] = ref[src]
    ref[src] = 0
    return torch.tensor([n], dtype=torch.int32, device=ref.device)


def _plain_logprobs(st):
    z = st["logits"].float() * st["inv_t"]
    V = z.shape[1]
    t = st["targets"].long()[:, None]
    m = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(dim=1, keepdim=True)
    lse = m + torch.log(total)
    if st["grad"]:
        p = e / total
        logp = z - lse
        h = -(p * logp).sum(dim=1, keepdim=True)
        g = -(st["d_logp"][:, None] * p) - st["d_entropy"][:, None] * p * (logp + h)
        g.scatter_add_(1, t, st["d_logp"][:, None])
        return dict(grad=(g * st["inv_t"]).to(st["logits"].dtype))
    entropy = (lse - (e * z).sum(dim=1, keepdim=True) / total).squeeze(1)
    res = dict(logp=(z.gather(1, t) - lse).squeeze(1), lse=lse.squeeze(1), entropy=entropy)
    del e
    if st["top"]:
        # order by value, equal values by the lower id: the value's bits as an ordered whole number above the reversed id
        bits = (st["logits"].float() + 0.0).view(torch.int32).long()
        key = (torch.where(bits >= 0, bits, -2147483648 - bits) << 32) + (V - 1 - torch.arange(V, device=z.device))[None, :]
        ids = V - 1 - (torch.topk(key, st["top"], dim=1).values & 0xFFFFFFFF)
        res["top_ids"] = ids.int()
        res["top_logp"] = z.gather(1, ids) - lse
    return res


def _run_plain(st):
    kind = st["kind"]
    if kind == "prompt":
        return _plain_prompt(st)
    if kind == "logprobs":
        return _plain_logprobs(st)
    if kind == "token":
        return _plain_token(st)
    st["book"].copy_(st["start"])
    _plain_take_parents(st)
    if kind == "fork":
        status = _plain_extend(st)
        _plain_write(st)
        return dict(book=st["book"], status=status, pool=st["pool"])
    return dict(live=_plain_compact(st), book=st["book"], pool=st["pool"])


# ---- the package's operators ---------------------------------------------------------------------------
def _run_own(st):
    import paper_2504_09135_b200 as disc
    kind = st["kind"]
    if kind == "prompt":
        out, lse = disc.disc_attend_prompt(st["q"], st["k"], st["v"], st["cu"], max_len=st["max_len"], scale=st["scale"])
        return dict(out=out, lse=lse)
    if kind == "logprobs":
        if st["grad"]:
            return dict(grad=disc.disc_logprobs_grad(st["logits"], st["targets"], st["lse"], st["entropy"], st["d_logp"], st["d_entropy"],
                                                     inv_temperature=st["inv_t"]))
        r = disc.disc_logprobs(st["logits"], st["targets"], top=st["top"], inv_temperature=st["inv_t"])
        res = dict(logp=r["logp"], lse=r["lse"], entropy=r["entropy"])
        if st["top"]:
            res["top_ids"], res["top_logp"] = r["top_ids"], r["top_logp"]
        return res
    cache = st.get("cache")
    if cache is None:                                   # the handle a program keeps: the buffers and their sizes
        cache = st["cache"] = disc.DiscCache(st["pool"], st["rows"], st["width"], book=st["book"])
    if kind == "token":
        plan = disc.disc_attend_plan(cache, st["q"].shape[1], group=st["group"])
        out, lse = disc.disc_attend_cached(cache, 0, st["q"], plan, scale=st["scale"])
        return dict(out=out, lse=lse)
    st["book"].copy_(st["start"])
    disc.disc_cache_fork(cache, st["parent"])
    if kind == "fork":
        status = disc.disc_cache_extend(cache)
        disc.disc_cache_write(cache, 0, st["k"], st["v"])
        return dict(book=st["book"], status=status, pool=st["pool"])
    return dict(live=disc.disc_cache_compact(cache), book=st["book"], pool=st["pool"])


def run(state):
    with torch.no_grad():
        return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------
def _attend64(q, k, v, scale, first):
    """q [n, heads, d] against k, v [m, kv heads, d]; query i sees the keys 0 .. first + i."""
    n, hq, d = q.shape
    m, hkv = k.shape[0], k.shape[1]
    out = torch.empty((n, hq, d), dtype=torch.float64, device=q.device)
    lse = torch.empty((n, hq), dtype=torch.float64, device=q.device)
    hidden = torch.arange(m, device=q.device)[None, :] > first + torch.arange(n, device=q.device)[:, None]
    for h in range(hq):
        g = h * hkv // hq
        s = (q[:, h].double() @ k[:, g].double().T * scale).masked_fill_(hidden, -math.inf)
        lse[:, h] = torch.logsumexp(s, dim=1)
        out[:, h] = torch.softmax(s, dim=1) @ v[:, g].double()
    return out, lse


def exact(case, seed):
    kind = case["kind"]
    if kind in ("fork", "retire"):
        return None                                     # whole numbers and copies
    st = prepare(case, seed)
    if kind == "prompt":
        parts = []
        cu = st["cu"].tolist()
        for a, b in zip(cu[:-1], cu[1:]):
            parts.append(_attend64(st["q"][a:b], st["k"][a:b], st["v"][a:b], st["scale"], 0))
        return dict(out=torch.cat([p[0] for p in parts]), lse=torch.cat([p[1] for p in parts]))
    if kind == "token":
        t = _tables(case)
        P = case["page"]
        q = st["q"]
        R, hq, d = q.shape
        if R * hq > 1 << 17:
            return None
        hkv = case["hkv"]
        outs, lses = [], []
        for r in range(R):
            n = int(t["len"][r])
            ids = torch.as_tensor(t["table"][r, :(n + P - 1) // P].astype(np.int64)).cuda()
            k = st["pool"][0, 0][ids].transpose(1, 2).reshape(-1, hkv, d)[:n].double()
            v = st["pool"][0, 1][ids].transpose(1, 2).reshape(-1, hkv, d)[:n].double()
            s = torch.einsum("hgd,lhd->hgl", q[r].double().view(hkv, hq // hkv, d), k) * st["scale"]
            lses.append(torch.logsumexp(s, dim=-1).reshape(hq))
            outs.append(torch.einsum("hgl,lhd->hgd", torch.softmax(s, dim=-1), v).reshape(hq, d))
        return dict(out=torch.stack(outs), lse=torch.stack(lses))
    rows = []
    for i in range(0, case["n"], 256):
        z = st["logits"][i:i + 256].double() * st["inv_t"]
        lp = torch.log_softmax(z, dim=1)
        t = st["targets"][i:i + 256].long()
        h = -(lp.exp() * lp).sum(dim=1)
        if case["grad"]:
            a, b = st["d_logp"][i:i + 256].double(), st["d_entropy"][i:i + 256].double()
            one = torch.zeros_like(lp).scatter_(1, t[:, None], 1.0)
            rows.append(dict(grad=((one - lp.exp()) * a[:, None] - lp.exp() * (lp + h[:, None]) * b[:, None]) * st["inv_t"]))
            continue
        r = dict(logp=lp.gather(1, t[:, None])[:, 0], lse=torch.logsumexp(z, dim=1), entropy=h)
        if case["top"]:
            r["top_ids"] = None
            r["top_logp"] = torch.topk(lp, case["top"], dim=1).values
        rows.append(r)
    return {k: None if rows[0][k] is None else torch.cat([r[k] for r in rows]) for k in rows[0]}
