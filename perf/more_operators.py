"""Measured cases of the operators that stand before the attention of a decode: head norms and rotation of queries and
keys with their gradient, and a key-value cache held in 8 bits: written, read back, and attended to by one new token per row.

`run` computes an operator either in its plain form (elementary torch operations in 32 bits) or, with `own` set, through the
package's public entry points.  Both take the same state from `prepare`.  `exact` gives the floating-point outputs from the
definitions in 64 bits.

A vector held in 8 bits is one code per value and a power of two, 2^e: pool uint8 [layers][2][pages][kv heads][page size * (head dim + 1)]
(index 1: keys, values), where a page and head have the codes of their tokens and behind them one byte e per token.  `book` as in a
DiscCache: the page table [rows][width], the lengths [rows], the reference counts [pages].
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---- the cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # queries and keys of one new token of one sequence: latency
        dict(name="rope_single", kind="rope", n=1, far=2000, hq=16, hkv=4, d=128, rot=128, inter=False, norm=True, type="bf16", grad=False),
        # the prompts of a batch, 16384 tokens, wide model
        dict(name="rope_prompt", kind="rope", n=16384, far=8192, hq=32, hkv=8, d=128, rot=128, inter=False, norm=True, type="bf16", grad=False),
        # an odd number of tokens, half of each vector rotated, neighbouring values as pairs, positions far out, no norm
        dict(name="rope_partial", kind="rope", n=4097, far=1000000, hq=16, hkv=4, d=64, rot=32, inter=True, norm=False, type="f16", grad=False),
        # gradients of a short sequence
        dict(name="rope_grad_small", kind="rope", n=67, far=67, hq=8, hkv=2, d=64, rot=64, inter=False, norm=True, type="bf16", grad=True),
        # gradients of a training step's 8191 tokens
        dict(name="rope_grad", kind="rope", n=8191, far=8191, hq=32, hkv=8, d=128, rot=128, inter=False, norm=True, type="bf16", grad=True),
        # keys and values of 64 prompts of very different lengths go into the pages
        dict(name="write_ragged", kind="write", queries=64, cands=1, lo=1, hi=2048, tail=0, hkv=8, d=128, page=32, held="e4m3", type="bf16", layout=11),
        # eight long rows read back for the attention of a prompt that goes on
        dict(name="read_long", kind="read", queries=8, cands=1, lo=2000, hi=8191, tail=0, hkv=8, d=128, page=64, held="i8", type="bf16", layout=12),
        # the next 512 or fewer tokens of each of 16 prompts: norm, rotation, into the pages, and all tokens read back
        dict(name="chunk", kind="chunk", queries=16, cands=1, lo=600, hi=4000, tail=0, new=512, hq=16, hkv=4, d=128, page=16, held="e4m3", type="f16", layout=13),
        # one sequence, one new token of an attention layer: norm, rotation, into the pages, attention; latency
        dict(name="layer_single", kind="layer", queries=1, cands=1, lo=1500, hi=1500, tail=0, hq=16, hkv=4, d=128, page=16, held="e4m3", type="bf16", layout=14),
        # the same for 64 unrelated sequences of one to some thousand tokens
        dict(name="layer_ragged", kind="layer", queries=64, cands=1, lo=1, hi=8191, tail=0, hq=32, hkv=8, d=128, page=64, held="e4m3", type="bf16", layout=15),
        # 96 sequences of a small model, half precision
        dict(name="layer_small", kind="layer", queries=96, cands=1, lo=100, hi=1023, tail=0, hq=8, hkv=4, d=64, page=32, held="i8", type="f16", layout=16),
        # 128 queries with 32 candidates each, which share the pages of their query's prompt
        dict(name="layer_candidates", kind="layer", queries=128, cands=32, lo=500, hi=1024, tail=16, hq=16, hkv=4, d=128, page=16, held="e4m3", type="bf16", layout=17),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "write", "read", "chunk", "layer", "layer"])
    d, ty, held = rng.choice([64, 80, 128]), rng.choice(["bf16", "f16"]), rng.choice(["e4m3", "i8"])
    hkv, g = rng.choice([(8, 4), (4, 4), (2, 8), (8, 1), (1, 16), (4, 2)])
    if kind == "rope":
        return dict(kind=kind, n=_log_int(rng, 1, 8191), far=_log_int(rng, 100, 1000000), hq=hkv * g, hkv=hkv, d=d, rot=rng.choice([d, d // 2 // 8 * 8, 16]),
                    inter=rng.random() < 0.4, norm=rng.random() < 0.7, type=ty, grad=rng.random() < 0.5)
    case = dict(kind=kind, queries=1, cands=1, lo=1, hi=1, tail=0, hq=hkv * g, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 128]), held=held, type=ty,
                layout=rng.randrange(1 << 30))
    if kind == "layer" and rng.random() < 0.4:
        case["cands"] = rng.choice([4, 5, 16, 32])
        case["tail"] = rng.randint(1, 16)
        case["hi"] = _log_int(rng, 16, 1024)
        # no more rows x tokens x heads than the largest listed case
        case["queries"] = _log_int(rng, 1, max(1, min(128, 128 * 32 * 4 // (case["cands"] * hkv))))
    else:
        case["hi"] = _log_int(rng, 1, 8191)
        case["queries"] = _log_int(rng, 1, max(1, min(64, 64 * 8191 * 8 // 4 // (case["hi"] * hkv))))
    case["lo"] = rng.randint(1, case["hi"])
    if kind == "chunk":
        case["new"] = _log_int(rng, 1, 512)
    return case


# ---- layouts: decided by the case alone ---------------------------------------------------------------
def _tables(case):
    """Page tables as a decode leaves them, over a pool whose pages lie scattered.  Row q * cands + c is candidate c of query q
    after `tail` (or fewer) tokens of its own; the full pages of the prompt are shared, the page where the prompt ends is
    each candidate's own copy.  `fresh`: the newest tokens of each row, which a pass writes."""
    r = np.random.RandomState(case["layout"] % (1 << 31))
    B, K, P = case["queries"], case["cands"], case["page"]
    lens = r.randint(case["lo"], case["hi"] + 1, B).astype(np.int64)
    lens[r.randint(B)] = case["hi"]
    rows = B * K
    if case["kind"] == "write":
        fresh = lens.copy()
    elif case["kind"] == "chunk":
        fresh = r.randint(1, case["new"] + 1, rows)
    else:
        fresh = np.full(rows, 1 if case["kind"] == "layer" else 0)
    total = lens.copy()
    if K > 1:
        total = np.repeat(lens, K) + r.randint(1, case["tail"] + 1, rows)
    elif case["kind"] == "chunk":
        total = lens + fresh
    used = (total + P - 1) // P
    width = int(used.max()) + 1
    shared = np.repeat(lens // P, K) if K > 1 else np.zeros(rows, np.int64)
    private = used - shared
    n_shared = int(shared[::K].sum())
    pages = n_shared + int(private.sum()) + 64
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
    return dict(table=table, len=total.astype(np.int32), ref=ref, pages=pages, width=width, rows=rows, fresh=fresh)


# ---- 8 bits ----------------------------------------------------------------------------------------------
def _hold(x, held):
    """x [..., d] -> (codes uint8 [..., d], exponents int8 [...])."""
    x = x.float()
    amax = x.abs().amax(dim=-1)
    fine = torch.isfinite(amax)
    lead = torch.frexp(torch.where(fine, amax, torch.ones_like(amax))).exponent - 1      # floor(log2(amax))
    lead = torch.where(amax > 0, lead, torch.full_like(lead, -200))
    e = (lead - (8 if held == "e4m3" else 6)).clamp(min=-126)
    top = torch.ldexp(amax, -e)
    e = e + ((top > 448) if held == "e4m3" else (torch.round(top) > 127)).int()
    y = torch.ldexp(torch.where(fine[..., None], x, torch.zeros_like(x)), -e[..., None])
    codes = y.to(torch.float8_e4m3fn).view(torch.uint8) if held == "e4m3" else torch.round(y).to(torch.int8).view(torch.uint8)
    return codes, torch.where(fine, e, torch.full_like(e, -128)).to(torch.int8)


def _values(codes, e, held):
    """The values that codes [..., d] and exponents [...] stand for, in 32 bits."""
    x = (codes.view(torch.float8_e4m3fn) if held == "e4m3" else codes.view(torch.int8)).float()
    e = e.int()
    scale = torch.where(e == -128, torch.full_like(e, 0).float() + math.nan, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e))
    return x * scale[..., None]


def _planes(pool, layer, kv, page, d):
    """Codes [pages, heads, page, d] and exponents [pages, heads, page] of a plane, as views."""
    p = pool[layer, kv]
    return p[:, :, :page * d].unflatten(-1, (page, d)), p[:, :, page * d:].view(torch.int8)


# ---- inputs --------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _rotation(case, gen, st):
    rot = case.get("rot", case["d"])
    st["inter"], st["norm"], st["eps"] = case.get("inter", False), case.get("norm", True), 1e-6
    st["inv_freq"] = torch.exp(torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) * (-math.log(10000.0) / rot)).float()
    st["qw"] = st["kw"] = None
    if st["norm"]:
        st["qw"], st["kw"] = 1.0 + _normal(gen, (case["d"],), torch.float32, 0.1), 1.0 + _normal(gen, (case["d"],), torch.float32, 0.1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, dt, d, hkv = case["kind"], _TYPES[case["type"]], case["d"], case["hkv"]
    st = dict(kind=kind, d=d)
    if kind == "rope":
        n, hq = case["n"], case["hq"]
        # one fused projection output, sliced as a model does
        st["q"], st["k"], _ = _normal(gen, (n, hq + 2 * hkv, d), dt, 2.0).split([hq, hkv, hkv], dim=1)
        st["pos"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda", dtype=torch.int32)
        _rotation(case, gen, st)
        st["grad"] = case["grad"]
        if case["grad"]:
            st["dq"], st["dk"] = _normal(gen, (n, hq, d), dt, 1e-3), _normal(gen, (n, hkv, d), dt, 1e-3)
        return st
    t = _tables(case)
    P, held = case["page"], case["held"]
    pool = torch.zeros((1, 2, t["pages"], hkv, P * (d + 1)), dtype=torch.uint8, device="cuda")
    if kind != "write":
        for kv in range(2):
            codes, exps = _planes(pool, 0, kv, P, d)
            for a in range(0, t["pages"], 4096):
                b = min(t["pages"], a + 4096)
                # the vectors of a head differ in size from token to token
                x = _normal(gen, (b - a, hkv, P, d), torch.float32) * torch.exp(_normal(gen, (b - a, hkv, P, 1), torch.float32, 0.3))
                c, e = _hold(x, held)
                codes[a:b], exps[a:b] = c, e
    book = torch.as_tensor(np.concatenate([t["table"].ravel(), t["len"], t["ref"]])).cuda()
    st.update(pool=pool, book=book, rows=t["rows"], width=t["width"], page=P, held=held, hkv=hkv, type=dt, max_len=int(t["len"].max()), group=case["cands"])
    st["fresh"] = torch.as_tensor(np.concatenate([[0], np.cumsum(t["fresh"])]).astype(np.int32)).cuda()
    st["n_fresh"] = int(t["fresh"].sum())
    st["all"] = torch.as_tensor(np.concatenate([[0], np.cumsum(t["len"])]).astype(np.int32)).cuda()
    st["n_all"] = int(t["len"].sum())
    if kind == "write":
        _, st["k"], st["v"] = _normal(gen, (st["n_fresh"], 3 * hkv, d), dt).split([hkv, hkv, hkv], dim=1)
    if kind in ("chunk", "layer"):
        hq = case["hq"]
        st["q"], st["k"], st["v"] = _normal(gen, (st["n_fresh"], hq + 2 * hkv, d), dt, 1.5).split([hq, hkv, hkv], dim=1)
        _rotation(case, gen, st)
        st["scale"] = 1.0 / math.sqrt(d)
    return st


def work(case):
    kind, d, hkv = case["kind"], case["d"], case["hkv"]
    if kind == "rope":
        n, heads = case["n"], case["hq"] + hkv
        return dict(bytes=n * heads * d * 2 * (3 if case["grad"] else 2) + n * 4, flops=n * heads * d * (16 if case["grad"] else 8))
    t = _tables(case)
    lens, P = t["len"].astype(np.int64), case["page"]
    token, wide = 2 * hkv * (d + 1), 2 * hkv * d * 2         # bytes of a token's keys and values in the cache, and as vectors
    fresh = int(t["fresh"].sum())
    books = int((t["table"] >= 0).sum()) * 4
    if kind == "write":
        return dict(bytes=fresh * (token + wide) + books, flops=fresh * 4 * hkv * d)
    if kind == "read":
        return dict(bytes=int(lens.sum()) * (token + wide) + books, flops=int(lens.sum()) * 2 * hkv * d)
    queries = fresh * case["hq"] * d * 2
    if kind == "chunk":
        return dict(bytes=2 * queries + fresh * (wide + token) + int(lens.sum()) * (token + wide) + books, flops=fresh * (case["hq"] + hkv) * d * 8)
    # a page that several rows share is read once
    first = np.unique(t["table"][t["table"] >= 0], return_index=True)[1]
    filled = np.clip(lens[:, None] - np.arange(t["width"])[None, :] * P, 0, P)[t["table"] >= 0]
    return dict(bytes=int(filled[first].sum()) * token + fresh * (wide + token) + 3 * queries + fresh * case["hq"] * 4 + books,
                flops=4 * d * case["hq"] * int(lens.sum()))


# ---- plain forms -----------------------------------------------------------------------------------------
def _angles(pos, inv_freq):
    """cos and sin [n, 1, rot / 2], the angles in 64 bits: in 32 a far position's is off by a hundredth."""
    a = pos.double()[:, None] * inv_freq.double()[None, :]
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _rotate(x, cos, sin, inter, back=False):
    half = cos.shape[-1]
    if half == 0:
        return x
    if back:
        sin = -sin
    rest = x[..., 2 * half:]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if inter else (x[..., :half], x[..., half:2 * half])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([ya, yb], dim=-1).flatten(-2) if inter else torch.cat([ya, yb], dim=-1)
    return torch.cat([y, rest], dim=-1)


def _norm_rope(x, w, cos, sin, st):
    y = x.float()
    if st["norm"]:
        y = y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + st["eps"])
        if w is not None:
            y = y * w
    return _rotate(y, cos, sin, st["inter"]).to(x.dtype)


def _norm_rope_grad(x, dy, w, cos, sin, st):
    g = _rotate(dy.float(), cos, sin, st["inter"], back=True)
    if not st["norm"]:
        return g.to(x.dtype), None
    x32 = x.float()
    r = torch.rsqrt(x32.square().mean(dim=-1, keepdim=True) + st["eps"])
    c = g * w
    dx = r * c - x32 * (r * r * r * (c * x32).mean(dim=-1, keepdim=True))
    return dx.to(x.dtype), (g * x32 * r).sum(dim=(0, 1))


def _views(st):
    book, rows, width = st["book"], st["rows"], st["width"]
    return book[:rows * width].view(rows, width), book[rows * width:rows * width + rows]


def _places(st, cu, n, newest):
    """Page and place in it of n packed tokens: sequence i is row i, its first or newest tokens."""
    table, lens = _views(st)
    tok = torch.arange(n, device=cu.device)
    cu = cu.long()
    row = torch.searchsorted(cu, tok, right=True) - 1
    pos = tok - cu[row]
    if newest:
        pos = pos + lens.long()[row] - (cu[row + 1] - cu[row])
    return table[row, pos // st["page"]].long(), pos % st["page"], pos


def _write(st, k, v):
    page, off, _ = _places(st, st["fresh"], st["n_fresh"], True)
    for kv, x in enumerate((k, v)):
        codes, exps = _planes(st["pool"], 0, kv, st["page"], st["d"])
        codes[page, :, off], exps[page, :, off] = _hold(x, st["held"])


def _read(st):
    page, off, _ = _places(st, st["all"], st["n_all"], False)
    most = torch.finfo(st["type"]).max
    got = []
    for kv in range(2):
        codes, exps = _planes(st["pool"], 0, kv, st["page"], st["d"])
        got.append(_values(codes[page, :, off], exps[page, :, off], st["held"]).clamp_(-most, most).to(st["type"]))
    return got


def _attend(st, q):
    table, lens = _views(st)
    P, hkv, d = st["page"], st["hkv"], st["d"]
    R, hq, _ = q.shape
    pos = torch.arange(st["max_len"], device=q.device)
    page = table.long()[:, pos // P].clamp_(min=0)
    at = (page, slice(None), (pos % P)[None, :])
    codes, exps = _planes(st["pool"], 0, 0, P, d)
    k = _values(codes[at], exps[at], st["held"])
    s = torch.matmul(q.float().view(R, hkv, hq // hkv, d), k.permute(0, 2, 3, 1)) * st["scale"]
    del k
    ok = (pos[None, :] < lens[:, None])[:, None, None, :]
    s = torch.where(ok, s, torch.full_like(s, -math.inf))
    m = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - m)
    total = p.sum(dim=-1, keepdim=True)
    lse = (m + torch.log(total)).squeeze(-1)
    del s
    codes, exps = _planes(st["pool"], 0, 1, P, d)
    v = _values(codes[at], exps[at], st["held"])
    o = torch.matmul(p, torch.where((pos[None, :] < lens[:, None])[:, :, None, None], v, torch.zeros_like(v)).permute(0, 2, 1, 3)) / total
    return o.view(R, hq, d).to(q.dtype), lse.reshape(R, hq)


def _run_plain(st):
    kind = st["kind"]
    if kind == "rope":
        cos, sin = _angles(st["pos"], st["inv_freq"])
        if not st["grad"]:
            return dict(q=_norm_rope(st["q"], st["qw"], cos, sin, st), k=_norm_rope(st["k"], st["kw"], cos, sin, st))
        (dq, dqw), (dk, dkw) = _norm_rope_grad(st["q"], st["dq"], st["qw"], cos, sin, st), _norm_rope_grad(st["k"], st["dk"], st["kw"], cos, sin, st)
        return dict(dq=dq, dk=dk, dqw=dqw, dkw=dkw)
    if kind == "write":
        _write(st, st["k"], st["v"])
        return dict(pool=st["pool"])
    if kind == "read":
        k, v = _read(st)
        return dict(k=k, v=v)
    cos, sin = _angles(_places(st, st["fresh"], st["n_fresh"], True)[2], st["inv_freq"])
    q = _norm_rope(st["q"], st["qw"], cos, sin, st)
    _write(st, _norm_rope(st["k"], st["kw"], cos, sin, st), st["v"])
    if kind == "chunk":
        k, v = _read(st)
        return dict(q=q, k=k, v=v)
    out, lse = _attend(st, q)
    return dict(q=q, out=out, lse=lse)


# ---- the package's operators ---------------------------------------------------------------------------
def _run_own(st):
    import paper_2504_09135_b200 as disc
    kind = st["kind"]
    if kind != "rope" and "cache" not in st:             # the handle a program keeps: the buffers and their sizes
        st["cache"] = disc.DiscCache(st["pool"], st["rows"], st["width"], book=st["book"], held=st["held"], dtype=st["type"], page_size=st["page"])
    if kind == "write":
        disc.disc_cache_write(st["cache"], 0, st["k"], st["v"], cu=st["fresh"])
        return dict(pool=st["pool"])
    if kind == "read":
        k, v = disc.disc_cache_read(st["cache"], 0, st["all"], st["n_all"])
        return dict(k=k, v=v)
    how = dict(norm=st["norm"], q_weight=st["qw"], k_weight=st["kw"], eps=st["eps"], interleaved=st["inter"])
    if kind == "rope":
        if not st["grad"]:
            q, k = disc.disc_norm_rope(st["q"], st["k"], st["pos"], st["inv_freq"], **how)
            return dict(q=q, k=k)
        dq, dk, dqw, dkw = disc.disc_norm_rope_grad(st["q"], st["k"], st["pos"], st["inv_freq"], st["dq"], st["dk"], **how)
        return dict(dq=dq, dk=dk, dqw=dqw, dkw=dkw)
    cache = st["cache"]
    q = disc.disc_norm_rope_write(cache, 0, st["q"], st["k"], st["v"], st["inv_freq"], cu=None if kind == "layer" else st["fresh"], **how)
    if kind == "chunk":
        k, v = disc.disc_cache_read(cache, 0, st["all"], st["n_all"])
        return dict(q=q, k=k, v=v)
    plan = disc.disc_attend_plan(cache, q.shape[1], group=st["group"])
    out, lse = disc.disc_attend_cached(cache, 0, q, plan, scale=st["scale"])
    return dict(q=q, out=out, lse=lse)


def run(state):
    with torch.no_grad():
        return _run_own(state) if own else _run_plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------
def _turn64(x, pos, inv_freq, inter, sign):
    """Each pair as a complex number times e^(i sign position frequency); x [n, heads, d] in 64 bits."""
    half = inv_freq.numel()
    if half == 0:
        return x
    n, h, _ = x.shape
    pairs = x[..., :2 * half]
    z = pairs.reshape(n, h, half, 2) if inter else pairs.reshape(n, h, 2, half).transpose(-1, -2)
    z = torch.view_as_complex(z.contiguous())
    turn = torch.polar(torch.ones((n, half), dtype=torch.float64, device=x.device), sign * pos.double()[:, None] * inv_freq.double())
    y = torch.view_as_real(z * turn[:, None])
    y = y.reshape(n, h, 2 * half) if inter else y.transpose(-1, -2).reshape(n, h, 2 * half)
    return torch.cat([y, x[..., 2 * half:]], dim=-1)


def _norm64(x, w, st):
    x = x.double()
    if not st["norm"]:
        return x
    return x / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / x.shape[-1] + st["eps"]) * w.double()


def _grad64(x, dy, w, st):
    """By autograd of the definition."""
    x = x.double().requires_grad_()
    w = None if w is None else w.double().requires_grad_()
    with torch.enable_grad():
        y = _turn64(_norm64(x, w, st), st["pos"], st["inv_freq"], st["inter"], 1.0)
        got = torch.autograd.grad(y, [x] if w is None else [x, w], dy.double())
    return got[0], got[1] if len(got) > 1 else None


def _held64(x, held):
    """What vectors x [..., d] are held as, code by code from a table of all values a code can have."""
    x = x.double()
    amax = x.abs().amax(dim=-1, keepdim=True)
    lead = torch.floor(torch.log2(amax.clamp(min=2.0 ** -140)))
    lead = torch.where(torch.exp2(lead) > amax, lead - 1, torch.where(torch.exp2(lead + 1) <= amax, lead + 1, lead))
    e = (lead - (8 if held == "e4m3" else 6)).clamp(min=-126.0)
    top = amax / torch.exp2(e)
    e = e + (top > 448 if held == "e4m3" else top >= 127.5).double()
    y = x / torch.exp2(e)
    if held == "i8":
        return torch.round(y) * torch.exp2(e)
    # three binary digits after the leading one, none below 2^-9
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / unit) * unit * torch.exp2(e)


def _row64(st, table, kv, row, n):
    """The first n tokens' keys or values of a row, [n, heads, d] in 64 bits."""
    P, d = st["page"], st["d"]
    ids = torch.as_tensor(table[row, :(n + P - 1) // P].astype(np.int64)).cuda()
    part = st["pool"][0, kv][ids]
    codes = part[:, :, :P * d].reshape(-1, st["hkv"], P, d)
    e = part[:, :, P * d:].contiguous().view(torch.int8)
    x = codes.contiguous().view(torch.float8_e4m3fn).float() if st["held"] == "e4m3" else codes.contiguous().view(torch.int8).float()
    return (x.double() * torch.exp2(e.double())[..., None]).transpose(1, 2).reshape(-1, st["hkv"], d)[:n]


def exact(case, seed):
    kind = case["kind"]
    if kind == "write":
        return None                                     # whole numbers
    if kind == "layer" and case["queries"] * case["cands"] * case["hq"] > 1 << 17:
        return None
    st = prepare(case, seed)
    if kind == "rope":
        if case["grad"]:
            (dq, dqw), (dk, dkw) = _grad64(st["q"], st["dq"], st["qw"], st), _grad64(st["k"], st["dk"], st["kw"], st)
            return dict(dq=dq, dk=dk, dqw=dqw, dkw=dkw)
        return {x: _turn64(_norm64(st[x], st[x + "w"], st), st["pos"], st["inv_freq"], st["inter"], 1.0) for x in "qk"}
    t = _tables(case)
    lens, fresh = t["len"].astype(np.int64), t["fresh"].astype(np.int64)
    res = {}
    if kind in ("chunk", "layer"):
        pos = torch.as_tensor(np.concatenate([np.arange(n - f, n) for n, f in zip(lens, fresh)])).cuda()
        turned = {x: _turn64(_norm64(st[x], st[x + "w"], st), pos, st["inv_freq"], st["inter"], 1.0) for x in "qk"}
        res["q"] = turned["q"]
        # what is held, and what attends, are vectors of the model's type
        new = [_held64(turned["k"].to(st["type"]), st["held"]), _held64(st["v"], st["held"])]
    if kind in ("read", "chunk"):
        at = np.concatenate([[0], np.cumsum(fresh)])
        for kv, name in enumerate("kv"):
            parts = []
            for r in range(t["rows"]):
                n, f = int(lens[r]), int(fresh[r])
                parts.append(_row64(st, t["table"], kv, r, n - f))
                if f:
                    parts.append(new[kv][int(at[r]):int(at[r]) + f])
            res[name] = torch.cat(parts)
        if kind == "chunk":
            res["k"] = None                             # what lies next to the border of two codes is held as either
        return res
    q = res["q"].to(st["type"]).double()
    R, hq, d = q.shape
    hkv = case["hkv"]
    outs, lses = [], []
    for r in range(R):
        n = int(lens[r])
        k, v = (torch.cat([_row64(st, t["table"], kv, r, n - 1), new[kv][r:r + 1]]) for kv in range(2))
        s = torch.einsum("hgd,lhd->hgl", q[r].view(hkv, hq // hkv, d), k) * st["scale"]
        lses.append(torch.logsumexp(s, dim=-1).reshape(hq))
        outs.append(torch.einsum("hgl,lhd->hgd", torch.softmax(s, dim=-1), v).reshape(hq, d))
    return dict(res, out=torch.stack(outs), lse=torch.stack(lses))
