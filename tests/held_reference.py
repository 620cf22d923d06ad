"""Plain references of the head norms, the rotation and the vectors held in 8 bits, in 64 bits."""
import math

import numpy as np
import torch

from model_ops_reference import UNIT


# ---- norm and rotation -----------------------------------------------------------------------------------
def norm_rope64(x, w, pos, inv_freq, *, norm=True, eps=1e-6, interleaved=False):
    """x [n, heads, D] in float64 (differentiable), pos int, inv_freq float32 or None -> y, and |u_a| + |u_b| of each value."""
    u = x
    if norm:
        u = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + eps)
        if w is not None:
            u = u * w
    half = 0 if inv_freq is None else inv_freq.numel()
    if half == 0:
        return u, u.abs()
    t = pos.double()[:, None] * inv_freq.double()[None, :]
    cos, sin = torch.cos(t)[:, None], torch.sin(t)[:, None]
    ia = torch.arange(half, device=x.device)
    ia, ib = (2 * ia, 2 * ia + 1) if interleaved else (ia, ia + half)
    y, size = u.clone(), u.abs()
    a, b = u[..., ia], u[..., ib]
    y[..., ia] = a * cos - b * sin
    y[..., ib] = b * cos + a * sin
    size = size.clone()
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return y, size


def tol_forward(y, size, dtype):
    """What a result may be off by.  In fp32 a sum of D <= 128 squares is off by D 2^-24 of itself at most, its inverse root by half of
    that and 2 units more, each of the products with it, the weight, and the sines by 2^-24: below 2^-17 in all.  A sine's argument is
    a fraction of a turn, at most 1/2, rounded to fp32: 2^-26 of a turn, 2^-23.3.  So 2^-16 of |u_a| + |u_b| holds all of that, and the
    result is rounded once: u of it, or half of the type's smallest step, 2^-25 in f16."""
    return UNIT[dtype] * y.abs() + 2.0 ** -16 * size + 2.0 ** -25


# ---- 8 bits ------------------------------------------------------------------------------------------------
E4M3 = np.array([(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127])


def hold64(x, held):
    """x [..., D] (float64 array of finite values or not) -> codes uint8 [..., D], exponents int8 [...]; by a table of the codes' values."""
    amax = np.abs(x).max(axis=-1)
    fine = np.isfinite(amax)
    with np.errstate(divide="ignore"):
        lead = np.where(fine & (amax > 0), np.frexp(np.where(fine, amax, 1.0))[1] - 1, -10000)
    e = np.maximum(lead - (8 if held == "e4m3" else 6), -126)
    top = np.where(fine, amax, 0.0) * np.exp2(-e.astype(np.float64))
    e = e + ((top > 448) if held == "e4m3" else (np.rint(top) > 127))
    y = np.where(fine[..., None], x, 0.0) * np.exp2(-e.astype(np.float64))[..., None]
    if held == "i8":
        code = np.rint(y).astype(np.int8).view(np.uint8)
    else:
        a = np.abs(y)
        hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
        lo = hi - 1
        dl, dh = a - E4M3[lo], E4M3[hi] - a
        code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
        code = np.where(np.signbit(y), code | 0x80, code).astype(np.uint8)
    return code, np.where(fine, e, -128).astype(np.int8)


def values64(code, e, held):
    x = code.view(np.int8).astype(np.float64) if held == "i8" else np.where(code & 0x80, -1.0, 1.0) * E4M3[np.minimum(code & 0x7f, 126)]
    return np.where((e == -128)[..., None], math.nan, x * np.exp2(np.where(e == -128, 0, e).astype(np.float64))[..., None])


def parts(cache):
    """Codes [layers, 2, pages, heads, page, D] and exponents [layers, 2, pages, heads, page] of a held cache, as numpy arrays."""
    p = cache.pool.cpu().numpy()
    n = cache.page_size * cache.head_dim
    return p[..., :n].reshape(*p.shape[:-1], cache.page_size, cache.head_dim), p[..., n:].view(np.int8)


def place(cache, row, pos):
    table = cache.table.cpu().numpy()
    return int(table[row, pos // cache.page_size]), pos % cache.page_size


def held_rows(cache, layer, row, n):
    """Keys and values of a row's first n tokens as they are held, float64 [n, heads, D] each."""
    code, e = parts(cache)
    at = [place(cache, row, i) for i in range(n)]
    pages, offs = np.array([a[0] for a in at], np.int64), np.array([a[1] for a in at], np.int64)
    return [values64(code[layer, kv, pages, :, offs], e[layer, kv, pages, :, offs], cache.held) for kv in range(2)]


def tol_held(k, v, q, scale, u_out):
    """What attend64's bounds leave out, for one row: q [heads, D], k, v [n, kv heads, D] float64.  Probabilities times the values' powers of two
    are rounded to f16 relative to their largest, which loses 2^-25 of that for each token: with codes of at most 448 times
    2^e, of which the largest of a vector is at least 224 (e4m3) or 63 (i8), 2^e is at most amax / 63."""
    hq, hkv = q.shape[0], k.shape[1]
    out = torch.zeros(hq, q.shape[1], dtype=torch.float64, device=q.device)
    for h in range(hq):
        g = h * hkv // hq
        p = torch.softmax(k[:, g] @ q[h] * scale, dim=0)
        amax = v[:, g].abs().amax(dim=1).clamp(min=2.0 ** -140)
        weight = (p * amax).max()
        out[h] = 2.0 ** -25 * weight * (v[:, g].abs() / amax[:, None]).sum(dim=0) * 8
    return out
