"""Plain references of the model-side operators: attention in 64 bits with error bounds, and the page cache as a
sequential program over Python lists."""
import math

import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # relative rounding of a value to the type


def attend64(q, k, v, scale, sees):
    """q [n, hq, d], k and v [m, hkv, d]; query i sees the first sees[i] keys.  Returns out, lse in float64 and the bounds the
    kernels are held to.

    The bounds, for inputs of a type with unit roundoff u, fp32 accumulation (2^-23 per step to allow for truncation):
      score    e = 2^-23 d sum|q k| scale + 2^-21 |s|, the second part for the scaling and for 2^x of an argument rounded to fp32
      lse      max e + 2^-20 max(1, |lse|)
      out      every probability is off by a factor 1 + u + 2 max e + 2^-20 (rounded to the type for the product, and
               normalised), the sum rounded once more:  (u + 2 max e + 2^-18) sum p|v| + u |out|, and in f16 probabilities
               below 2^-24 vanish: 2^-24 sum|v| over the keys seen, relative to a sum of at least 1."""
    n, hq, d = q.shape
    m, hkv = k.shape[0], k.shape[1]
    dev = q.device
    u = UNIT[q.dtype]
    q64, k64, v64 = q.double(), k.double(), v.double()
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=dev)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=dev)
    tol_out = torch.zeros_like(out)
    tol_lse = torch.zeros_like(lse)
    if m == 0 or n == 0:
        return out, lse, tol_out, tol_lse
    hidden = torch.arange(m, device=dev)[None, :] >= torch.as_tensor(sees, device=dev)[:, None]
    some = ~hidden.all(dim=1)
    for h in range(hq):
        g = h * hkv // hq
        s = (q64[:, h] @ k64[:, g].T) * scale
        e = 2.0 ** -23 * d * scale * (q64[:, h].abs() @ k64[:, g].abs().T) + 2.0 ** -21 * s.abs()
        e = e.masked_fill(hidden, 0.0).amax(dim=1)
        s = s.masked_fill(hidden, -math.inf)
        lse[:, h] = torch.logsumexp(s, dim=1)
        p = torch.softmax(s, dim=1)
        p[~some] = 0.0
        vis = torch.where(hidden[:, :, None], 0.0, v64[None, :, g]) if not torch.isfinite(v64).all() else None
        o = p @ v64[:, g] if vis is None else torch.einsum("nm,nmd->nd", p, vis)
        out[:, h] = o
        av = p @ v64[:, g].abs() if vis is None else torch.einsum("nm,nmd->nd", p, vis.abs())
        tol_out[:, h] = (u + 2 * e[:, None] + 2.0 ** -18) * av + u * o.abs() + 2.0 ** -30
        if q.dtype == torch.float16:
            tol_out[:, h] += 2.0 ** -24 * ((~hidden).double() @ torch.nan_to_num(v64[:, g]).abs())
        tol_lse[:, h] = e + 2.0 ** -20 * torch.nan_to_num(lse[:, h], neginf=0.0).abs().clamp(min=1.0)
    return out, lse, tol_out, tol_lse


def assert_attend(out, lse, ref):
    o, l, to, tl = ref
    none = torch.isinf(l) & (l < 0)
    assert torch.equal(torch.isinf(lse) & (lse < 0), none)
    assert torch.all(out[none] == 0)
    err = (out.double() - o).abs()
    assert torch.all(err <= to), (float((err - to).max()), float(err.max()))
    err = (lse.double() - l).abs()[~none]
    assert torch.all(err <= tl[~none]), float((err - tl[~none]).max())


class PlainCache:
    """The page cache, one row after the other, with the tokens' contents held as numpy arrays."""

    def __init__(self, pool, rows, width):
        self.pool = pool.copy()                      # [layers, 2, pages, heads, page, d]
        self.P = pool.shape[4]
        self.rows, self.width = rows, width
        self.pages = [[] for _ in range(rows)]
        self.len = [0] * rows
        self.n_pages = pool.shape[2]

    def ref(self):
        r = np.zeros(self.n_pages, np.int32)
        for ps in self.pages:
            for p in ps:
                r[p] += 1
        return r

    def table(self):
        t = np.full((self.rows, self.width), -1, np.int32)
        for r, ps in enumerate(self.pages):
            t[r, :len(ps)] = ps
        return t

    def fork(self, parent):
        old_pages, old_len = [list(p) for p in self.pages], list(self.len)
        for r, p in enumerate(parent):
            if 0 <= p < self.rows:
                self.pages[r], self.len[r] = list(old_pages[p]), old_len[p]
            else:
                self.pages[r], self.len[r] = [], 0

    def extend(self, add):
        P = self.P
        ref = self.ref()
        writers = {}
        fits_table = [add[r] > 0 and self.len[r] + add[r] <= self.width * P for r in range(self.rows)]
        for r in range(self.rows):
            if fits_table[r] and self.len[r] % P:
                writers.setdefault(self.pages[r][-1], []).append(r)
        need, copies = [], []
        for r in range(self.rows):
            c = 0
            if fits_table[r] and self.len[r] % P:
                page = self.pages[r][-1]
                stays = len(writers[page]) == ref[page] and writers[page][0] == r
                c = int(ref[page] > 1 and not stays)
            copies.append(c)
            need.append((-(-(self.len[r] + add[r]) // P) - len(self.pages[r]) + c) if fits_table[r] else 0)
        free = [p for p in range(self.n_pages) if ref[p] == 0]
        status = np.zeros(self.rows, np.uint8)
        at = 0
        before = self.pool.copy()
        for r in range(self.rows):
            if add[r] <= 0:
                continue
            if not fits_table[r]:
                status[r] = 32
                continue
            a, at = at, at + need[r]
            if need[r] and at > len(free):
                status[r] = 32
                continue
            got = free[a:at]
            if copies[r]:
                src, dst, fill = self.pages[r][-1], got[0], self.len[r] % P
                self.pool[:, :, dst, :, :fill] = before[:, :, src, :, :fill]
                self.pages[r][-1] = dst
                got = got[1:]
            self.pages[r] += got
            self.len[r] += int(add[r])
        return status

    def write(self, layer, k, v, seqs):
        """seqs: (row, first token in k, tokens) each"""
        for row, first, n in seqs:
            for j in range(n):
                pos = self.len[row] - n + j
                if pos >= 0:
                    page, off = self.pages[row][pos // self.P], pos % self.P
                    self.pool[layer, 0, page, :, off] = k[first + j]
                    self.pool[layer, 1, page, :, off] = v[first + j]

    def compact(self):
        ref = self.ref()
        n = int((ref > 0).sum())
        src = [p for p in range(n, self.n_pages) if ref[p] > 0]
        dst = [p for p in range(n) if ref[p] == 0]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.pool[:, :, d] = self.pool[:, :, s]
        self.pages = [[to.get(p, p) for p in ps] for ps in self.pages]
        return n
