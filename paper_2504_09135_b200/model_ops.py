"""Binding of the operators the language model around the decoding step runs (include/disc.h):
attention over prompts, the paged key-value cache and attention over it, log-probabilities.

Argument marshalling only, like binding.py; there is no CPU fallback.  Outputs made here belong to the stream the call is
given (None: the current one).  A cache, a plan or an output used on another stream than the call before needs an event between
the two.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import DISC_BF16, DISC_F16, DISC_F32, DiscError, _Cache, _check, _dev, _here, _stream_ptr, lib

_HALF = {torch.bfloat16: DISC_BF16, torch.float16: DISC_F16}
_LOGIT = {torch.float32: DISC_F32, torch.bfloat16: DISC_BF16}


def _without_grad(t, name: str):
    if t.requires_grad and torch.is_grad_enabled():
        raise TypeError(f"{name}: requires a gradient, which this call does not give; detach it, or call under torch.no_grad()")


def _vectors(t: torch.Tensor, dtype, name: str):
    """A CUDA tensor [tokens, heads, head_dim] whose innermost axis is contiguous: (pointer, the two strides)."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype:
        if t.requires_grad:
            _without_grad(t, name)
        st = t.stride()
        if len(st) == 3 and (st[2] == 1 or t.shape[2] == 1):
            return _here(t, name), st[0], st[1]
    raise TypeError(f"{name}: expected a CUDA tensor [tokens, heads, head_dim] of {dtype} with unit inner stride")


def _spread(t: torch.Tensor, stream) -> torch.Tensor:
    """A copy where one vector stands for several tokens or heads (a stride of 0), which tensor maps do not take."""
    return _alloc(stream, t.contiguous) if 0 in t.stride() else t


def _rows(t: torch.Tensor, name: str):
    """Logits [n, V]: (pointer, dtype code, row stride)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.ndim == 2 and (t.stride(1) == 1 or t.shape[1] == 1)):
        raise TypeError(f"{name}: expected a CUDA tensor [n, V] with unit inner stride")
    if t.dtype not in _LOGIT:
        raise DiscError(-7, name)
    return _here(t, name), _LOGIT[t.dtype], t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _own(t):
    """Pointer of an output made here."""
    return 0 if t is None else t.data_ptr()


def _want(t, n: int, name: str):
    if t is not None and t.numel() != n:
        raise TypeError(f"{name}: expected {n} entries, got {t.numel()}")


def _empty(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


def _alloc(stream, make, *args):
    """make(*args) with its memory from the stream the kernel runs on: memory of another stream may still be in use there."""
    if stream is None:
        return make(*args)
    with torch.cuda.stream(stream):
        return make(*args)


# ---- log-probabilities ------------------------------------------------------------------------------
_LOGPROBS = ("logp", "entropy", "lse", "top_ids", "top_logp", "status")


class _Logprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, top, inv_temperature, stream):
        r = disc_logprobs(logits, targets, top=top, inv_temperature=inv_temperature, stream=stream)
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(r[k] for k in ("lse", "top_ids", "top_logp", "status") if r[k] is not None))
        ctx.save_for_backward(logits, targets, r["lse"], r["entropy"])
        ctx.inv_temperature = inv_temperature
        return tuple(r[k] for k in _LOGPROBS)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logp, d_entropy, *_):
        logits, targets, lse, entropy = ctx.saved_tensors
        if d_logp is None and d_entropy is None:
            return (None,) * 5
        d_logp, d_entropy = (None if d is None else d.contiguous() for d in (d_logp, d_entropy))
        return disc_logprobs_grad(logits, targets, lse, entropy, d_logp, d_entropy, inv_temperature=ctx.inv_temperature), None, None, None, None


def _logprobs_outputs(n: int, top: int, targets: bool, dev):
    f = torch.float32
    return {"logp": torch.empty(n, dtype=f, device=dev) if targets else None,
            "entropy": torch.empty(n, dtype=f, device=dev), "lse": torch.empty(n, dtype=f, device=dev),
            "top_ids": torch.empty_strided((n, top), (top, 1), dtype=torch.int32, device=dev) if top > 0 else None,
            "top_logp": torch.empty_strided((n, top), (top, 1), dtype=f, device=dev) if top > 0 else None,
            "status": torch.empty(n, dtype=torch.uint8, device=dev)}


def disc_logprobs(logits: torch.Tensor, targets: torch.Tensor | None = None, *, top: int = 0, inv_temperature=1.0,
                  out=None, stream=None):
    """logits [n, V] float32 or bfloat16 (any row stride), targets int32[n] (-1 = none) ->
    dict(logp, entropy, lse float[n], top_ids int32[n, top], top_logp float[n, top], status uint8[n]).
    Where logits require a gradient, logp and entropy have one (disc_logprobs_grad; its call goes to the current stream of
    this one); lse and the alternatives have none, and `out` is refused."""
    if isinstance(logits, torch.Tensor) and logits.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise TypeError("out: given buffers have no history; detach the logits, or call under torch.no_grad()")
        return dict(zip(_LOGPROBS, _Logprobs.apply(logits, targets, top, inv_temperature, stream)))
    ptr, dt, ld = _rows(logits, "disc_logprobs")
    n, V = logits.shape
    _want(targets, n, "targets")
    if out is None:
        out = _alloc(stream, _logprobs_outputs, n, top, targets is not None, logits.device)
    else:
        for k in _LOGPROBS:
            _want(out[k], n * top if k.startswith("top") else n, k)
            _dev(out[k], torch.int32 if k == "top_ids" else torch.uint8 if k == "status" else torch.float32, k)
    rc = lib().disc_logprobs(ptr, dt, ld, n, V, float(inv_temperature), _dev(targets, torch.int32, "targets"), int(top),
                             _own(out["logp"]), _own(out["entropy"]), _own(out["lse"]), _own(out["top_ids"]),
                             _own(out["top_logp"]), _own(out["status"]), _stream_ptr(stream))
    _check(rc, "disc_logprobs")
    return out


def disc_logprobs_grad(logits: torch.Tensor, targets, lse: torch.Tensor, entropy, d_logp, d_entropy=None, *,
                       inv_temperature=1.0, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gradient of sum(d_logp * logp + d_entropy * entropy) with respect to the logits, in their dtype.
    lse, entropy: what disc_logprobs gave for these logits.  out may be `logits` itself."""
    ptr, dt, ld = _rows(logits, "disc_logprobs_grad")
    n, V = logits.shape
    if logits.requires_grad:
        _without_grad(logits, "logits")
    for t, name in ((targets, "targets"), (lse, "lse"), (entropy, "entropy"), (d_logp, "d_logp"), (d_entropy, "d_entropy")):
        if t is not None and (t.requires_grad or t.numel() != n):
            _want(t, n, name)
            _without_grad(t, name)
    if out is None:
        out = _alloc(stream, _empty, (n, V), logits.dtype, logits.device)
    elif out.shape != logits.shape or out.dtype != logits.dtype:
        raise TypeError("out: expected the shape and dtype of the logits")
    optr, _, old = _rows(out, "out")
    rc = lib().disc_logprobs_grad(ptr, dt, ld, n, V, float(inv_temperature), _dev(targets, torch.int32, "targets"),
                                  _dev(lse, torch.float32, "lse"), _dev(entropy, torch.float32, "entropy"),
                                  _dev(d_logp, torch.float32, "d_logp"), _dev(d_entropy, torch.float32, "d_entropy"),
                                  optr, old, _stream_ptr(stream))
    _check(rc, "disc_logprobs_grad")
    return out


# ---- attention over prompts -------------------------------------------------------------------------
_F32, _DENSE = torch.float32, torch.contiguous_format


def _attend_outputs(q: torch.Tensor, out, lse):
    if out is None:
        out = torch.empty_like(q, memory_format=_DENSE)
    elif out.shape != q.shape or not _dev(out, q.dtype, "out") and out.numel():
        raise TypeError("out: expected q's shape")
    if lse is None:
        n, h, _ = q.shape
        lse = torch.empty_strided((n, h), (h, 1), dtype=_F32, device=q.device)
    elif lse.shape != q.shape[:2] or not _dev(lse, _F32, "lse") and lse.numel():
        raise TypeError("lse: expected [tokens, heads] of q")
    return out, lse


_error_words: dict = {}


def attend_error_word(device: torch.device) -> torch.Tensor:
    """The word an attention kernel sets when a bounded wait ran out, one per device."""
    w = _error_words.get(device)
    if w is None:
        w = _error_words[device] = torch.zeros(1, dtype=torch.int32, device=device)
        torch.cuda.synchronize(device)          # zero before any other stream uses it
    return w


def disc_attend_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k=None, *, max_len: int,
                       scale: float | None = None, causal: bool = True, out=None, lse=None, stream=None):
    """Attention over packed sequences: q [n_q, Hq, D], k and v [n_k, Hkv, D] (bf16 or f16, slices of a fused projection are
    fine), cu_q / cu_k int32[n_seqs + 1] on the device (cu_k None: the same sequences), max_len: no sequence
    has more queries -> (out [n_q, Hq, D], lse float[n_q, Hq]).  The first call on a device makes the word that
    disc_attend_check reads and waits for it: it comes before any stream capture."""
    dtype = q.dtype
    dt = _HALF.get(dtype)
    if dt is None:
        raise DiscError(-7, "disc_attend_prompt")
    qp, qt, qh = _vectors(q, dtype, "q")
    kp, kt, kh = _vectors(k, dtype, "k")
    vp, vt, vh = _vectors(v, dtype, "v")
    if not (qt and qh and kt and kh and vt and vh):
        q, k, v = _spread(q, stream), _spread(k, stream), _spread(v, stream)
        (qp, qt, qh), (kp, kt, kh), (vp, vt, vh) = _vectors(q, dtype, "q"), _vectors(k, dtype, "k"), _vectors(v, dtype, "v")
    n_q, hq, d = q.shape
    n_k, hkv, dk = k.shape
    if v.shape != k.shape or dk != d:
        raise TypeError("k, v: expected the same shape [n_k, Hkv, D] with q's head dim")
    n_seqs = cu_q.numel() - 1
    if cu_k is not None:
        _want(cu_k, n_seqs + 1, "cu_k")
    out, lse = _alloc(stream, _attend_outputs, q, out, lse)
    rc = lib().disc_attend_prompt(qp, qt, qh, kp, kt, kh, vp, vt, vh, dt, hq, hkv, d, n_q, n_k, _dev(cu_q, torch.int32, "cu_q"), _dev(cu_k, torch.int32, "cu_k"), n_seqs,
                                  int(max_len), int(causal), 1.0 / math.sqrt(d) if scale is None else float(scale),
                                  _own(out), _own(lse), attend_error_word(q.device).data_ptr(),
                                  _stream_ptr(stream))
    _check(rc, "disc_attend_prompt")
    return out, lse


def disc_attend_check(device="cuda", stream=None, *, plan: "AttendPlan | None" = None):
    """Synchronises and raises DiscError when a prompt attention on the device, or a cached attention with this plan, has given up
    on one of its bounded waits since the last check."""
    if plan is not None:
        word = plan.error
    else:
        dev = torch.device(device)
        if dev.index is None:
            dev = torch.device(dev.type, torch.cuda.current_device())
        word = attend_error_word(dev)
    rc = lib().disc_attend_error(word.data_ptr(), _stream_ptr(stream))
    try:
        if rc:
            _alloc(stream, word.zero_)          # reported once
    finally:
        _check(rc, "disc_attend_error")


# ---- the key-value cache ----------------------------------------------------------------------------
class DiscCache:
    """A key-value cache in pages: pool [layers, 2, pages, kv heads, page size, head dim] (bf16 or f16) and its
    books, one int32 buffer holding the page table [rows, table_width], the lengths [rows] and the reference
    counts [pages].  Without `book` the cache starts empty; a given buffer is used as it is."""

    def __init__(self, pool: torch.Tensor, n_rows: int, table_width: int, *, book: torch.Tensor | None = None):
        if not (isinstance(pool, torch.Tensor) and pool.is_cuda and pool.ndim == 6 and pool.shape[1] == 2 and pool.is_contiguous()):
            raise TypeError("pool: expected a contiguous CUDA tensor [layers, 2, pages, kv heads, page size, head dim]")
        if pool.dtype not in _HALF:
            raise DiscError(-7, "DiscCache")
        self.pool, self.n_rows, self.table_width = pool, int(n_rows), int(table_width)
        self.n_layers, _, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = pool.shape
        a, b = self.n_rows * self.table_width, self.n_rows * self.table_width + self.n_rows
        if book is None:
            book = torch.zeros(b + self.n_pages, dtype=torch.int32, device=pool.device)
            book[:a] = -1
        if not (book.is_cuda and book.dtype == torch.int32 and book.is_contiguous() and book.numel() == b + self.n_pages):
            raise TypeError(f"book: expected a contiguous int32 CUDA tensor of {b + self.n_pages} entries")
        self.book = book
        self.table, self.len, self.ref = book[:a].view(self.n_rows, self.table_width), book[a:b], book[b:]
        self._c = _Cache(pool.data_ptr(), self.table.data_ptr(), self.len.data_ptr(), self.ref.data_ptr(), None, 0,
                         self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim, self.n_rows,
                         self.table_width, _HALF[pool.dtype])
        self._p = C.addressof(self._c)
        need = lib().disc_cache_scratch_bytes(self._p)
        if need < 0:
            raise DiscError(int(need), "disc_cache_scratch_bytes")
        self._scratch = torch.empty(int(need), dtype=torch.uint8, device=pool.device)
        self._c.scratch, self._c.scratch_bytes = self._scratch.data_ptr(), int(need)
        self._plans: dict = {}
        self._sizes = tuple(pool.shape) + (self.n_rows, self.table_width, pool.dtype)

    @staticmethod
    def empty(n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, n_rows: int, table_width: int, *,
              dtype=torch.bfloat16, device="cuda") -> "DiscCache":
        pool = torch.zeros((n_layers, 2, n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device)
        return DiscCache(pool, n_rows, table_width)


def _books(cache: DiscCache) -> int:
    """Address of the cache's sizes and pointers; its memory is on one device."""
    _here(cache.pool, "cache")
    return cache._p


def disc_cache_fork(cache: DiscCache, parent: torch.Tensor, stream=None):
    """Row r becomes what row parent[r] was (int32[n_rows] on the device; outside [0, n_rows): emptied)."""
    _want(parent, cache.n_rows, "parent")
    _check(lib().disc_cache_fork(_books(cache), _dev(parent, torch.int32, "parent"), _stream_ptr(stream)), "disc_cache_fork")


def disc_cache_free(cache: DiscCache, freed: torch.Tensor, stream=None):
    """The rows with freed[r] != 0 (uint8[n_rows] on the device) become empty."""
    _want(freed, cache.n_rows, "freed")
    _check(lib().disc_cache_free(_books(cache), _dev(freed, torch.uint8, "freed"), _stream_ptr(stream)), "disc_cache_free")


def disc_cache_extend(cache: DiscCache, add: torch.Tensor | None = None, *, status: torch.Tensor | None = None,
                      stream=None) -> torch.Tensor:
    """Room for add[r] more tokens in every row (int32[n_rows] on the device, None: one each) -> status uint8[n_rows]."""
    _want(add, cache.n_rows, "add")
    if status is None:
        status = _alloc(stream, _empty, cache.n_rows, torch.uint8, cache.pool.device)
    else:
        _want(status, cache.n_rows, "status")
    _check(lib().disc_cache_extend(_books(cache), _dev(add, torch.int32, "add"), _dev(status, torch.uint8, "status"),
                                   _stream_ptr(stream)), "disc_cache_extend")
    return status


def disc_cache_write(cache: DiscCache, layer: int, k: torch.Tensor, v: torch.Tensor, *, cu: torch.Tensor | None = None,
                     rows: torch.Tensor | None = None, status: torch.Tensor | None = None, stream=None):
    """k, v [tokens, kv heads, head dim]: the newest tokens of sequence i (row rows[i], None: row i) are
    cu[i] .. cu[i+1]-1 (None: one token each)."""
    kp, kt, kh = _vectors(k, cache.pool.dtype, "k")
    vp, vt, vh = _vectors(v, cache.pool.dtype, "v")
    n, h, d = k.shape
    if v.shape != k.shape or h != cache.n_kv_heads or d != cache.head_dim:
        raise TypeError("k, v: expected [tokens, kv heads, head dim] of the cache")
    n_seqs = n if cu is None else cu.numel() - 1
    if rows is not None:
        _want(rows, n_seqs, "rows")
    _want(status, cache.n_rows, "status")
    _check(lib().disc_cache_write(_books(cache), int(layer), kp, kt, kh, vp, vt, vh, n, _dev(cu, torch.int32, "cu"), n_seqs,
                                  _dev(rows, torch.int32, "rows"), _dev(status, torch.uint8, "status"), _stream_ptr(stream)),
           "disc_cache_write")


def disc_cache_compact(cache: DiscCache, *, live: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The n pages in use move to the ids 0 .. n-1 -> n as int32[1] on the device."""
    if live is None:
        live = _alloc(stream, _empty, 1, torch.int32, cache.pool.device)
    _check(lib().disc_cache_compact(_books(cache), _dev(live, torch.int32, "live"), _stream_ptr(stream)), "disc_cache_compact")
    return live


# ---- attention of one new token per row ---------------------------------------------------------------
class AttendPlan:
    """Buffer of a plan (disc_attend_plan) and what it was made for; error: int32[1], not 0 once a cached attention with this
    plan gave up on a bounded wait, until disc_attend_check reports it."""

    def __init__(self, cache: DiscCache, n_q_heads: int, group: int):
        need = lib().disc_attend_plan_bytes(cache._p, int(n_q_heads), int(group))
        if need < 0:
            raise DiscError(int(need), "disc_attend_plan_bytes")
        self.n_q_heads, self.group, self.nbytes, self.sizes = int(n_q_heads), int(group), int(need), cache._sizes
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=cache.pool.device)
        self.error = self.buf[:4].view(torch.int32).zero_()
        self.made = False


def _of_cache(plan: AttendPlan, cache: DiscCache):
    # what lies where in the buffer hangs on the sizes: another layout would be read as page numbers
    if plan.sizes != cache._sizes:
        raise TypeError("plan: made for a cache of other sizes")


def disc_attend_plan(cache: DiscCache, n_q_heads: int, *, group: int = 1, plan: AttendPlan | None = None,
                     stream=None) -> AttendPlan:
    """The plan of one position for all layers: `group` consecutive rows (the K candidates of a query) may share
    leading pages.  Without `plan` the cache's own buffer for these sizes is used (and reused)."""
    if plan is None:
        plan = cache._plans.get((n_q_heads, group))
        if plan is None:
            plan = cache._plans[(n_q_heads, group)] = _alloc(stream, AttendPlan, cache, n_q_heads, group)
    else:
        _of_cache(plan, cache)
    _check(lib().disc_attend_plan(_books(cache), plan.n_q_heads, plan.group, plan.buf.data_ptr(), plan.nbytes, _stream_ptr(stream)),
           "disc_attend_plan")
    plan.made = True
    return plan


def disc_attend_cached(cache: DiscCache, layer: int, q: torch.Tensor, plan: AttendPlan, *, scale: float | None = None,
                       out=None, lse=None, stream=None):
    """One new token per row: q [rows, Hq, D] against the row's tokens in layer `layer` -> (out [rows, Hq, D],
    lse float[rows, Hq])."""
    qp, qr, qh = _vectors(q, cache.pool.dtype, "q")
    if not (qr and qh):
        q = _spread(q, stream)
        qp, qr, qh = _vectors(q, cache.pool.dtype, "q")
    n, h, d = q.shape
    if n != cache.n_rows or h != plan.n_q_heads or d != cache.head_dim:
        raise TypeError("q: expected [rows, Hq, head dim] of the cache and the plan")
    _of_cache(plan, cache)
    if not plan.made:
        raise TypeError("plan: not made yet (disc_attend_plan)")
    out, lse = _alloc(stream, _attend_outputs, q, out, lse)
    _check(lib().disc_attend_cached(_books(cache), int(layer), qp, qr, qh, plan.n_q_heads, plan.group,
                                    1.0 / math.sqrt(cache.head_dim) if scale is None else float(scale), plan.buf.data_ptr(),
                                    plan.nbytes, _own(out), _own(lse),
                                    _stream_ptr(stream)), "disc_attend_cached")
    return out, lse
