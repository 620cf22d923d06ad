"""Binding of the operators the language model around the decoding step runs (include/disc.h):
head norms and rotation, attention over prompts, the paged key-value cache and attention over it, log-probabilities.

Argument marshalling only, like binding.py; there is no CPU fallback.  Outputs made here belong to the stream the call is
given (None: the current one).  A cache, a plan or an output used on another stream than the call before needs an event between
the two.
"""
from __future__ import annotations

import ctypes as C
import math
import struct

import torch
import torch.autograd.forward_ad as _forward
from torch.autograd.graph import increment_version as _written      # what kernels write through a pointer, a graph that has saved it has to be told

from .binding import DISC_BF16, DISC_F16, DISC_F32, DISC_HELD_E4M3, DISC_HELD_I8, DiscError, _Cache, _check, _dev, _here, _stream_ptr, lib

_HALF = {torch.bfloat16: DISC_BF16, torch.float16: DISC_F16}
_LOGIT = {torch.float32: DISC_F32, torch.bfloat16: DISC_BF16}


def _without_grad(t, name: str):
    if t.requires_grad and torch.is_grad_enabled():
        raise TypeError(f"{name}: requires a gradient, which this call does not give; detach it, or call under torch.no_grad()")


def _without_tangent(t, name: str):
    if t is not None and _forward.unpack_dual(t).tangent is not None:
        raise TypeError(f"{name}: has a tangent, which this call's results would not have; take its primal")


def _vectors(t: torch.Tensor, dtype, name: str):
    """A CUDA tensor [tokens, heads, head_dim] whose innermost axis is contiguous: (pointer, the two strides)."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype:
        if t.requires_grad:
            _without_grad(t, name)
        if _forward._current_level >= 0:
            _without_tangent(t, name)
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
    if _forward._current_level >= 0:
        _without_tangent(t, name)
    return _here(t, name), _LOGIT[t.dtype], t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _own(t):
    """Pointer of an output made here."""
    return 0 if t is None else t.data_ptr()


def _want(t, n: int, name: str):
    if t is not None and t.numel() != n:
        raise TypeError(f"{name}: expected {n} entries, got {t.numel()}")


def _empty(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


def _two(shape, dtype, device):
    """Two contiguous tensors of three axes."""
    stride = (shape[1] * shape[2], shape[2], 1)
    return torch.empty_strided(shape, stride, dtype=dtype, device=device), torch.empty_strided(shape, stride, dtype=dtype, device=device)


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
    given = out is not None
    if not given:
        out = _alloc(stream, _logprobs_outputs, n, top, targets is not None, logits.device)
    else:
        for k in _LOGPROBS:
            _want(out[k], n * top if k.startswith("top") else n, k)
            _dev(out[k], torch.int32 if k == "top_ids" else torch.uint8 if k == "status" else torch.float32, k)
    rc = lib().disc_logprobs(ptr, dt, ld, n, V, float(inv_temperature), _dev(targets, torch.int32, "targets"), int(top),
                             _own(out["logp"]), _own(out["entropy"]), _own(out["lse"]), _own(out["top_ids"]),
                             _own(out["top_logp"]), _own(out["status"]), _stream_ptr(stream))
    _check(rc, "disc_logprobs")
    if given:
        _written([out[k] for k in _LOGPROBS if out[k] is not None])
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
        if _forward._current_level >= 0:
            _without_tangent(t, name)
    given = out is not None
    if not given:
        out = _alloc(stream, _empty, (n, V), logits.dtype, logits.device)
    elif out.shape != logits.shape or out.dtype != logits.dtype:
        raise TypeError("out: expected the shape and dtype of the logits")
    optr, _, old = _rows(out, "out")
    rc = lib().disc_logprobs_grad(ptr, dt, ld, n, V, float(inv_temperature), _dev(targets, torch.int32, "targets"),
                                  _dev(lse, torch.float32, "lse"), _dev(entropy, torch.float32, "entropy"),
                                  _dev(d_logp, torch.float32, "d_logp"), _dev(d_entropy, torch.float32, "d_entropy"),
                                  optr, old, _stream_ptr(stream))
    _check(rc, "disc_logprobs_grad")
    if given:
        _written(out)
    return out


_F32, _DENSE = torch.float32, torch.contiguous_format


# ---- head norms and rotation --------------------------------------------------------------------------
def _weights(dtype, d: int, norm, q_weight, k_weight):
    """Pointers of the norm's weights and their type."""
    if not norm:
        raise TypeError("q_weight, k_weight: the weights are the norm's; there is none")
    w = k_weight if q_weight is None else q_weight
    wt = dtype if w.dtype is dtype else _F32
    _want(q_weight, d, "q_weight")
    _want(k_weight, d, "k_weight")
    return _dev(q_weight, wt, "q_weight"), _dev(k_weight, wt, "k_weight"), DISC_F32 if wt is _F32 else _HALF[wt]


def _how(dtype, d: int, inv_freq, norm, q_weight, k_weight, interleaved):
    """What is done to the vectors, with the checks that need the tensors: the three pointers, then rot, interleaved, norm, weight type."""
    qw, kw, wt = (0, 0, 0) if q_weight is None and k_weight is None else _weights(dtype, d, norm, q_weight, k_weight)
    if _forward._current_level >= 0:
        for t, name in ((inv_freq, "inv_freq"), (q_weight, "q_weight"), (k_weight, "k_weight")):
            _without_tangent(t, name)
    if inv_freq is None:
        return (0, qw, kw), (0, 0, 1 if norm else 0, wt)
    return (_dev(inv_freq, _F32, "inv_freq"), qw, kw), (2 * inv_freq.numel(), 1 if interleaved else 0, 1 if norm else 0, wt)


# disc_norm_rope_t
_pack_call = struct.Struct("5Q10q4Qq3Q8ifi").pack


def _positions(positions, n: int, inv_freq):
    if positions is None:
        if inv_freq is not None:
            raise TypeError("positions: expected one per token")
        return 0
    if positions.numel() != n:
        _want(positions, n, "positions")
    return _dev(positions, torch.int32, "positions")


def _heads(q, k, where: str):
    """Shapes of q [n, Hq, D] and k [n, Hkv, D], either of which may be None: (dtype, n, Hq, Hkv, D)."""
    t = k if q is None else q
    if t is None:
        raise TypeError(f"{where}: neither queries nor keys")
    dtype, shape = t.dtype, t.shape
    if dtype not in _HALF:
        raise DiscError(-7, where)
    if len(shape) != 3:
        raise TypeError("q, k: expected [tokens, heads, head_dim]")
    n, hq, d = shape
    if q is None:
        return dtype, n, 0, hq, d
    if k is None:
        return dtype, n, hq, 0, d
    if k.dim() != 3 or k.shape[0] != n or k.shape[2] != d:
        raise TypeError("q, k: expected the same tokens and head_dim")
    return dtype, n, hq, k.shape[1], d


_NONE = (0, 0, 0)


def _given(t, out, name: str):
    """Pointer and strides of a given output for vectors t, which may be strided."""
    if out.shape != t.shape:
        raise TypeError(f"{name}: expected the shape of the vectors")
    v = _vectors(out, t.dtype, name)
    for size, stride in zip(out.shape[:2], v[1:]):
        if size > 1 and stride == 0:
            raise TypeError(f"{name}: one place for several tokens or heads")
    return v


def _dense(t, stream):
    """An output for vectors t, made here: the tensor, its pointer and strides."""
    o = torch.empty_like(t, memory_format=_DENSE) if stream is None else _alloc(stream, lambda: torch.empty_like(t, memory_format=_DENSE))
    _, h, d = t.shape
    return o, (o.data_ptr(), h * d, d)


def _aligned(t, stream):
    """Gradients come as autograd makes them: a copy where strides or base are not what the kernels take."""
    if t is None:
        return t
    a, b, c = t.stride()
    if c != 1 or (a | b) & 7 or t.data_ptr() & 15:
        t = _alloc(stream, lambda: t.clone(memory_format=torch.contiguous_format))
    return t


# A backward pass that is captured into a graph.  A leaf's node in autograd's graph lives as long as something holds it, and adds on the stream on
# which it came to be.  Another stream joins the capture, but the default stream's wait would end the process from a thread of autograd's.  So
# the node has a note: True for the default stream, False for another one, None where it is not known.
_NOTE, _ALIVE = "disc_default_stream", "disc_alive"


def _leaves(node):
    """Of a node of autograd's graph: the nodes behind it that add to a leaf's gradient."""
    return [n for n, _ in node.next_functions if type(n).__name__ == "AccumulateGrad"]


def _leaf_node(t):
    return torch.autograd.graph.get_gradient_edge(t).node


def _note_foreign(*tensors) -> bool:
    """Before a call: notes the leaves among `tensors` whose nodes something else holds, made who knows where, and says whether there are any.
    What is put on a node that nothing holds goes with it."""
    some = False
    for t in tensors:
        if t is not None and t.requires_grad and t.is_leaf:
            _leaf_node(t).metadata[_ALIVE] = True
            if _leaf_node(t).metadata.pop(_ALIVE, False):
                _leaf_node(t).metadata.setdefault(_NOTE, None)
                some = True
    return some


def _note_new(node, on_default: bool):
    """After a call: leaves without a note."""
    for n in _leaves(node):
        n.metadata.setdefault(_NOTE, on_default)


def _find_out(node):
    """In a backward pass that is not captured, before the leaves' nodes run: which stream they run on."""
    for n in _leaves(node):
        notes = n.metadata
        if notes.get(_NOTE, False) is None:
            n.register_prehook(lambda grads, notes=notes: notes.__setitem__(_NOTE, _stream_ptr() == 0))


def _not_default(node):
    """In a captured one."""
    for n in _leaves(node):
        if n.metadata.get(_NOTE, False) is not False:
            raise RuntimeError("disc_norm_rope: a backward pass is captured while results of an earlier call, or something else, hold graphs of the same leaf that "
                               "were made on the default stream, or nobody knows where; release them before the capture, or run a backward pass on another "
                               "stream before it, which finds out")


class _NormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, inv_freq, q_weight, k_weight, norm, eps, interleaved, stream):
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(q, k, positions, inv_freq, q_weight, k_weight)
        ctx.how, ctx.foreign = (norm, eps, interleaved), False
        return disc_norm_rope(q, k, positions, inv_freq, norm=norm, q_weight=q_weight, k_weight=k_weight, eps=eps, interleaved=interleaved, stream=stream)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_q, d_k):
        q, k, positions, inv_freq, qw, kw = ctx.saved_tensors
        norm, eps, interleaved = ctx.how
        need_q, need_k, _, _, need_qw, need_kw = ctx.needs_input_grad[:6]
        if d_q is None or not (need_q or need_qw):
            q = d_q = qw = None
        if d_k is None or not (need_k or need_kw):
            k = d_k = kw = None
        if q is None and k is None:
            return (None,) * 10
        if torch.cuda.is_current_stream_capturing():
            _not_default(ctx)
        elif ctx.foreign:
            _find_out(ctx)
        d_q, d_k, d_qw, d_kw = disc_norm_rope_grad(q, k, positions, inv_freq, d_q, d_k, norm=norm, q_weight=qw, k_weight=kw, eps=eps, interleaved=interleaved,
                                                   q_weight_grad=need_qw, k_weight_grad=need_kw)
        if d_qw is not None:
            d_qw = d_qw.to(qw.dtype)
        if d_kw is not None:
            d_kw = d_kw.to(kw.dtype)
        return d_q, d_k, None, None, d_qw, d_kw, None, None, None, None


def disc_norm_rope(q, k, positions, inv_freq=None, *, norm: bool = True, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                   out=None, stream=None):
    """Each head's RMS norm and the rotation by the token's position: q [n, Hq, D], k [n, Hkv, D] (bf16 or f16, slices of a fused
    projection are fine; either may be None), positions int32[n] -> (q', k').  inv_freq float32[rot / 2]: the first `rot` values
    of a vector are rotated (None: none); q_weight, k_weight [D] float32 or the vectors' type (None: 1).
    out: a pair of buffers of the same shapes, which may be q and k themselves, each its own, and otherwise overlap nothing.  Where
    an input or a weight requires a gradient the results have one (disc_norm_rope_grad; its call goes to the current stream of this
    one), and `out` is refused.  A backward pass that is captured into a graph is refused while something holds a graph of the same
    leaf, given to this call as it is, that was made on the default stream, or nobody knows where until a call on another stream
    has had a backward pass.  (Leaves that reach the call through other operations are not seen: the default stream's wait then ends
    the process, as it does under torch's own operations.)"""
    if torch.is_grad_enabled():
        if inv_freq is not None and inv_freq.requires_grad:
            _without_grad(inv_freq, "inv_freq")
        if any(t is not None and t.requires_grad for t in (q, k, q_weight, k_weight)):
            if out is not None:
                raise TypeError("out: given buffers have no history; detach the inputs, or call under torch.no_grad()")
            on_default = _stream_ptr() == 0
            foreign = not on_default and _note_foreign(q, k, q_weight, k_weight)
            y = _NormRope.apply(q, k, positions, inv_freq, q_weight, k_weight, norm, eps, interleaved, stream)
            node = (y[1] if y[0] is None else y[0]).grad_fn
            node.foreign = foreign
            _note_new(node, on_default)
            return y
    dtype, n, hq, hkv, d = _heads(q, k, "disc_norm_rope")
    qv = _NONE if q is None else _vectors(q, dtype, "q")
    kv = _NONE if k is None else _vectors(k, dtype, "k")
    ptrs, how = _how(dtype, d, inv_freq, norm, q_weight, k_weight, interleaved)
    pos = _positions(positions, n, inv_freq)
    if out is None:
        q_out, qo = (None, _NONE) if q is None else _dense(q, stream)
        k_out, ko = (None, _NONE) if k is None else _dense(k, stream)
    else:
        q_out, k_out = out
        qo, ko = _NONE if q is None else _given(q, q_out, "out"), _NONE if k is None else _given(k, k_out, "out")
    call = _pack_call(qv[0], kv[0], 0, qo[0], ko[0], qv[1], qv[2], kv[1], kv[2], 0, 0, qo[1], qo[2], ko[1], ko[2], pos, *ptrs, n, 0, 0, 0,
                      _HALF[dtype], hq, hkv, d, *how, eps, 0)
    _check(lib().disc_norm_rope(call, _stream_ptr(stream)), "disc_norm_rope")
    if out is not None:
        _written([o for t, o in ((q, q_out), (k, k_out)) if t is not None])
    return (q_out if q is not None else None), (k_out if k is not None else None)


def disc_norm_rope_grad(q, k, positions, inv_freq, d_q, d_k, *, norm: bool = True, q_weight=None, k_weight=None, eps: float = 1e-6,
                        interleaved: bool = False, q_weight_grad: bool = True, k_weight_grad: bool = True, stream=None):
    """From the gradients d_q, d_k of disc_norm_rope's results those of its inputs: (dq, dk, dq_weight, dk_weight), the weights' in
    float32 (None for a weight that is not given, or whose gradient is not asked for)."""
    dtype, n, hq, hkv, d = _heads(q, k, "disc_norm_rope_grad")
    if (q is None) != (d_q is None) or (q is not None and d_q.shape != q.shape):
        raise TypeError("d_q: expected the shape of the queries")
    if (k is None) != (d_k is None) or (k is not None and d_k.shape != k.shape):
        raise TypeError("d_k: expected the shape of the keys")
    d_q, d_k = _aligned(d_q, stream), _aligned(d_k, stream)
    qv, gqv = (_NONE, _NONE) if q is None else (_vectors(q, dtype, "q"), _vectors(d_q, dtype, "d_q"))
    kv, gkv = (_NONE, _NONE) if k is None else (_vectors(k, dtype, "k"), _vectors(d_k, dtype, "d_k"))
    if torch.is_grad_enabled():
        for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight"), (inv_freq, "inv_freq")):
            if w is not None and w.requires_grad:
                _without_grad(w, name)
    ptrs, how = _how(dtype, d, inv_freq, norm, q_weight, k_weight, interleaved)
    pos = _positions(positions, n, inv_freq)
    need = 0
    # the call's pointers are taken: from here on the weights stand for their gradients
    if not q_weight_grad:
        q_weight = None
    if not k_weight_grad:
        k_weight = None
    if q_weight is not None or k_weight is not None:
        need = lib().disc_norm_rope_scratch_bytes(hq, hkv, d, n)
        if need < 0:
            raise DiscError(int(need), "disc_norm_rope_scratch_bytes")
    gq, gk, gqw, gkw, scratch = _alloc(stream, _grad_outputs, q, k, q_weight, k_weight, need)
    call = _pack_call(qv[0], kv[0], 0, gqv[0], gkv[0], qv[1], qv[2], kv[1], kv[2], 0, 0, gqv[1], gqv[2], gkv[1], gkv[2], pos, *ptrs, n, 0, 0, 0,
                      _HALF[dtype], hq, hkv, d, *how, eps, 0)
    _check(lib().disc_norm_rope_grad(call, _own(gq), _own(gk), _own(gqw), _own(gkw), _own(scratch), need, _stream_ptr(stream)), "disc_norm_rope_grad")
    return gq, gk, gqw, gkw


def _grad_outputs(q, k, q_weight, k_weight, need: int):
    like = torch.empty_like
    return (None if q is None else like(q, memory_format=_DENSE), None if k is None else like(k, memory_format=_DENSE),
            None if q_weight is None else like(q_weight, dtype=_F32), None if k_weight is None else like(k_weight, dtype=_F32),
            torch.empty_strided((need,), (1,), dtype=torch.uint8, device=(k if q is None else q).device) if need else None)


# ---- attention over prompts -------------------------------------------------------------------------
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
    given = [t for t in (out, lse) if t is not None]
    out, lse = _alloc(stream, _attend_outputs, q, out, lse)
    rc = lib().disc_attend_prompt(qp, qt, qh, kp, kt, kh, vp, vt, vh, dt, hq, hkv, d, n_q, n_k, _dev(cu_q, torch.int32, "cu_q"), _dev(cu_k, torch.int32, "cu_k"), n_seqs,
                                  int(max_len), int(causal), 1.0 / math.sqrt(d) if scale is None else float(scale),
                                  _own(out), _own(lse), attend_error_word(q.device).data_ptr(),
                                  _stream_ptr(stream))
    _check(rc, "disc_attend_prompt")
    if given:
        _written(given)
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
_HELD = {None: 0, "e4m3": DISC_HELD_E4M3, "i8": DISC_HELD_I8}


class DiscCache:
    """A key-value cache in pages: pool [layers, 2, pages, kv heads, page size, head dim] (bf16 or f16) and its
    books, one int32 buffer holding the page table [rows, table_width], the lengths [rows] and the reference
    counts [pages].  Without `book` the cache starts empty; a given buffer is used as it is.

    held="e4m3" or "i8": vectors of type `dtype` held in 8 bits, one code per value and a power of two per vector; the pool is then
    uint8 [layers, 2, pages, kv heads, page_size * (head dim + 1)], a page and head's codes and behind them its exponents."""

    def __init__(self, pool: torch.Tensor, n_rows: int, table_width: int, *, book: torch.Tensor | None = None, held: str | None = None,
                 dtype: torch.dtype | None = None, page_size: int | None = None):
        if held not in _HELD:
            raise TypeError(f"held: expected None, 'e4m3' or 'i8', got {held!r}")
        if not (isinstance(pool, torch.Tensor) and pool.is_cuda and pool.ndim == (5 if held else 6) and pool.shape[1] == 2 and pool.is_contiguous()):
            raise TypeError("pool: expected a contiguous CUDA tensor [layers, 2, pages, kv heads, " + ("page size * (head dim + 1)]" if held else "page size, head dim]"))
        self.pool, self.n_rows, self.table_width, self.held = pool, int(n_rows), int(table_width), held
        if held:
            self.dtype = torch.bfloat16 if dtype is None else dtype
            if pool.dtype != torch.uint8 or not page_size or pool.shape[4] % page_size:
                raise TypeError("pool: expected uint8, with page_size tokens to a page")
            self.n_layers, _, self.n_pages, self.n_kv_heads, part = pool.shape
            self.page_size, self.head_dim = int(page_size), part // int(page_size) - 1
        else:
            self.dtype = pool.dtype
            self.n_layers, _, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = pool.shape
            if (dtype or pool.dtype) != pool.dtype or (page_size or self.page_size) != self.page_size:
                raise TypeError("pool: not of this dtype or page_size")
        if self.dtype not in _HALF:
            raise DiscError(-7, "DiscCache")
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
                         self.table_width, _HALF[self.dtype] | _HELD[held])
        self._p = C.addressof(self._c)
        need = lib().disc_cache_scratch_bytes(self._p)
        if need < 0:
            raise DiscError(int(need), "disc_cache_scratch_bytes")
        self._scratch = torch.empty(int(need), dtype=torch.uint8, device=pool.device)
        self._c.scratch, self._c.scratch_bytes = self._scratch.data_ptr(), int(need)
        self._plans: dict = {}
        self._sizes = tuple(pool.shape) + (self.n_rows, self.table_width, self.dtype, held, self.page_size)

    @staticmethod
    def empty(n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, n_rows: int, table_width: int, *,
              dtype=torch.bfloat16, device="cuda", held: str | None = None) -> "DiscCache":
        if held:
            pool = torch.zeros((n_layers, 2, n_pages, n_kv_heads, page_size * (head_dim + 1)), dtype=torch.uint8, device=device)
        else:
            pool = torch.zeros((n_layers, 2, n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device)
        return DiscCache(pool, n_rows, table_width, held=held, dtype=dtype, page_size=page_size)


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
    kp, kt, kh = _vectors(k, cache.dtype, "k")
    vp, vt, vh = _vectors(v, cache.dtype, "v")
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


def disc_norm_rope_write(cache: DiscCache, layer: int, q, k: torch.Tensor, v: torch.Tensor, inv_freq=None, *, positions=None, norm: bool = True,
                         q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False, cu: torch.Tensor | None = None,
                         rows: torch.Tensor | None = None, status: torch.Tensor | None = None, out=None, stream=None):
    """disc_norm_rope of the newest tokens' q (None: no queries) and k, and disc_cache_write of the resulting keys and of v, in one
    launch -> q'.  positions None: each token's place in its row.  out: a buffer for q', which may be q itself."""
    hq = 0 if q is None else q.shape[1]
    qv = _NONE if q is None else _vectors(q, cache.dtype, "q")
    kv, vv = _vectors(k, cache.dtype, "k"), _vectors(v, cache.dtype, "v")
    n, h, d = k.shape
    if v.shape != k.shape or h != cache.n_kv_heads or d != cache.head_dim:
        raise TypeError("k, v: expected [tokens, kv heads, head dim] of the cache")
    if q is not None and (q.shape[0] != n or q.shape[2] != d):
        raise TypeError("q: expected [tokens, Hq, head dim] with the keys' tokens")
    if torch.is_grad_enabled():
        for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight"), (inv_freq, "inv_freq")):
            if w is not None and w.requires_grad:
                _without_grad(w, name)
    ptrs, how = _how(cache.dtype, d, inv_freq, norm, q_weight, k_weight, interleaved)
    n_seqs = n if cu is None else cu.numel() - 1
    if rows is not None:
        _want(rows, n_seqs, "rows")
    _want(status, cache.n_rows, "status")
    _want(positions, n, "positions")
    given = q is not None and out is not None
    if q is None:
        out, qo = None, _NONE
    elif given:
        qo = _given(q, out, "out")
    else:
        out, qo = _dense(q, stream)
    call = _pack_call(qv[0], kv[0], vv[0], qo[0], 0, qv[1], qv[2], kv[1], kv[2], vv[1], vv[2], qo[1], qo[2], 0, 0, _dev(positions, torch.int32, "positions"),
                      *ptrs, n, _dev(cu, torch.int32, "cu"), _dev(rows, torch.int32, "rows"), _dev(status, torch.uint8, "status"),
                      _HALF[cache.dtype], hq, h, d, *how, eps, n_seqs)
    _check(lib().disc_norm_rope_write(_books(cache), int(layer), call, _stream_ptr(stream)), "disc_norm_rope_write")
    if given:
        _written(out)
    return out


def disc_cache_read(cache: DiscCache, layer: int, cu: torch.Tensor, n_tokens: int, *, rows: torch.Tensor | None = None,
                    start: torch.Tensor | None = None, out=None, stream=None):
    """Tokens of some rows, packed, in the cache's type: token cu[i] + j of the result is token start[i] + j (None: j) of row rows[i]
    (None: row i) -> (k, v) [n_tokens, kv heads, head dim]; zeros for tokens the row does not have.  n_tokens: cu[-1], or more
    (what lies behind is left as it is).  out: a pair of contiguous buffers of that shape."""
    n_seqs = cu.numel() - 1
    if rows is not None:
        _want(rows, n_seqs, "rows")
    if start is not None:
        _want(start, n_seqs, "start")
    shape = (int(n_tokens), cache.n_kv_heads, cache.head_dim)
    if out is None:
        k, v = _alloc(stream, _two, shape, cache.dtype, cache.pool.device)
    else:
        k, v = out
        for t, name in ((k, "k"), (v, "v")):
            _dev(t, cache.dtype, name)
            if t.shape != shape:
                raise TypeError(f"{name}: expected [n_tokens, kv heads, head dim]")
    _check(lib().disc_cache_read(_books(cache), int(layer), _dev(cu, torch.int32, "cu"), n_seqs, _dev(rows, torch.int32, "rows"),
                                 _dev(start, torch.int32, "start"), int(n_tokens), k.data_ptr(), v.data_ptr(), _stream_ptr(stream)), "disc_cache_read")
    if out is not None:
        _written(out)
    return k, v


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
    if plan.sizes is not cache._sizes and plan.sizes != cache._sizes:
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
    qp, qr, qh = _vectors(q, cache.dtype, "q")
    if not (qr and qh):
        q = _spread(q, stream)
        qp, qr, qh = _vectors(q, cache.dtype, "q")
    n, h, d = q.shape
    if n != cache.n_rows or h != plan.n_q_heads or d != cache.head_dim:
        raise TypeError("q: expected [rows, Hq, head dim] of the cache and the plan")
    _of_cache(plan, cache)
    if not plan.made:
        raise TypeError("plan: not made yet (disc_attend_plan)")
    given = [t for t in (out, lse) if t is not None]
    out, lse = _alloc(stream, _attend_outputs, q, out, lse)
    _check(lib().disc_attend_cached(_books(cache), int(layer), qp, qr, qh, plan.n_q_heads, plan.group,
                                    1.0 / math.sqrt(cache.head_dim) if scale is None else float(scale), plan.buf.data_ptr(),
                                    plan.nbytes, _own(out), _own(lse),
                                    _stream_ptr(stream)), "disc_attend_cached")
    if given:
        _written(given)
    return out, lse
