"""disc_norm_rope and its gradient against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2504_09135_b200 as disc
from held_reference import norm_rope64, tol_forward
from model_ops_reference import UNIT

pytestmark = pytest.mark.gpu
DEV = "cuda"


def frequencies(rot, base=10000.0):
    return torch.exp(torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) * (-math.log(base) / rot)).float() if rot else None


def inputs(n, hq, hkv, d, dtype, *, far=5000, seed=0, scale=1.0, weights=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    qkv = (torch.randn((n, hq + 2 * hkv, d), generator=g, device=DEV) * scale).to(dtype)
    q, k, _ = qkv.split([hq, hkv, hkv], dim=1)
    pos = torch.randint(0, far, (n,), generator=g, device=DEV, dtype=torch.int32)
    qw, kw = ((1 + 0.2 * torch.randn(d, generator=g, device=DEV)).to(weights) for _ in range(2))
    return q, k, pos, qw, kw


def check(got, x, w, pos, freq, **how):
    y, size = norm_rope64(x.double(), None if w is None else w.double(), pos, freq, **how)
    assert got.dtype == x.dtype and got.shape == x.shape
    err = (got.double() - y).abs()
    tol = tol_forward(y, size, x.dtype)
    assert torch.all(err <= tol), float((err - tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,hq,hkv,d,rot,inter,norm", [
    (1, 1, 1, 8, 8, False, True), (1, 16, 4, 128, 128, False, True), (3, 7, 1, 64, 64, True, True), (257, 8, 2, 128, 64, False, True),
    (33, 5, 3, 80, 40, True, False), (100, 4, 4, 96, 16, False, False), (64, 32, 8, 128, 128, True, True), (19, 2, 2, 72, 72, False, True),
    (50, 40, 8, 64, 0, False, True), (1000, 1, 1, 40, 8, False, True), (5, 3, 17, 112, 112, False, True)])
def test_forward(n, hq, hkv, d, rot, inter, norm, dtype):
    q, k, pos, qw, kw = inputs(n, hq, hkv, d, dtype)
    freq = frequencies(rot)
    w = (qw, kw) if norm else (None, None)
    a, b = disc.disc_norm_rope(q, k, pos if rot else None, freq, norm=norm, q_weight=w[0], k_weight=w[1], interleaved=inter)
    check(a, q, w[0], pos, freq, norm=norm, interleaved=inter)
    check(b, k, w[1], pos, freq, norm=norm, interleaved=inter)
    assert a.is_contiguous() and b.is_contiguous()


@pytest.mark.parametrize("inter", [False, True])
def test_far_and_negative_positions(inter):
    q, k, _, qw, kw = inputs(6, 4, 2, 128, torch.float16)
    pos = torch.tensor([0, 1 << 20, (1 << 31) - 1, -1, -(1 << 31), 999999], dtype=torch.int32, device=DEV)
    freq = frequencies(128)
    a, b = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw, interleaved=inter)
    check(a, q, qw, pos, freq, interleaved=inter)
    check(b, k, kw, pos, freq, interleaved=inter)


def test_one_of_the_two_weights_of_either_type_and_one_of_q_and_k():
    q, k, pos, qw, kw = inputs(21, 6, 2, 64, torch.bfloat16, weights=torch.bfloat16)
    freq = frequencies(32)
    a, b = disc.disc_norm_rope(q, k, pos, freq, k_weight=kw)
    check(a, q, None, pos, freq)
    check(b, k, kw, pos, freq)
    a2, none = disc.disc_norm_rope(q, None, pos, freq)
    assert none is None and torch.equal(a2, a)
    none, b2 = disc.disc_norm_rope(None, k, pos, freq, k_weight=kw)
    assert none is None and torch.equal(b2, b)
    b3 = disc.disc_norm_rope(q, k, pos, freq, k_weight=kw.float())[1]
    assert torch.equal(b3, b)


def test_in_place_strided_broadcast_and_empty():
    q, k, pos, qw, kw = inputs(40, 6, 2, 64, torch.bfloat16)
    freq = frequencies(64)
    want = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw)
    # every other token, into places of a wider buffer
    wide = torch.full((20, 16, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    got = disc.disc_norm_rope(q[::2], k[::2], pos[::2].contiguous(), freq, q_weight=qw, k_weight=kw, out=(wide[:, 2:8], wide[:, 10:12]))
    assert got[0].data_ptr() == wide[:, 2:8].data_ptr()
    assert torch.equal(wide[:, 2:8], want[0][::2]) and torch.equal(wide[:, 10:12], want[1][::2])
    assert bool((wide[:, :2] == 7).all() and (wide[:, 8:10] == 7).all() and (wide[:, 12:] == 7).all())
    one = q[:1, :1].expand(5, 3, 64)
    got = disc.disc_norm_rope(one, None, pos[:5], freq, q_weight=qw)[0]
    check(got, one, qw, pos[:5], freq)
    got = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    e = disc.disc_norm_rope(q[:0], k[:0], pos[:0], freq)
    assert e[0].shape == (0, 6, 64) and e[1].shape == (0, 2, 64)


def test_zeros_and_values_that_are_not_finite_stay_in_their_vector():
    q, k, pos, qw, kw = inputs(8, 4, 2, 128, torch.float16)
    q, k = q.contiguous(), k.contiguous()
    freq = frequencies(128)
    want = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw)
    q[2, 1, 5], q[3, 0, 0], q[4, 2] = math.nan, math.inf, 0.0
    got = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw)
    keep = torch.ones(8, 4, dtype=torch.bool, device=DEV)
    keep[2, 1] = keep[3, 0] = keep[4, 2] = False
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1], want[1])
    assert torch.isnan(got[0][2, 1]).all() and bool((got[0][4, 2] == 0).all())


def reference_grads(q, k, pos, freq, dq, dk, qw, kw, **how):
    x = [t.double().requires_grad_() for t in (q, k)]
    w = [None if t is None else t.double().requires_grad_() for t in (qw, kw)]
    y = [norm_rope64(a, b, pos, freq, **how)[0] for a, b in zip(x, w)]
    leaves = x + [t for t in w if t is not None]
    g = list(torch.autograd.grad(y, leaves, [dq.double(), dk.double()]))
    return g[:2] + [g.pop(2) if t is not None else None for t in w]


def grad_tol(x, dy, w, pos, freq, dtype, *, norm=True, eps=1e-6, interleaved=False):
    """Per vector: with r the inverse norm and G a bound of the rotated-back |g| (its pair's |dy_a| + |dy_b|), dx = r w g - x r^3 mean(w g x).  Each
    factor is off by less than 2^-16 of itself as in tol_forward, r^3 by three times that, the mean of D products by D 2^-24 more:
    2^-13 of r |w| G + |x| r^3 mean(|w| G |x|) holds both terms; and one rounding."""
    size = norm_rope64(dy.double(), None, pos, freq, norm=False, interleaved=interleaved)[1]
    if not norm:
        return size * 2.0 ** -13, None
    x = x.double()
    r = 1 / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + eps)
    c = size if w is None else size * w.double().abs()
    per_w = size * x.abs() * r
    return 2.0 ** -13 * (r * c + x.abs() * r ** 3 * (c * x.abs()).mean(dim=-1, keepdim=True)), per_w


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,hq,hkv,d,rot,inter,norm,weights", [
    (1, 1, 1, 8, 8, False, True, True), (1, 16, 4, 128, 128, False, True, True), (67, 8, 2, 64, 64, True, True, True), (130, 3, 1, 128, 32, False, True, False),
    (41, 5, 3, 80, 40, True, False, False), (1031, 4, 2, 96, 96, False, True, True), (9, 33, 1, 72, 0, False, True, True)])
def test_gradient(n, hq, hkv, d, rot, inter, norm, weights, dtype):
    q, k, pos, qw, kw = inputs(n, hq, hkv, d, dtype, far=100000)
    if not weights:
        qw = kw = None
    freq = frequencies(rot)
    g = torch.Generator(device=DEV).manual_seed(9)
    dq, dk = (torch.randn(t.shape, generator=g, device=DEV).to(dtype) for t in (q, k))
    how = dict(norm=norm, interleaved=inter)
    got = disc.disc_norm_rope_grad(q, k, pos if rot else None, freq, dq, dk, q_weight=qw, k_weight=kw, **how)
    want = reference_grads(q, k, pos, freq, dq, dk, qw, kw, **how)
    again = disc.disc_norm_rope_grad(q, k, pos if rot else None, freq, dq, dk, q_weight=qw, k_weight=kw, **how)
    for i, (x, dy, w) in enumerate(((q, dq, qw), (k, dk, kw))):
        tol, per_w = grad_tol(x, dy, w, pos, freq, dtype, **how)
        err = (got[i].double() - want[i]).abs()
        tol = tol + UNIT[dtype] * want[i].abs() + 2.0 ** -25
        assert got[i].dtype == dtype and torch.all(err <= tol), float((err - tol).max())
        if w is None:
            assert got[2 + i] is None
        else:
            # every term as above; a sum of N terms in fp32 is off by at most N 2^-24 of the sum of their sizes
            err, size = (got[2 + i].double() - want[2 + i]).abs(), per_w.sum(dim=(0, 1))
            terms = x.shape[0] * x.shape[1]
            assert got[2 + i].dtype == torch.float32 and torch.all(err <= size * (2.0 ** -14 + terms * 2.0 ** -24)), float(err.max())
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))


def test_gradient_against_differences():
    """<dy, (f(x + h) - f(x - h)) / 2> for small h along a random direction, f in 64 bits: the third-order term is below 1e-6 for |h| = 1e-3."""
    q, k, pos, qw, kw = inputs(12, 4, 2, 64, torch.float16)
    freq = frequencies(64)
    g = torch.Generator(device=DEV).manual_seed(3)
    dq, dk = (torch.randn(t.shape, generator=g, device=DEV).half() for t in (q, k))
    got = disc.disc_norm_rope_grad(q, k, pos, freq, dq, dk, q_weight=qw, k_weight=kw)
    for x, w, dy, dx, dw in ((q, qw, dq, got[0], got[2]), (k, kw, dk, got[1], got[3])):
        f = lambda a, b: (norm_rope64(a, b, pos, freq)[0] * dy.double()).sum()  # noqa: E731
        h = torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64) * 1e-3
        diff = float(f(x.double() + h, w.double()) - f(x.double() - h, w.double())) / 2
        size = float((dx.double() * h).abs().sum())
        assert abs(diff - float((dx.double() * h).sum())) <= size * (2.0 ** -11 + 2.0 ** -13) + 1e-6 * float(dy.double().abs().sum())
        h = torch.randn(w.shape, generator=g, device=DEV, dtype=torch.float64) * 1e-3
        diff = float(f(x.double(), w.double() + h) - f(x.double(), w.double() - h)) / 2
        size = float((norm_rope64(dy.double(), None, pos, freq, norm=False)[1] * 4 * h.abs()).sum())
        assert abs(diff - float((dw.double() * h).sum())) <= size * 2.0 ** -13


def test_autograd():
    q, k, pos, qw, kw = inputs(30, 4, 2, 64, torch.bfloat16)
    freq = frequencies(64)
    leaves = [t.detach().clone().requires_grad_() for t in (q, k, qw, kw.bfloat16())]
    y = disc.disc_norm_rope(leaves[0], leaves[1], pos, freq, q_weight=leaves[2])
    # a gradient that is broadcast, and one that is a transposed view
    (y[0].sum() + (y[1].transpose(0, 2) * torch.arange(30, device=DEV)).sum()).backward()
    ones = torch.ones_like(q)
    dk = torch.arange(30, device=DEV, dtype=torch.bfloat16)[:, None, None].expand(k.shape)
    want = disc.disc_norm_rope_grad(q, k, pos, freq, ones, dk, q_weight=qw)
    assert torch.equal(leaves[0].grad, want[0]) and torch.equal(leaves[1].grad, want[1]) and torch.equal(leaves[2].grad, want[2]) and leaves[3].grad is None
    # one of the results alone; a weight of the vectors' type has a gradient of that type
    leaves[0].grad = leaves[1].grad = None
    y = disc.disc_norm_rope(leaves[0], leaves[1], pos, freq, k_weight=leaves[3])
    y[1].float().square().sum().backward()
    assert leaves[0].grad is None and leaves[1].grad is not None and leaves[3].grad.dtype == torch.bfloat16
    # shared heads: one key head read by all
    one = torch.randn(30, 1, 64, device=DEV).bfloat16().requires_grad_()
    y = disc.disc_norm_rope(one.expand(30, 4, 64), None, pos, freq)
    y[0].backward(ones)
    parts = disc.disc_norm_rope_grad(one.detach().expand(30, 4, 64), None, pos, freq, ones, None)[0]
    assert torch.equal(one.grad, parts.sum(dim=1, keepdim=True))


def test_captured_and_on_another_stream():
    q, k, pos, qw, kw = inputs(50, 8, 2, 128, torch.bfloat16)
    freq = frequencies(128)
    want = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw)
    dq, dk = torch.randn_like(want[0]), torch.randn_like(want[1])
    want_g = disc.disc_norm_rope_grad(q, k, pos, freq, dq, dk, q_weight=qw, k_weight=kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw, stream=side)
    got_g = disc.disc_norm_rope_grad(q, k, pos, freq, dq, dk, q_weight=qw, k_weight=kw, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got + got_g, want + want_g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = disc.disc_norm_rope(q, k, pos, freq, q_weight=qw, k_weight=kw)
        got_g = disc.disc_norm_rope_grad(q, k, pos, freq, dq, dk, q_weight=qw, k_weight=kw)
    for _ in range(2):
        for t in got + got_g:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + got_g, want + want_g))


def test_a_captured_backward_pass_and_an_eager_graph_of_the_same_leaves():
    q, k, pos, qw, _ = inputs(40, 4, 2, 64, torch.bfloat16)
    freq, dy = frequencies(64), torch.randn((40, 4, 64), device=DEV).bfloat16()
    want = disc.disc_norm_rope_grad(q, None, pos, freq, dy, None, q_weight=qw)
    leaf, weight = q.clone().requires_grad_(), qw.clone().requires_grad_()

    def both():
        disc.disc_norm_rope(leaf, None, pos, freq, q_weight=weight)[0].backward(dy)

    held = disc.disc_norm_rope(leaf, None, pos, freq, q_weight=weight)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="release them"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            both()
    assert leaf.grad is None and weight.grad is None
    held[0].backward(dy)               # as before
    assert torch.equal(leaf.grad, want[0]) and torch.equal(weight.grad, want[2])
    del held
    leaf.grad = weight.grad = None
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for scale in (2.0, 1.0):
        dy.copy_(dy * scale)
        graph.replay()
    torch.cuda.synchronize()
    want = disc.disc_norm_rope_grad(q, None, pos, freq, dy, None, q_weight=qw)
    assert torch.equal(leaf.grad, want[0]) and torch.equal(weight.grad, want[2])


def test_a_captured_backward_pass_after_eager_ones_on_a_stream_of_their_own():
    q, _, pos, qw, _ = inputs(40, 4, 2, 64, torch.bfloat16)
    freq, dy = frequencies(64), torch.randn((40, 4, 64), device=DEV).bfloat16()
    want = disc.disc_norm_rope_grad(q, None, pos, freq, dy, None, q_weight=qw)
    leaf, weight = q.clone().requires_grad_(), qw.clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = disc.disc_norm_rope(leaf, None, pos, freq, q_weight=weight)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            disc.disc_norm_rope(leaf, None, pos, freq, q_weight=weight)[0].backward(dy)
    graph.replay()
    torch.cuda.synchronize()
    assert held[0].grad_fn is not None
    assert torch.equal(leaf.grad, want[0]) and torch.equal(weight.grad, want[2])


def test_calls_that_are_refused():
    q, k, pos, qw, kw = inputs(4, 4, 2, 64, torch.bfloat16)
    freq = frequencies(64)
    for bad, args, kw_args in [
            (TypeError, (None, None, pos, freq), {}), (TypeError, (q, k[:3], pos, freq), {}), (TypeError, (q, k, pos[:3], freq), {}),
            (TypeError, (q, k, None, freq), {}), (TypeError, (q, k, pos.long(), freq), {}), (TypeError, (q, k, pos, freq.double()), {}),
            (TypeError, (q, k.half(), pos, freq), {}), (disc.DiscError, (q.float(), k.float(), pos, freq), {}),
            (TypeError, (q, k, pos, freq), dict(q_weight=qw[:32])), (TypeError, (q, k, pos, freq), dict(q_weight=qw.double())),
            (TypeError, (q, k, pos, freq), dict(q_weight=qw, k_weight=kw.bfloat16())), (TypeError, (q, k, pos, freq), dict(q_weight=qw, norm=False)),
            (disc.DiscError, (q, k, pos, freq[:6]), {}), (disc.DiscError, (q, k, pos, frequencies(128)), {}), (disc.DiscError, (q, k, pos, freq), dict(eps=-1.0)),
            (disc.DiscError, (q, k, pos, freq), dict(eps=math.nan)), (TypeError, (q, k, pos, freq), dict(out=(k, k))),
            (TypeError, (q, k, pos, freq), dict(out=(q[:, :1].expand(4, 4, 64), k))), (disc.DiscError, (q[:, :, :60], None, pos, freq[:4]), {}),
            (TypeError, (q.cpu(), k, pos, freq), {}), (TypeError, (q, k, pos.cpu(), freq), {})]:
        with pytest.raises(bad):
            disc.disc_norm_rope(*args, **kw_args)
    with pytest.raises(TypeError):
        disc.disc_norm_rope(q.detach().requires_grad_(), k, pos, freq, out=(q, k))
    with pytest.raises(TypeError):
        disc.disc_norm_rope(q, k, pos, freq.clone().requires_grad_())
    with pytest.raises(TypeError):
        disc.disc_norm_rope_grad(q, k, pos, freq, q, None)
