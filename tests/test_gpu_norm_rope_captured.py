"""Captured backward passes of disc_norm_rope beside graphs of the same leaves that other operations have made."""
import pytest
import torch

import paper_2504_09135_b200 as disc
from paper_2504_09135_b200.model_ops import _NOTE, _leaf_node

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Call:
    def __init__(self):
        g = torch.Generator(device=DEV).manual_seed(3)
        self.q = torch.randn((40, 4, 64), generator=g, device=DEV).bfloat16().requires_grad_()
        self.w = (1 + 0.2 * torch.randn(64, generator=g, device=DEV)).requires_grad_()
        self.dy = torch.randn((40, 4, 64), generator=g, device=DEV).bfloat16()
        self.pos = torch.arange(40, dtype=torch.int32, device=DEV)
        self.freq = torch.exp(torch.arange(32, device=DEV) * (-0.2))
        self.want = disc.disc_norm_rope_grad(self.q.detach(), None, self.pos, self.freq, self.dy, None, q_weight=self.w.detach())
        torch.cuda.synchronize()

    def forward(self):
        return disc.disc_norm_rope(self.q, None, self.pos, self.freq, q_weight=self.w)[0]

    def both(self):
        self.forward().backward(self.dy)

    def clear(self):
        self.q.grad = self.w.grad = None

    def captured(self, stream=None):
        self.clear()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            self.both()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(self.q.grad, self.want[0]) and torch.equal(self.w.grad, self.want[2])
        return graph

    def refused(self, stream=None):
        self.clear()
        with pytest.raises(RuntimeError, match="release them"):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
                self.both()
        assert self.q.grad is None and self.w.grad is None


def test_the_first_call_is_the_captured_one():
    c = Call()
    penalty = c.w.square().sum()       # on the default stream
    c.refused()
    penalty.backward()                 # as before
    assert torch.equal(c.w.grad, 2 * c.w.detach())
    del penalty
    c.captured()


@pytest.mark.parametrize("backward_too", [False, True])
def test_earlier_calls_on_another_stream_and_a_graph_made_on_the_default_one(backward_too):
    c = Call()
    penalty = c.w.square().sum()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        if backward_too:
            c.both()
        else:
            held = c.forward()
    torch.cuda.synchronize()
    assert _leaf_node(c.w).metadata[_NOTE] is (True if backward_too else None)
    c.refused(side)
    held = penalty = None  # noqa: F841
    c.captured(side)


def test_a_graph_made_on_another_stream():
    c = Call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        penalty = c.w.square().sum()
    c.refused(side)                    # nobody knows yet
    with torch.cuda.stream(side):
        c.both()
    torch.cuda.synchronize()
    assert _leaf_node(c.w).metadata[_NOTE] is False
    c.captured(side)
    assert penalty.grad_fn is not None
