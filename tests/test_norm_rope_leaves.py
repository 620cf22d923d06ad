"""What disc_norm_rope knows of the leaves it is given before a backward pass is captured: the books alone, on the CPU."""
import pytest
import torch

from paper_2504_09135_b200 import model_ops
from paper_2504_09135_b200.model_ops import _NOTE, _find_out, _leaf_node, _not_default, _note_foreign, _note_new


def leaf():
    return torch.ones(3, requires_grad=True)


def test_a_leaf_that_nothing_holds_is_new():
    x = leaf()
    assert not _note_foreign(x, None, torch.ones(3), leaf() * 2)
    (x * 2).sum().backward()           # a graph that is gone
    assert not _note_foreign(x)
    x.register_hook(lambda g: g)       # holds no node, nor does the next
    x.register_post_accumulate_grad_hook(lambda t: None)
    assert not _note_foreign(x)
    for on_default in (False, True):
        y = x * 2
        _note_new(y.grad_fn, on_default)
        assert _leaf_node(x).metadata[_NOTE] is on_default
        if on_default:
            with pytest.raises(RuntimeError, match="release them"):
                _not_default(y.grad_fn)
        else:
            _not_default(y.grad_fn)
        del y
        assert _NOTE not in _leaf_node(x).metadata


@pytest.mark.parametrize("stream", [0, 7])
def test_a_leaf_that_another_operation_holds(stream, monkeypatch):
    x, free = leaf(), leaf()
    other = (x * x).sum()
    assert _note_foreign(free, x)
    y = x * free
    _note_new(y.grad_fn, False)
    assert _leaf_node(x).metadata[_NOTE] is None and _leaf_node(free).metadata[_NOTE] is False
    with pytest.raises(RuntimeError, match="release them"):
        _not_default(y.grad_fn)
    # a backward pass shows where it runs
    monkeypatch.setattr(model_ops, "_stream_ptr", lambda: stream)
    _find_out(y.grad_fn)
    y.sum().backward()
    assert _leaf_node(x).metadata[_NOTE] is (stream == 0)
    assert _note_foreign(x) and _leaf_node(x).metadata[_NOTE] is (stream == 0)      # what is known stays
    z = x * 2
    if stream:
        _not_default(z.grad_fn)
    else:
        with pytest.raises(RuntimeError, match="release them"):
            _not_default(z.grad_fn)
    assert other.grad_fn is not None
    del other, y, z
    assert not _note_foreign(x) and _NOTE not in _leaf_node(x).metadata


def test_a_node_that_is_held_by_itself():
    x = leaf()
    held = _leaf_node(x)
    assert _note_foreign(x) and held.metadata[_NOTE] is None
    del held
    assert not _note_foreign(x)
