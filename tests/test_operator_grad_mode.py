"""Tensors that autograd follows: the operators around the network know nothing of graphs, so they refuse them where a graph is being
recorded (no GPU needed)."""
import pytest
import torch

from paper_2112_05387_amd import ops

X, W, Y = torch.zeros(4, 16), torch.zeros(10, 16), torch.zeros(4, dtype=torch.int32)


def _calls(follow):
    """Every entry point with one of its tensors followed by autograd."""
    p = lambda t: t.clone().requires_grad_(follow)
    table = (((4, 16), "f32", True, 0, 0),)
    b, lse, u, flat = torch.zeros(10), torch.zeros(4), torch.zeros(256, dtype=torch.uint8), torch.zeros(64)
    yield lambda: ops.linear_ce_forward(p(X), W, Y)
    yield lambda: ops.linear_ce_forward(X, p(W), Y)
    yield lambda: ops.linear_ce_forward(X, W, Y, bias=p(b))
    yield lambda: ops.linear_ce_backward(X, p(W), Y, lse)
    yield lambda: ops.linear_ce_backward(X, W, Y, p(lse))
    yield lambda: ops.orthogonalize([X, p(W)])
    yield lambda: ops.muon_update(table, u, flat, flat.clone(), p(flat), lr=0.1)
    yield lambda: ops.muon_update(table, u, p(flat), flat.clone(), lr=0.1)


def test_followed_tensors_are_refused():
    for call in _calls(True):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()


def test_without_a_graph_they_are_taken():
    """... as far as the check of the device, which these fail."""
    with torch.no_grad():
        for call in _calls(True):
            with pytest.raises(ValueError, match="GPU"):
                call()
    for call in _calls(False):
        with pytest.raises(ValueError, match="GPU"):
            call()
