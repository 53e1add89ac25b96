"""Buffers of the orthogonalised update of a network: lists that are too short, or tensors of another size or type, are refused before the library reads their
addresses (no GPU needed)."""
import pytest
import torch

from paper_2112_05387_amd.runtime import _check_like

GRADS = [torch.zeros(64), torch.zeros(128), torch.zeros(32)]


def test_taken():
    _check_like("velocity", [torch.zeros_like(g) for g in GRADS], GRADS, 7)
    _check_like("velocity", [torch.zeros(200) for _ in range(4)], GRADS, 7)               # larger ones, more of them
    _check_like("velocity", [None, torch.zeros(128), None], GRADS, 2)                     # of the modules that are not selected: nothing


@pytest.mark.parametrize("mask,tensors", [
    (7, None), (7, []), (7, [torch.zeros(64)]), (4, [torch.zeros(64), torch.zeros(128)]), (7, [torch.zeros(64), None, torch.zeros(32)]), (2, [None, torch.zeros(127), None]),
    (1, [torch.zeros(64, dtype=torch.bfloat16), None, None]), (1, [torch.zeros(64, dtype=torch.float64), None, None]), (1, [torch.zeros(128)[::2], None, None]),
    (1, [torch.zeros(64, device="meta"), None, None])])
def test_refused(mask, tensors):
    with pytest.raises(ValueError, match="velocity"):
        _check_like("velocity", tensors, GRADS, mask)
