"""What the operators around the network refuse, before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_2112_05387_amd import binding as B
from paper_2112_05387_amd import ops

FAKE = 0x10000000      # aligned, never dereferenced: every call below fails before a launch


def _refused(status, fn, *a):
    with pytest.raises(B.LpError) as e:
        fn(*a)
    assert e.value.status == status, str(e.value)


def _desc(rows=4, channels=16, classes=10, dtype=B.LP_F32, ldx=0, ldw=0, lddx=0):
    return B.lp_linear_ce_desc(rows, channels, classes, dtype, ldx, ldw, lddx)


@pytest.mark.parametrize("backward", [False, True])
def test_classifier_descriptors(backward):
    size = lambda **k: B.lp_linear_ce_workspace_bytes(_desc(**k), backward)
    for bad in (dict(rows=-1), dict(channels=0), dict(classes=0)):
        _refused(B.LP_ERR_INVALID_ARG, lambda: size(**bad))
    for bad in (dict(channels=65537), dict(classes=(1 << 24) + 1), dict(rows=(1 << 26) + 1), dict(ldx=15), dict(ldw=8), dict(lddx=-1)):
        _refused(B.LP_ERR_SHAPE, lambda: size(**bad))
    _refused(B.LP_ERR_DTYPE, lambda: size(dtype=2))
    assert size(rows=0) > 0
    # more rows of the same classes need no less
    assert size(rows=64, classes=5000) >= size(rows=8, classes=5000) > 0


def test_classifier_workspace_does_not_grow_with_the_logits():
    """Probabilities exist a piece at a time: 32 Gi of them, a workspace of a few per cent."""
    d = _desc(rows=65536, channels=1024, classes=500000, dtype=B.LP_BF16)
    assert B.lp_linear_ce_workspace_bytes(d, True) < 4 * 65536 * 500000 // 50
    assert B.lp_linear_ce_workspace_bytes(d, False) < 4 * 65536 * 500000 // 50


def test_classifier_calls():
    d = _desc()
    need = B.lp_linear_ce_workspace_bytes(d, False)
    ok = dict(features=FAKE, weight=FAKE, bias=None, labels=FAKE, loss=FAKE, row_loss=None, lse=FAKE, ws=FAKE, size=need)

    def forward(**k):
        a = {**ok, **k}
        B.lp_linear_ce_forward(d, None, a["features"], a["weight"], a["bias"], a["labels"], a["loss"], a["row_loss"], a["lse"], a["ws"], a["size"])

    for name in ("features", "weight", "labels", "loss", "lse"):
        _refused(B.LP_ERR_INVALID_ARG, lambda: forward(**{name: None}))
    for name in ("features", "weight", "ws"):
        _refused(B.LP_ERR_INVALID_ARG, lambda: forward(**{name: FAKE + 8}))
    _refused(B.LP_ERR_WORKSPACE, lambda: forward(ws=None))
    _refused(B.LP_ERR_WORKSPACE, lambda: forward(size=need - 1))

    need_b = B.lp_linear_ce_workspace_bytes(d, True)

    def backward(**k):
        a = {**dict(ok, size=need_b, dx=FAKE, dw=FAKE, db=None), **k}
        B.lp_linear_ce_backward(d, None, a["features"], a["weight"], a["bias"], a["labels"], a["lse"], 1.0, a["dx"], a["dw"], a["db"], a["ws"], a["size"])

    for name in ("features", "weight", "labels", "lse"):
        _refused(B.LP_ERR_INVALID_ARG, lambda: backward(**{name: None}))
    for name in ("features", "weight", "dw", "ws"):
        _refused(B.LP_ERR_INVALID_ARG, lambda: backward(**{name: FAKE + 4}))
    _refused(B.LP_ERR_WORKSPACE, lambda: backward(size=need_b - 1))
    backward(dx=None, dw=None, db=None)            # nothing asked for: nothing launched


def test_operators_take_gpu_tensors_only():
    x, w, y = torch.zeros(4, 16), torch.zeros(10, 16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        ops.linear_ce_forward(x, w, y)
    with pytest.raises(ValueError, match="GPU"):
        ops.linear_ce_backward(x, w, y, torch.zeros(4))
