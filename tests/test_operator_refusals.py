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


def _mats(*m):
    return (B.lp_matrix * len(m))(*[B.lp_matrix(*v) for v in m])


def test_orthogonalisation():
    good = (8, 20, B.LP_F32, B.LP_BF16, FAKE, FAKE, 0, 0)
    need = B.lp_orthogonalize_workspace_bytes(_mats(good))
    assert need > 0 and B.lp_orthogonalize_workspace_bytes(_mats()) > 0
    for at, value, status in ((0, -1, B.LP_ERR_SHAPE), (1, (1 << 20) + 1, B.LP_ERR_SHAPE), (2, 2, B.LP_ERR_DTYPE), (3, -1, B.LP_ERR_DTYPE),
                              (6, 19, B.LP_ERR_SHAPE), (7, 3, B.LP_ERR_SHAPE)):
        bad = list(good)
        bad[at] = value
        _refused(status, lambda: B.lp_orthogonalize_workspace_bytes(_mats(bad)))
    _refused(B.LP_ERR_SHAPE, lambda: B.lp_orthogonalize_workspace_bytes(_mats((16385, 16385, 0, 0, FAKE, FAKE, 0, 0))))
    run = lambda m=good, steps=5, ws=FAKE, size=need: B.lp_orthogonalize(None, _mats(m), steps, ws, size)
    for steps in (0, B.LP_ORTHO_MAX_STEPS + 1):
        _refused(B.LP_ERR_INVALID_ARG, lambda: run(steps=steps))
    for at, value in ((4, None), (5, None), (4, FAKE + 2), (5, FAKE + 1)):
        bad = list(good)
        bad[at] = value
        _refused(B.LP_ERR_INVALID_ARG, lambda: run(bad))
    _refused(B.LP_ERR_WORKSPACE, lambda: run(ws=None))
    _refused(B.LP_ERR_WORKSPACE, lambda: run(size=need - 1))
    _refused(B.LP_ERR_INVALID_ARG, lambda: run(ws=FAKE + 16))
    many = (B.lp_matrix * (B.LP_ORTHO_MAX_MATRICES + 1))()
    _refused(B.LP_ERR_INVALID_ARG, lambda: B.lp_orthogonalize_workspace_bytes(many))
    empty = _mats((0, 5, 0, 0, None, None, 0, 0))          # nothing to do: nothing launched
    B.lp_orthogonalize(None, empty, 5, FAKE, B.lp_orthogonalize_workspace_bytes(empty))


def test_update_of_a_packed_set():
    tens = lambda *t: (B.lp_muon_tensor * len(t))(*[B.lp_muon_tensor(*v) for v in t])
    good = (8, 20, B.LP_BF16, 1, 256, 512)
    need = B.lp_muon_step_workspace_bytes(tens(good, (1, 16, B.LP_F32, 0, 0, 0)))
    for bad, status in (((0, 20, 0, 1, 0, 0), B.LP_ERR_INVALID_ARG), ((8, 0, 0, 0, 0, 0), B.LP_ERR_INVALID_ARG), ((8, 20, 7, 1, 0, 0), B.LP_ERR_DTYPE),
                        ((8, 20, B.LP_BF16, 1, 1, 0), B.LP_ERR_INVALID_ARG), ((8, 20, B.LP_F32, 1, 2, 0), B.LP_ERR_INVALID_ARG),
                        ((8, 20, B.LP_F32, 1, 0, 6), B.LP_ERR_INVALID_ARG), ((20000, 20000, B.LP_F32, 1, 0, 0), B.LP_ERR_SHAPE)):
        _refused(status, lambda: B.lp_muon_step_workspace_bytes(tens(bad)))
    ok = dict(params=FAKE, grads=FAKE, velocity=FAKE, master=None, opts=B.lp_muon_opts(0.1, 0.9, 0.0, 0.1, 1, 5), ws=FAKE, size=need)

    def run(**k):
        a = {**ok, **k}
        B.lp_muon_step(None, tens(good), a["params"], a["grads"], a["velocity"], a["master"], a["opts"], a["ws"], a["size"])

    for name in ("params", "grads", "velocity"):
        _refused(B.LP_ERR_INVALID_ARG, lambda: run(**{name: None}))
    for name in ("params", "grads", "velocity", "master"):
        _refused(B.LP_ERR_INVALID_ARG, lambda: run(**{name: FAKE + 8}))
    _refused(B.LP_ERR_INVALID_ARG, lambda: run(opts=B.lp_muon_opts(0.1, 0.9, 0.0, 0.1, 1, 0)))
    _refused(B.LP_ERR_WORKSPACE, lambda: run(size=256))


def test_update_of_a_network():
    import workloads as wl
    net = wl.make_config("tiny")
    h = B.lp_net_create(net.modules, None, "f32", 1e-5)
    try:
        opts = B.lp_muon_opts(0.1, 0.9, 0.0, 0.1, 1, 5)
        need = B.lp_muon_workspace_bytes(h, 0, 3, 0)
        assert B.lp_muon_workspace_bytes(h, 0, 1, 0) < need
        ok = dict(aux=0, mask=3, params=[FAKE] * 2, grads=[FAKE] * 2, vel=[FAKE] * 2, master=None, ws=FAKE, size=need)

        def run(**k):
            a = {**ok, **k}
            B.lp_muon_update(h, None, a["aux"], a["mask"], 0, a["params"], a["grads"], a["vel"], a["master"], opts, a["ws"], a["size"])

        for bad in (dict(params=None), dict(grads=None), dict(vel=None), dict(vel=[FAKE, None]), dict(params=[FAKE + 4, FAKE]), dict(master=[FAKE, FAKE + 2]),
                    dict(mask=0), dict(mask=4)):
            if bad.get("vel", 1) is None or bad.get("params", 1) is None or bad.get("grads", 1) is None:
                _refused(B.LP_ERR_INVALID_ARG, lambda: B.lp_muon_update(h, None, 0, 3, 0, *[{**ok, **bad}[k] for k in ("params", "grads", "vel", "master")], opts, FAKE, need))
            else:
                _refused(B.LP_ERR_INVALID_ARG, lambda: run(**bad))
        _refused(B.LP_ERR_STATE, lambda: run(aux=1, mask=1))
        _refused(B.LP_ERR_STATE, lambda: B.lp_muon_workspace_bytes(h, 1, 1, 0))
        _refused(B.LP_ERR_WORKSPACE, lambda: run(size=need - 1))
    finally:
        B.lp_net_destroy(h)


def test_operators_take_gpu_tensors_only():
    x, w, y = torch.zeros(4, 16), torch.zeros(10, 16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        ops.linear_ce_forward(x, w, y)
    with pytest.raises(ValueError, match="GPU"):
        ops.linear_ce_backward(x, w, y, torch.zeros(4))
    with pytest.raises(ValueError, match="GPU"):
        ops.orthogonalize([x])
    with pytest.raises(ValueError, match="GPU"):
        ops.muon_update((((4, 16), "f32", True, 0, 0),), torch.zeros(256, dtype=torch.uint8), torch.zeros(64), torch.zeros(64), lr=0.1)
    assert ops.orthogonalize([]) == []
