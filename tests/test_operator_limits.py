"""What the operators around the network refuse because of its size or place: packed tensors that lie outside their buffers or over
each other, launches larger than the device takes, sizes beyond the C ABI's integers (no GPU needed)."""
import pytest

from paper_2112_05387_amd import binding as B
from paper_2112_05387_amd import ops


def _refused(status, fn, *a):
    with pytest.raises(B.LpError) as e:
        fn(*a)
    assert e.value.status == status, str(e.value)


def _tensors(*t):
    return (B.lp_muon_tensor * len(t))(*[B.lp_muon_tensor(*v) for v in t])


FIRST = ((8, 20), "f32", True, 0, 0)


@pytest.mark.parametrize("entry", [((8, 20), "f32", True, -640, 1024), ((8, 20), "f32", True, 1024, -640), ((16,), "bf16", False, -2, 1024), ((16,), "f32", False, 1024, -(1 << 40))])
def test_packed_tensors_in_front_of_their_buffers(entry):
    with pytest.raises(ValueError, match="tensor 1: .*offset"):
        ops._muon_table((FIRST, entry))


def test_packed_tensors_far_outside():
    """An offset that wrapped round: the C entry knows no buffer's end, but none is as large as that."""
    for bad in ((8, 20, B.LP_F32, 1, 2 ** 64 - 640, 0), (8, 20, B.LP_F32, 1, 0, 2 ** 64 - 640), (8, 20, B.LP_F32, 1, 1 << 50, 0)):
        _refused(B.LP_ERR_INVALID_ARG, lambda: B.lp_muon_step_workspace_bytes(_tensors(bad)))
        _refused(B.LP_ERR_INVALID_ARG, lambda: B.lp_muon_step(None, _tensors(bad), 0x10000000, 0x10000000, 0x10000000, None, B.lp_muon_opts(0.1, 0.9, 0.0, 0.1, 1, 5), 0x10000000, 1 << 30))


@pytest.mark.parametrize("other", [((8, 20), "f32", True, 0, 640), ((8, 20), "f32", True, 640, 0), ((4,), "f32", False, 636, 1024), ((4,), "f32", False, 1024, 636),
                                   ((8, 20), "bf16", True, 320, 1024), ((1,), "f32", False, 300, 1024)])
def test_packed_tensors_over_each_other(other):
    """Shared parameters, or shared gradients and velocities, in either order of the list."""
    for table in ((FIRST, other), (other, FIRST), (FIRST, ((3,), "f32", False, 2048, 2048), other)):
        with pytest.raises(B.LpError, match="share"):
            ops._muon_table(table)
    # side by side they are taken
    ops._muon_table((FIRST, ((4,), "f32", False, 640, 640)))


def test_packed_tensors_beyond_the_integers():
    for shape in ((1, 1 << 31), (1 << 32, 3), ((1 << 32) + 5,), (1 << 33, 1 << 33)):
        with pytest.raises(ValueError, match="tensor 0"):
            ops._muon_table(((shape, "f32", False, 0, 0),))
    assert ops._muon_table((((1, (1 << 31) - 1), "f32", False, 0, 0),))[2] == 4 * ((1 << 31) - 1)


def test_classifier_launches():
    """A launch has fewer than 2^32 threads: the workspace query says so, not the launch behind the first kernels."""
    d = lambda n, c, v, t=B.LP_BF16: B.lp_linear_ce_desc(n, c, v, t, 0, 0, 0)
    _refused(B.LP_ERR_SHAPE, lambda: B.lp_linear_ce_workspace_bytes(d(65536, 64, 1 << 24), False))      # 2^24 tiles of 512 threads
    assert B.lp_linear_ce_workspace_bytes(d(65536, 64, 1 << 24), True) > 0                              # piece by piece
    assert B.lp_linear_ce_workspace_bytes(d(65536, 64, 1 << 22), False) > 0
    for backward in (False, True):
        _refused(B.LP_ERR_SHAPE, lambda: B.lp_linear_ce_workspace_bytes(d(1 << 26, 8, 4), backward))    # 2^24 workgroups of 256 for the rows
        assert B.lp_linear_ce_workspace_bytes(d((1 << 26) - 4, 8, 4), backward) > 0
    _refused(B.LP_ERR_SHAPE, lambda: B.lp_linear_ce_workspace_bytes(d(1 << 25, 65536, 4), True))        # dfeatures: 2^25 tiles and more


def test_orthogonalisation_launches():
    mats = lambda n, r, c: (B.lp_matrix * n)(*[B.lp_matrix(r, c, B.LP_F32, B.LP_F32, 0x10000000, 0x10000000, 0, 0) for _ in range(n)])
    assert B.lp_orthogonalize_workspace_bytes(mats(3, 1 << 20, 16384)) > 0
    _refused(B.LP_ERR_SHAPE, lambda: B.lp_orthogonalize_workspace_bytes(mats(4, 1 << 20, 16384)))       # 2^24 pieces, 256 threads each
    plain = lambda rows, cols: B.lp_muon_step_workspace_bytes(_tensors((rows, cols, B.LP_F32, 0, 0, 0)))
    assert plain((1 << 20) - 1, 1 << 15) > 0
    _refused(B.LP_ERR_SHAPE, lambda: plain(1 << 20, 1 << 15))                                           # 2^23 pieces of 4096 elements, 512 threads each


def test_matrices_beyond_the_integers(monkeypatch):
    """2^32 + 4 rows are not 4 rows."""
    import torch
    monkeypatch.setattr(ops, "_device", lambda *t: torch.device("cuda", 0))
    many = (1 << 32) + 4
    meta = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device="meta")
    for n, v in ((many, 10), (4, many)):
        with pytest.raises(ValueError, match="rows"):
            ops.linear_ce_forward(meta(n, 8), meta(v, 8), meta(n, t=torch.int32))
        with pytest.raises(ValueError, match="rows"):
            ops.linear_ce_backward(meta(n, 8), meta(v, 8), meta(n, t=torch.int32), meta(n))
    for shape in ((many, 4), (4, many)):
        with pytest.raises(ValueError, match="matrix 0"):
            ops.orthogonalize([meta(*shape)])
