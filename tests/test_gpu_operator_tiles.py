"""The operators around the network in every tile and cut that a call of them can take (test_operator_plans holds the lists to that): values against the
definitions in 64 bits, at the smallest odd sizes that take them."""
import math

import pytest

from tests.test_gpu_classes import _compare, _inputs, _reference, _run
from tests.test_gpu_ortho import _check, _matrix, _polynomial, _tolerance, _view

pytestmark = pytest.mark.gpu

CLASSES = {
    "bf16": [(1, 9, 1870), (1, 133, 22686), (2, 66, 17006), (3, 3125, 60), (8, 1030, 121), (52, 2268, 81), (70, 9, 17347), (75, 17, 34338), (1215, 391, 2546), (1266, 8, 3),
             (1545, 865, 485), (2395, 992, 4099), (5540, 758, 2875), (17669, 67, 2), (33971, 65, 4), (1000, 2040, 50000),
             # several pieces of the classes
             (1, 8, 1052321), (1, 71, 1067861), (36, 15, 1176952), (72, 98, 1264743), (942, 132, 98413), (950, 8, 94619), (2476, 155, 38073), (5389, 84, 17088), (5713, 10, 15827),
             (9582, 445, 9378), (24025, 84, 3784), (42108, 15, 2181), (50056, 167, 1815)],
    "f32": [(1, 10, 1882), (2, 74, 17049), (4, 1063, 121), (783, 1227, 1442), (1043, 9, 3), (1148, 2059, 463), (16974, 69, 5), (17072, 8, 71),
            (1, 70, 1137216), (6, 8, 1059975), (72, 10, 1066320), (11383, 71, 7966), (103985, 77, 854), (194829, 8, 455)],
}
MATRICES = [[(2048, 4096)] * 2, [(4096, 2048)] * 2, [(2040, 2050)], [(2050, 2040)], [(4090, 4100)], [(4100, 4090)], [(1001, 333)] * 6, [(333, 1001)] * 6, [(512, 2048)], [(2047, 513)],
            [(8000, 2000), (70, 75)]]


@pytest.mark.parametrize("dtype,n,c,v", [(t, *s) for t in CLASSES for s in CLASSES[t]])
def test_classifier(dtype, n, c, v):
    x, w, b, y = _inputs(n, c, v, dtype, bias=(n + v) % 3 != 0, ignored=0.1 if n > 3 else 0.0, seed=n + v)
    got = _run(x, w, b, y, scale=2.0)
    assert bool((got["row_loss"] >= 0).all())
    _compare(got, _reference(x, w, b, y, scale=2.0), f"{n} x {c} -> {v} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", MATRICES, ids=lambda s: f"{len(s)}x{s[0][0]}x{s[0][1]}")
def test_orthogonalisation(shapes, dtype):
    from paper_2112_05387_amd import ops
    us = [_matrix(m, n, "noise", 7 * i + m, dtype) for i, (m, n) in enumerate(shapes)]
    for u, o in zip(us, ops.orthogonalize(us)):
        _check(o, u, f"{tuple(u.shape)} {dtype}")


@pytest.mark.parametrize("low,master", [(True, True), (True, False), (False, False)])
@pytest.mark.parametrize("shapes", MATRICES, ids=lambda s: f"{len(s)}x{s[0][0]}x{s[0][1]}")
def test_update(shapes, low, master):
    """The same with momentum before and the parameters behind: three fp32 operations, 2^-22 of the magnitudes, and the step times the tolerance of the
    orthogonalisation; bf16 parameters one rounding more."""
    import torch
    from paper_2112_05387_amd import ops
    dt = "bf16" if low else "f32"
    table, off, goff = [], 0, 0
    for shape in shapes:
        n = math.prod(shape)
        table.append((shape, dt, True, off, goff))
        off += -(-n * (2 if low else 4) // 256) * 256
        goff += -(-n * 4 // 64) * 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    r = lambda: torch.randn(goff // 4, generator=gen, device="cuda")
    grads, vel, full = 1e-2 * r(), 1e-1 * r(), r()
    params = torch.zeros(off, dtype=torch.uint8, device="cuda")
    for shape, _, _, o, go in table:
        _view(params, dt, o, math.prod(shape)).copy_(full[go // 4:go // 4 + math.prod(shape)])
    before, v_before = params.clone(), vel.clone()
    m = full.clone() if master else None
    lr, mu, wd = 0.05, 0.9, 0.1
    ops.muon_update(tuple(table), params, grads, vel, m, lr=lr, momentum=mu, weight_decay=wd)
    for shape, _, _, o, go in table:
        n, part = math.prod(shape), slice(go // 4, go // 4 + math.prod(shape))
        v = mu * v_before[part].double() + grads[part].double()
        assert float((vel[part].double() - v).norm()) <= 2.0 ** -22 * float(v.norm() + grads[part].norm())
        u = (grads[part].double() + mu * v).view(shape)
        old = (full[part] if master else _view(before, dt, o, n)).double()
        scale = lr * math.sqrt(max(1.0, shape[0] / shape[1]))
        new = old * (1 - lr * wd) - scale * _polynomial(u).reshape(-1)
        got = m[part] if master else _view(params, dt, o, n)
        tol = scale * _tolerance(u) + 2.0 ** -22 * float(old.norm() + new.norm()) + (2.0 ** -8 * float(new.norm()) if low and not master else 0.0)
        assert float((got.double() - new).norm()) <= tol
        if master:
            assert torch.equal(_view(params, dt, o, n), got.to(torch.bfloat16 if low else torch.float32))
