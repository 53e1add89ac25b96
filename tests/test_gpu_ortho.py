"""Orthogonalisation by Newton-Schulz products and the parameter update by it, against the same polynomial in 64 bits.

Tolerances.  How far a rounding is carried depends on the matrix (a small singular value grows 3.4445 times a step, and what is
rounded in its direction with it), so the polynomial is evaluated in 64 bits a second time with every operand and every result
of its products disturbed at random, by p of itself and of its matrix's root mean square; four times the distance of the
two is the tolerance.  p = (sqrt(K) + K / 16 + 4) 2^-24: the walk and the drift of a sum of K products in fp32 on the matrix cores, and
the 2^-22 of an operand held in two fp16 parts.  A result in bf16 is rounded once more, 2^-8 of itself."""
import math

import pytest

from tests.gpu_common import say

pytestmark = pytest.mark.gpu

A, B_, C = 3.4445, -4.7750, 2.0315


def _polynomial(u, steps=5, p=0.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(99)

    def off(m):
        return m if p == 0.0 else m + p * (m.abs() + m.pow(2).mean().sqrt()) * torch.randn(m.shape, generator=g, device="cuda", dtype=torch.float64)

    x = u.double()
    x = off(x / x.norm().clamp(min=1e-7))
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    for _ in range(steps):
        s = off(x @ x.t())
        x = off(off(A * torch.eye(len(s), dtype=s.dtype, device=s.device) + B_ * s + C * off(s @ s)) @ x)
    return x.t() if tall else x


def _tolerance(u, steps=5):
    k = max(u.shape)
    p = (math.sqrt(k) + k / 16 + 4) * 2.0 ** -24
    return 4 * float((_polynomial(u, steps, p) - _polynomial(u, steps)).norm())


def _matrix(m, n, kind, seed, dtype="f32"):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    u = {"noise": lambda: r(m, n), "low_rank": lambda: r(m, 2) @ r(2, n), "large": lambda: 1e25 * r(m, n), "small": lambda: 1e-25 * r(m, n) + 1e-6,
         "zero": lambda: 0 * r(m, n)}[kind]()
    return u.to(torch.bfloat16) if dtype == "bf16" else u


def _check(got, u, what, steps=5):
    import torch
    want = _polynomial(u, steps)
    assert got.shape == u.shape
    off = float((got.double() - want).norm())
    tol = _tolerance(u, steps) + (2.0 ** -8 * float(want.norm()) if got.dtype == torch.bfloat16 else 0.0)
    say(f"{what}: off by {off:.2e} of {float(want.norm()):.2f}, tolerance {tol:.2e}")
    assert bool(got.isfinite().all()) and off <= tol


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (16, 27), (16, 144), (64, 576), (65, 63), (100, 10), (333, 1001), (1001, 333), (129, 640), (512, 2048), (1500, 1500), (3, 20000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", SHAPES)
def test_one_matrix(m, n, dtype):
    from paper_2112_05387_amd import ops
    u = _matrix(m, n, "noise", m + n, dtype)
    _check(ops.orthogonalize([u])[0], u, f"{m} x {n} {dtype}")


@pytest.mark.parametrize("m,n", [(32, 1152), (32, 1153), (33, 576), (64, 576), (64, 577), (1152, 32), (576, 64), (577, 64), (5, 1152), (33, 33), (1, 1200)])
def test_where_small_matrices_end(m, n):
    """Up to 64 rows a matrix stays in one workgroup where its columns fit."""
    from paper_2112_05387_amd import ops
    u = _matrix(m, n, "noise", m * n)
    _check(ops.orthogonalize([u])[0], u, f"{m} x {n}")


@pytest.mark.parametrize("kind", ["low_rank", "large", "small", "zero"])
@pytest.mark.parametrize("m,n", [(48, 200), (300, 70)])
def test_ill_conditioned_and_extreme_values(m, n, kind):
    from paper_2112_05387_amd import ops
    u = _matrix(m, n, kind, 3)
    _check(ops.orthogonalize([u])[0], u, f"{m} x {n} {kind}")


def test_large_matrices_and_many():
    """The largest tiles; more matrices than lanes of a wave, of all sizes at once, empty ones among them."""
    from paper_2112_05387_amd import ops
    import torch
    us = [_matrix(2048, 4100, "noise", 1), _matrix(4100, 2050, "noise", 2, "bf16")]
    for u, o in zip(us, ops.orthogonalize(us)):
        _check(o, u, f"{tuple(u.shape)}")
    us = [_matrix(1 + (37 * i) % 90, 1 + (53 * i) % 130, "noise", i, "bf16" if i % 3 == 0 else "f32") for i in range(150)]
    us[7] = torch.zeros((0, 5), device="cuda")
    us[8] = torch.zeros((5, 0), device="cuda")
    out = ops.orthogonalize(us)
    for i, (u, o) in enumerate(zip(us, out)):
        if u.numel():
            assert float((o.double() - _polynomial(u)).norm()) <= _tolerance(u) + (2.0 ** -8 * math.sqrt(min(u.shape)) * 1.21 if o.dtype == torch.bfloat16 else 0), i
        assert o.shape == u.shape


@pytest.mark.parametrize("steps", [1, 2, 7])
def test_steps(steps):
    from paper_2112_05387_amd import ops
    u = _matrix(50, 120, "noise", 5)
    _check(ops.orthogonalize([u], steps=steps)[0], u, f"{steps} steps", steps)


def test_singular_values_come_near_one():
    import torch
    from paper_2112_05387_amd import ops
    u = _matrix(64, 576, "noise", 5)
    s = torch.linalg.svdvals(ops.orthogonalize([u])[0].double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25


def test_strides_types_and_places():
    import torch
    from paper_2112_05387_amd import binding as B
    from paper_2112_05387_amd import ops
    wide = torch.full((40, 100), float("nan"), device="cuda")
    wide[:, 3:73] = _matrix(40, 70, "noise", 1)
    u = wide[:, 3:73]
    _check(ops.orthogonalize([u])[0], u, "row stride 100, four bytes off")
    _check(ops.orthogonalize([u.t()])[0], u.t(), "columns first")
    _check(ops.orthogonalize([u], out_dtype=torch.bfloat16)[0], u, "fp32 to bf16")
    want = ops.orthogonalize([u])[0]
    # in place, in the wider tensor, whose other columns stay
    mats = (B.lp_matrix * 1)(B.lp_matrix(40, 70, B.LP_F32, B.LP_F32, u.data_ptr(), u.data_ptr(), 100, 100))
    size = B.lp_orthogonalize_workspace_bytes(mats)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.lp_orthogonalize(torch.cuda.current_stream().cuda_stream, mats, 5, ws.data_ptr(), size)
    assert torch.equal(u, want) and bool(wide[:, :3].isnan().all()) and bool(wide[:, 73:].isnan().all())


def test_not_a_number_stays_in_its_matrix():
    from paper_2112_05387_amd import ops
    us = [_matrix(30, 50, "noise", i) for i in range(3)]
    us[1][4, 5] = float("nan")
    out = ops.orthogonalize(us)
    _check(out[0], us[0], "beside a NaN")
    _check(out[2], us[2], "beside a NaN")
    assert bool(out[1].isnan().all())


def test_same_bits_in_a_graph_and_on_another_stream():
    import torch
    from paper_2112_05387_amd import ops
    us = [_matrix(64, 576, "noise", 1), _matrix(300, 200, "noise", 2, "bf16")]
    first = ops.orthogonalize(us)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = ops.orthogonalize(us)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = ops.orthogonalize(us)
    for turn in range(3):
        us[0].copy_(_matrix(64, 576, "noise", 10 + turn))
        us[1].copy_(_matrix(300, 200, "noise", 20 + turn, "bf16"))
        g.replay()
        eager = ops.orthogonalize(us)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), turn


# ---- the update -----------------------------------------------------------------------------------------------------------------

TABLE_SHAPES = [((64, 3, 3, 64), True), ((16, 3, 3, 3), True), ((64,), False), ((10, 77), False), ((40, 33), True), ((33, 40), True), ((5,), False), ((200, 10), True)]


def _packed(low, seed, master):
    import torch
    table, off, goff = [], 0, 0
    for shape, orth in TABLE_SHAPES:
        n = math.prod(shape)
        dt = "bf16" if low and orth else "f32"
        table.append((shape, dt, orth, off, goff))
        off += -(-n * (2 if dt == "bf16" else 4) // 256) * 256
        goff += -(-n * 4 // 64) * 64
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"table": tuple(table), "params": torch.zeros(off, dtype=torch.uint8, device="cuda")}
    for k in ("grads", "velocity") + (("master",) if master else ()):
        s[k] = torch.randn(goff // 4, generator=g, device="cuda") * {"grads": 1e-2, "velocity": 1e-1, "master": 0.3}[k]
    for shape, dt, orth, o, go in table:
        n = math.prod(shape)
        w = s["master"][go // 4:go // 4 + n] if master else torch.randn(n, generator=g, device="cuda") * 0.3
        _view(s["params"], dt, o, n).copy_(w)
    return s


def _view(buf, dt, off, n):
    import torch
    return buf[off:off + 2 * n].view(torch.bfloat16) if dt == "bf16" else buf[off:off + 4 * n].view(torch.float32)


@pytest.mark.parametrize("low,master,nesterov", [(False, False, True), (True, False, False), (True, True, True), (False, True, False)])
def test_update_of_a_packed_set(low, master, nesterov):
    """Two updates in a row.  Velocity and the tensors by momentum: three fp32 operations, 2^-22 of the magnitudes; the others that and
    lr * scale times the tolerance of the orthogonalisation; bf16 parameters one rounding more."""
    import torch
    from paper_2112_05387_amd import ops
    s = _packed(low, 1, master)
    lr, rest, mu, wd = 0.05, 0.01, 0.9, 0.1
    for turn in range(2):
        before = {k: v.clone() for k, v in s.items() if k != "table"}
        ops.muon_update(s["table"], s["params"], s["grads"], s["velocity"], s.get("master"), lr=lr, momentum=mu, nesterov=nesterov, weight_decay=wd, rest_lr=rest)
        touched = torch.zeros_like(s["velocity"], dtype=torch.bool)
        for shape, dt, orth, o, go in s["table"]:
            n = math.prod(shape)
            part = slice(go // 4, go // 4 + n)
            touched[part] = True
            g, v = s["grads"][part].double(), before["velocity"][part].double()
            old = (before["master"][part] if master else _view(before["params"], dt, o, n)).double()
            if orth:
                v = mu * v + g
                u = g + mu * v if nesterov else v
                step = _polynomial(u.view(shape[0], -1)).reshape(-1) * math.sqrt(max(1.0, shape[0] * shape[0] / n))
                new = old * (1 - lr * wd) - lr * step
                tol = lr * math.sqrt(max(1.0, shape[0] * shape[0] / n)) * _tolerance(u.view(shape[0], -1)) + 2.0 ** -22 * float(old.norm() + new.norm())
            else:
                v = mu * v + g + wd * old
                new = old - rest * v
                tol = 2.0 ** -22 * float(old.norm() + new.norm() + v.norm())
            assert float((s["velocity"][part].double() - v).norm()) <= 2.0 ** -22 * float(v.norm() + g.norm() + old.norm())
            got = s["master"][part] if master else _view(s["params"], dt, o, n)
            assert float((got.double() - new).norm()) <= tol + (2.0 ** -8 * float(new.norm()) if not master and dt == "bf16" else 0.0), (turn, shape)
            if master:
                assert torch.equal(_view(s["params"], dt, o, n), got.to(torch.bfloat16 if dt == "bf16" else torch.float32))
        # what lies between the tensors stays
        for k in ("velocity",) + (("master",) if master else ()):
            assert torch.equal(s[k][~touched], before[k][~touched])
        assert torch.equal(s["grads"], before["grads"])


def test_update_of_many_tensors():
    """Small matrices, large ones and vectors in turn, more than go to the device at once: each as alone."""
    import torch
    from paper_2112_05387_amd import ops
    shapes = [(70 + i, 65 + 3 * i) if i % 5 == 0 else (8 + i, 9) if i % 5 < 3 else (3 + i,) for i in range(160)]
    table, off, goff = [], 0, 0
    for i, shape in enumerate(shapes):
        dt = "bf16" if i % 2 else "f32"
        table.append((shape, dt, len(shape) > 1, off, goff))
        off += -(-math.prod(shape) * 4 // 256) * 256 + (4 if i % 7 == 0 else 0)       # some of them unaligned
        goff += math.prod(shape) * 4
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    grads, vel = (torch.randn(goff // 4, generator=g, device="cuda") for _ in range(2))
    params = torch.zeros(off, dtype=torch.uint8, device="cuda")
    for shape, dt, orth, o, go in table:
        _view(params, dt, o, math.prod(shape)).copy_(torch.randn(math.prod(shape), generator=g, device="cuda"))
    one_p, one_v = params.clone(), vel.clone()
    ops.muon_update(tuple(table), params, grads, vel, lr=0.1, momentum=0.9, weight_decay=0.1, rest_lr=0.05)
    for t in table:
        ops.muon_update((t,), one_p, grads, one_v, lr=0.1, momentum=0.9, weight_decay=0.1, rest_lr=0.05)
    assert torch.equal(vel, one_v)
    for shape, dt, orth, o, go in table:
        n = math.prod(shape)
        a, b = (_view(p, dt, o, n).double() for p in (params, one_p))
        # (other tiles may add up in another order: each within its own tolerance of the definition)
        tol = 0.0
        if orth:
            u = (grads[go // 4:go // 4 + n] + 0.9 * vel[go // 4:go // 4 + n]).view(shape)
            tol = 2 * (0.1 * math.sqrt(max(1.0, shape[0] / shape[1])) * _tolerance(u) + (2.0 ** -8 if dt == "bf16" else 2.0 ** -22) * float(a.norm()))
        assert float((a - b).norm()) <= tol, shape


def test_first_call_inside_a_capture():
    """The kernels' attributes are set by the first call, which may be a captured one: in a process of its own."""
    import subprocess
    import sys
    code = """
import torch
from paper_2112_05387_amd import ops
g = torch.Generator(device="cuda"); g.manual_seed(0)
r = lambda *s: torch.randn(s, generator=g, device="cuda")
x, w, y = r(600, 100), r(2000, 100), torch.randint(0, 2000, (600,), generator=g, device="cuda").to(torch.int32)
us = [r(300, 200), r(64, 576), r(600, 700)]
def step():
    loss, rows, lse = ops.linear_ce_forward(x, w, y)
    dx, dw, _ = ops.linear_ce_backward(x, w, y, lse)
    lb, _, sb = ops.linear_ce_forward(x.bfloat16(), w.bfloat16(), y)
    return [loss, lse, dx, dw, lb, *ops.linear_ce_backward(x.bfloat16(), w.bfloat16(), y, sb)[:2], *ops.orthogonalize(us)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = step()
for _ in range(3):
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, step()))
print("same", flush=True)
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "same" in done.stdout, done.stderr[-2000:]


@pytest.mark.parametrize("dtype,head", [("f32", False), ("bf16", True)])
def test_update_of_a_network(dtype, head):
    """LocalStep.muon_update: every filter of a network orthogonalised, the rest by lp_sgd_update's rule; AuxNets; one module only."""
    import torch
    import workloads as wl
    from paper_2112_05387_amd import LocalStep
    from paper_2112_05387_amd import binding as B
    net = wl.make_config("resnet56", batch=2)
    net.dtype = dtype
    ls = LocalStep(net)
    try:
        gen = torch.Generator(device="cuda")
        gen.manual_seed(0)
        for aux in (False, True):
            tables, params, grads = (ls.aux_tables, ls.aux_params, ls.daux_params) if aux else (ls.tables, ls.params, ls.dparams)
            vel = [torch.zeros_like(g) for g in grads]
            master = [torch.zeros_like(g) for g in grads]
            for k, t in enumerate(tables):
                grads[k].copy_(torch.randn(grads[k].shape, generator=gen, device="cuda"))
                for i in t:
                    n, o = int(i.numel), i.grad_offset // 4
                    w = torch.randn(n, generator=gen, device="cuda")
                    master[k][o:o + n] = w
                    _view(params[k], "bf16" if i.dtype == B.LP_BF16 else "f32", i.offset, n).copy_(w)
            before = [m.clone() for m in master]
            ls.muon_update(0.1, vel, momentum=0.5, weight_decay=0.01, rest_lr=0.2, master=master, head=head, aux=aux)
            for k, t in enumerate(tables):
                for i in t:
                    n, o = int(i.numel), i.grad_offset // 4
                    g, old, new = (x[k][o:o + n] for x in (grads, before, master))
                    rows = i.dims[0]
                    if i.kind == B.LP_T_CONV or (head and i.kind == B.LP_T_FC_W):
                        want = old.double() * (1 - 0.1 * 0.01) - 0.1 * math.sqrt(max(1.0, rows * rows / n)) * _polynomial(g.view(rows, -1)).reshape(-1)
                        tol = 0.1 * math.sqrt(max(1.0, rows * rows / n)) * _tolerance(g.view(rows, -1)) + 2.0 ** -22 * float(old.norm() + want.norm())
                    else:
                        want = old.double() - 0.2 * (g.double() + 0.01 * old.double())
                        tol = 2.0 ** -22 * float(old.norm() + want.norm() + g.norm())
                    assert float((new.double() - want).norm()) <= tol, (aux, k, i.kind)
                    assert torch.equal(_view(params[k], "bf16" if i.dtype == B.LP_BF16 else "f32", i.offset, n), new.to(torch.bfloat16 if i.dtype == B.LP_BF16 else torch.float32))
        # one module only
        before = [p.clone() for p in ls.params]
        ls.muon_update(0.1, [torch.zeros_like(g) for g in ls.dparams], mask=4)
        torch.cuda.synchronize()
        assert [not torch.equal(a, b) for a, b in zip(before, ls.params)] == [k == 2 for k in range(net.K)]
    finally:
        ls.close()
