"""The operators as a training step of one module uses them: forward pass, a classifier over the positions of the module's output
with its cross-entropy, the adjoint of that back through the module, and the update of the module's filters and of
the classifier by their orthogonalised momentum."""
import math

import numpy as np
import pytest

import workloads as wl
from oracle import lpref
from tests.gpu_common import TOL, gpu_mini_basic, gpu_mini_wide, load_step, say
from tests.helpers import rel_err, step_inputs
from tests.test_gpu_classes import _compare, _reference
from tests.test_gpu_ortho import _polynomial, _tolerance, _view

pytestmark = pytest.mark.gpu

LR, REST, MU, WD = 0.05, 0.02, 0.9, 0.01


class _Step:
    """Module 0 of a network with a classifier of its own at every position of its output."""

    def __init__(self, net, classes, seed=0):
        import torch
        from paper_2112_05387_amd import LocalStep
        self.net, self.inp = net, step_inputs(net, lpref)
        self.ls = LocalStep(net)
        self.ls.set_stream_lanes(None)
        load_step(self.ls, net, self.inp)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        rows, c = self.ls.y[0].numel() // self.ls.y[0].shape[-1], self.ls.y[0].shape[-1]
        self.low = net.dtype == "bf16"
        # the classifier's tensors packed like a module's: weight, bias
        size = -(-classes * c * (2 if self.low else 4) // 256) * 256
        self.table = (((classes, c), net.dtype, True, 0, 0), ((classes,), "f32", False, size, -(-classes * c // 64) * 256))
        self.head = torch.zeros(size + classes * 4, dtype=torch.uint8, device="cuda")
        self.dhead = torch.zeros(self.table[1][4] // 4 + classes, device="cuda")
        self.vhead = torch.zeros_like(self.dhead)
        self.weight = _view(self.head, net.dtype, 0, classes * c).view(classes, c)
        self.bias = _view(self.head, "f32", size, classes)
        self.weight.copy_(r(classes, c) / math.sqrt(c))
        self.bias.copy_(0.1 * r(classes))
        self.dweight = self.dhead[:classes * c].view(classes, c)
        self.dbias = self.dhead[self.table[1][4] // 4:]
        y = torch.randint(0, classes, (rows,), generator=g, device="cuda")
        self.labels = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.2, -1, y).to(torch.int32)
        self.velocity = [torch.zeros_like(t) for t in self.ls.dparams]
        self.state = [self.ls.params[0], self.velocity[0], self.head, self.vhead]

    def gradients(self):
        from paper_2112_05387_amd import ops
        ls = self.ls
        ls.module_forward(mask=1)
        rows = ls.y[0].view(-1, ls.y[0].shape[-1])
        self.loss, self.row_loss, self.lse = ops.linear_ce_forward(rows, self.weight, self.labels, bias=self.bias)
        self.dx, dw, db = ops.linear_ce_backward(rows, self.weight, self.labels, self.lse, bias=self.bias)
        self.dweight.copy_(dw)
        self.dbias.copy_(db)
        ls.dy[0].view(rows.shape).copy_(self.dx)
        ls.module_backward(mask=1)

    def update(self):
        from paper_2112_05387_amd import ops
        self.ls.muon_update(LR, self.velocity, momentum=MU, weight_decay=WD, rest_lr=REST, mask=1)
        ops.muon_update(self.table, self.head, self.dhead, self.vhead, lr=LR, momentum=MU, weight_decay=WD, rest_lr=REST)

    def host_loss(self, params, weight, bias):
        """The loss in 64 bits on the host."""
        y = lpref.module_forward(self.net.modules[0], self.inp["xs"][0], params, self.net.bn_eps)[0]
        x = y.reshape(-1, y.shape[-1])
        l = x @ weight.T + bias
        m = l.max(1)
        lse = m + np.log(np.exp(l - m[:, None]).sum(1))
        lab = self.labels.cpu().numpy()
        at = np.nonzero(lab >= 0)[0]
        return float((lse[at] - l[at, lab[at]]).mean())


@pytest.mark.parametrize("net", [gpu_mini_basic(), gpu_mini_basic(dtype="bf16"), gpu_mini_wide()], ids=["f32", "bf16", "bf16_wide"])
@pytest.mark.parametrize("classes", [11, 2500])
def test_a_module_and_its_classifier(net, classes):
    from paper_2112_05387_amd import binding as B
    s = _Step(net, classes)
    ls = s.ls
    try:
        for turn in range(2):
            before = [t.clone() for t in s.state]
            s.gradients()
            rows = ls.y[0].view(-1, ls.y[0].shape[-1])
            got = {"loss": s.loss, "row_loss": s.row_loss, "lse": s.lse, "dfeatures": s.dx, "dweight": s.dweight, "dbias": s.dbias}
            _compare(got, _reference(rows, s.weight, s.bias, s.labels), f"{net.name} {net.dtype} {classes} classes, step {turn}")
            if turn == 0:    # back through the module: the definition, from the adjoint as it is stored
                q = wl.round_bf16 if s.low else None
                m = net.modules[0]
                fwd = lpref.module_forward(m, s.inp["xs"][0], s.inp["params"][0], net.bn_eps, q)
                want = lpref.module_backward(m, fwd[2], dy=ls.to_host(ls.dy[0]), need_dx=False, q=q)[0]
                worst = [rel_err(a, b) for a, b in zip(ls.get_grads(0), want)]
                say(f"largest error of a parameter's gradient {max(worst):.1e}")
                assert max(worst) <= TOL[net.dtype]
            s.update()
            old, v_old = before[0], before[1]
            for i in ls.tables[0]:
                n, o = int(i.numel), i.grad_offset // 4
                dt = "bf16" if i.dtype == B.LP_BF16 else "f32"
                g, v = ls.dparams[0][o:o + n].double(), v_old[o:o + n].double()
                w, new = _view(old, dt, i.offset, n).double(), _view(s.state[0], dt, i.offset, n).double()
                if i.kind == B.LP_T_CONV:
                    step_scale = math.sqrt(max(1.0, i.dims[0] * i.dims[0] / n))
                    u = (g + MU * (MU * v + g)).view(i.dims[0], -1)
                    want = w * (1 - LR * WD) - LR * step_scale * _polynomial(u).reshape(-1)
                    tol = LR * step_scale * _tolerance(u)
                else:
                    want = w - REST * (MU * v + g + WD * w)
                    tol = 0.0
                tol += 2.0 ** -22 * float(w.norm() + want.norm()) + (2.0 ** -8 * float(want.norm()) if dt == "bf16" else 0.0)
                assert float((new - want).norm()) <= tol, (turn, tuple(i.dims[:i.ndim]))
    finally:
        ls.close()


def test_gradients_against_differences():
    """The loss along a random direction of all parameters: central differences in 64 bits, with two widths so that what the
    larger one is off by is seen, against the gradients' share of that direction.  Each gradient is held to TOL of its
    largest element, so the sum over a tensor may be off by that times the direction's magnitudes."""
    net = gpu_mini_basic()
    s = _Step(net, 9)
    try:
        s.gradients()
        rng = np.random.default_rng(3)
        have = [*s.ls.get_grads(0), s.ls.to_host(s.dweight), s.ls.to_host(s.dbias)]
        at = [*s.inp["params"][0], s.ls.to_host(s.weight), s.ls.to_host(s.bias)]
        for _ in range(3):
            d = [rng.standard_normal(np.shape(a)) for a in at]

            def slope(h):
                ends = [[np.asarray(a) + e * h * b for a, b in zip(at, d)] for e in (1, -1)]
                up, down = (s.host_loss(p[:-2], p[-2], p[-1]) for p in ends)
                return (up - down) / (2 * h)

            wide, narrow = slope(2e-6), slope(1e-6)
            mine = sum(float((g * b).sum()) for g, b in zip(have, d))
            tol = TOL["f32"] * sum(float(np.abs(g).max() * np.abs(b).sum()) for g, b in zip(have, d)) + 4 * abs(wide - narrow)
            say(f"slope {narrow:.6f} (wide {wide:.6f}), gradients {mine:.6f}, tolerance {tol:.1e}")
            assert abs(mine - narrow) <= tol
    finally:
        s.ls.close()


def test_the_step_as_a_graph():
    """Gradients and updates captured together and replayed, each replay against the eager step from the same state, bit by bit in the
    mode whose sums have a fixed order."""
    import torch
    from paper_2112_05387_amd import binding as B
    s = _Step(gpu_mini_wide(), 300)
    try:
        B.lp_net_set_deterministic(s.ls.net, True)
        start = [t.clone() for t in s.state]

        def restore():
            for t, v in zip(s.state, start):
                t.copy_(v)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.gradients()
            s.update()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        restore()
        eager = []
        for _ in range(3):
            s.gradients()
            s.update()
            eager.append([t.clone() for t in s.state] + [s.loss.clone()])
        restore()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.gradients()
            s.update()
        for turn in range(3):
            graph.replay()
            torch.cuda.synchronize()
            other = torch.randn(1000, 1000, device="cuda").sum()      # work of its own between the replays
            assert bool(other.isfinite())
            for a, b in zip(s.state + [s.loss], eager[turn]):
                assert torch.equal(a, b), turn
    finally:
        s.ls.close()
