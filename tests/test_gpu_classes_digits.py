"""Cross-entropy of a linear classifier where digits are easily lost: gradients in bf16 whose sums cancel, probabilities that have to be held to
fp32's 24 bits, rows that are all but certain, classes at the type's lowest value, pieces of the classes, differences of the loss.

Tolerances as in test_gpu_classes; where they are tighter the arithmetic stands with the test."""
import math

import pytest

from tests.gpu_common import say
from tests.test_gpu_classes import U32, _compare, _inputs, _reference, _run, _steps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,c,v", [(700, 16, 9000), (64, 512, 1000), (3000, 40, 60), (5, 64, 20000), (2000, 136, 300)])
def test_what_all_classes_have_in_common(n, c, v):
    """sum_v d_nv is zero, so what the rows of the weights have in common does not reach the gradient of the features.  A channel that is zero in
    all features and 64 in all weights: its logits are untouched, its gradient is 64 times the sum of d, off by what d is off by: the
    error of p (logits and lse) and 2^-16 of |d| for what is held of it; the features are small, so that the logits are exact
    to far less than bf16's 2^-9."""
    import torch
    x, w, b, y = _inputs(n, c, v, "bf16", seed=21)
    x = (x.float() / 16).bfloat16()
    x[:, 0] = 0
    w[:, 0] = 64
    got = _run(x, w, b, y, scale=float(n))["dfeatures"][:, 0].double()
    l = x.double() @ w.double().t() + b.double()
    # the channel of zeros adds nothing to any rounding
    tl = _steps(c) * (x.double().abs() @ w.double().abs().t() + b.double().abs()) + 4 * U32 * l.abs()
    lse = l.logsumexp(1, keepdim=True)
    p = torch.exp(l - lse)
    tp = p * (tl + tl.max(1, keepdim=True).values + 8 * U32 * (2 * lse.abs() + l.abs() + 1))
    d = p.scatter_add(1, y.long()[:, None], torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda"))
    tol = 64 * ((tp + 2.0 ** -16 * d.abs()).sum(1) + 2 * _steps(v) * d.abs().sum(1))
    exact = 64 * d.sum(1)
    worst = float(((got - exact).abs() / tol).max())
    say(f"{n} x {c} -> {v}: largest share of the tolerance {worst:.2f}")
    assert worst <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,v", [(256, 300), (64, 20000), (128, 1100), (512, 9000), (1040, 130)])
def test_probabilities_to_24_bits(n, v, dtype):
    """Features are the identity and the weights zero: the logits are the bias, and the gradient of the weights is d itself, transposed, every sum
    of one term.  p = exp(l - lse) from lse in fp32: the difference, its product with log2 e and that constant are off by
    3 |l - lse| 2^-24, exp2 and the scale by 2^-23 each, the parts in which d is held by 2^-24; p - 1 rounds once more.  The
    gradient of the bias is summed over four rows that count, three additions and exact zeros."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(v)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.eye(n, device="cuda").to(t)
    w = torch.zeros(v, n, dtype=t, device="cuda")
    b = torch.rand(v, generator=gen, device="cuda") - 0.5
    y = torch.randint(0, v, (n,), generator=gen, device="cuda").to(torch.int32)
    from paper_2112_05387_amd import ops
    lse = ops.linear_ce_forward(x, w, y, bias=b)[2]
    l = b.double().expand(n, v)
    off = l - lse.double()[:, None]
    p = off.exp()
    rel = (3 * off.abs() + 8) * U32
    for few in (False, True):
        if few:
            y = torch.where(torch.arange(n, device="cuda") % (n // 4) == 3, y, -1).to(torch.int32)
        keep = (y >= 0).double()[:, None]
        at = y.clamp(min=0).long()[:, None]
        d = p.scatter_add(1, at, torch.full((n, 1), -1.0, dtype=torch.float64, device="cuda")) * keep
        tol = (p * rel + 2 * U32 * d.abs()) * keep
        count = int(keep.sum())
        _, dw, db = ops.linear_ce_backward(x, w, y, lse, bias=b, scale=float(count))
        worst = float(((dw.double().t() - d).abs() / (tol + 1e-37)).max())
        say(f"{n} -> {v} {dtype}, {count} rows: dweight {worst:.2f} of the tolerance")
        assert worst <= 1.0
    worst = float(((db.double() - d.sum(0)).abs() / (tol.sum(0) + 4 * U32 * d.abs().sum(0))).max())
    say(f"{n} -> {v} {dtype}: dbias {worst:.2f} of the tolerance")
    assert worst <= 1.0


CERTAIN = [(33, 2026, 234), (256, 640, 100), (300, 512, 4000), (1, 2026, 3000), (33, 2048, 2048), (32, 2048, 2049), (20, 300, 9000), (2600, 200, 3000), (5000, 96, 64),
           (777, 333, 2345), (1, 2048, 60000)]


def _certain(n, c, v, dtype):
    """As rows are at the end of a training: the score of the right class stands out by 16 to 22 lengths of its weights."""
    x, w, b, y = _inputs(n, c, v, dtype, bias=n % 2 == 0, ignored=0.1 if n > 3 else 0.0, seed=18)
    x = (x.float() + 16 * w.float()[y.clamp(min=0).long()] * (y >= 0)[:, None]).to(x.dtype)
    want = _reference(x, w, b, y, certain=True)
    assert float(want["row_loss"][0].median()) < 0.05
    return x, w, b, y, want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,v", CERTAIN)
def test_losses_of_nearly_certain_rows(n, c, v, dtype):
    """A row's loss keeps its digits, however many rows and classes there are, and is never negative."""
    from paper_2112_05387_amd import ops
    x, w, b, y, want = _certain(n, c, v, dtype)
    got = dict(zip(("loss", "row_loss", "lse"), ops.linear_ce_forward(x, w, y, bias=b)))
    assert bool((got["row_loss"] >= 0).all())
    _compare(got, want, f"losses of nearly certain rows {n} x {c} -> {v} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,v", CERTAIN)
def test_gradients_of_nearly_certain_rows(n, c, v, dtype):
    """... and its gradient."""
    x, w, b, y, want = _certain(n, c, v, dtype)
    _compare(_run(x, w, b, y), want, f"gradients of nearly certain rows {n} x {c} -> {v} {dtype}")


@pytest.mark.parametrize("dtype,n,c,v", [("f32", 12, 32, 40), ("f32", 64, 512, 1000), ("f32", 300, 32, 9000), ("bf16", 300, 32, 9000), ("bf16", 64, 2048, 1000), ("bf16", 3000, 64, 300)])
def test_every_class_at_the_lowest_value(dtype, n, c, v):
    """The logits are lost in the bias, and all of them are the same: log v a row, and an lse that is the lowest value (log v is lost in it, so that the
    gradient, which starts from it, has no meaning)."""
    import torch
    from paper_2112_05387_amd import ops
    x, w, b, y = _inputs(n, c, v, dtype, ignored=0.2, seed=6)
    lowest = torch.finfo(torch.float32).min
    loss, rows, lse = ops.linear_ce_forward(x, w, y, bias=torch.full_like(b, lowest))
    keep = y >= 0
    assert bool((lse == lowest).all()) and bool((rows[~keep] == 0).all())
    assert float((rows[keep] / math.log(v) - 1).abs().max()) <= 8 * U32 + _steps(v)
    assert abs(float(loss[0]) / math.log(v) - 1) <= 16 * U32 + _steps(v)


PIECES = [("bf16", 8000, 2048, 45000), ("bf16", 8192, 60, 45003), ("f32", 8192, 40, 45003)]


@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("dtype,n,c,v", PIECES)
def test_large_pieces_of_the_classes(dtype, n, c, v, certain):
    """Probabilities of all classes would take more than the workspace holds at once: several pieces, the last one ragged, the gradient of the features added up
    over them; and rows whose own class lies in one piece and what is left of them in all."""
    from paper_2112_05387_amd import binding as B
    d = B.lp_linear_ce_desc(n, c, v, B.LP_BF16 if dtype == "bf16" else B.LP_F32, 0, 0, 0)
    assert B.lp_linear_ce_workspace_bytes(d, True) < 4 * n * c * 16 + 6 * n * v
    x, w, b, y = _inputs(n, c, v, dtype, ignored=0.1, seed=7)
    if certain:
        x = (x.float() + 16 * w.float()[y.clamp(min=0).long()] * (y >= 0)[:, None]).to(x.dtype)
    got = _run(x, w, b, y)
    assert bool((got["row_loss"] >= 0).all())
    _compare(got, _reference(x, w, b, y, certain=certain), f"pieces {n} x {c} -> {v} {dtype}")


@pytest.mark.parametrize("n,c,v", [(30, 12, 40), (300, 32, 9000), (64, 512, 1000), (1500, 24, 3000)])
def test_gradient_along_itself(n, c, v):
    """Central differences of the loss along the gradient, where they are far above what they are off by: the losses (row by row, added in 64 bits) by
    the tolerance of a row's loss over the step, the third derivative of log sum exp by at most 2 (2 m)^3 / 6 h^2 where no logit moves by more
    than m; h m = 1/32."""
    import torch
    from paper_2112_05387_amd import ops
    x, w, b, y = _inputs(n, c, v, "f32", ignored=0.1, seed=4)
    want = _reference(x, w, b, y)
    count = int((y >= 0).sum())
    _, _, lse = ops.linear_ce_forward(x, w, y, bias=b)
    grads = ops.linear_ce_backward(x, w, y, lse, bias=b)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for i, (t, name) in enumerate(((x, "dfeatures"), (w, "dweight"), (b, "dbias"))):
        ref = want[name][0]
        d = ref + 0.5 * ref.norm() * torch.randn(ref.shape, generator=gen, device="cuda", dtype=torch.float64) / math.sqrt(ref.numel())
        d = (d / d.norm()).float()
        dd = d.double()
        move = float((dd @ w.double().t() if i == 0 else x.double() @ dd.t() if i == 1 else dd[None]).abs().max())
        h = 2.0 ** math.floor(math.log2(1 / 32 / move))
        f, step = [], []
        for s in (h, -h):
            a = [x, w, b]
            a[i] = t + s * d
            f.append(float(ops.linear_ce_forward(a[0], a[1], y, bias=a[2])[1].double().sum()) / count)
            step.append((a[i].double() - t.double()))
        real = step[0] - step[1]                      # (the step that the rounded operands take)
        slope = f[0] - f[1]
        mine = float((grads[i].double() * real).sum())
        tol = 2 * h * (h * h * (2 * move) ** 3 / 3) + 2 * float(want["loss"][1])
        say(f"{name}: difference {slope:.3e}, gradient {mine:.3e}, tolerance {tol:.1e}")
        assert abs(mine) > 4 * tol
        assert abs(slope - mine) <= tol


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,v", [(64, 48, 300), (700, 64, 9000), (64, 512, 1000)])
def test_infinities_stay_in_their_row(n, c, v, dtype):
    """An infinity or NaN in the features of a row that counts: no value in that row, every other row's loss and gradient as without it."""
    import torch
    x, w, b, y = _inputs(n, c, v, dtype, seed=2)
    want = _reference(x, w, b, y)
    bad = x.clone()
    bad[5, 3], bad[6, 3], bad[7, 3] = float("nan"), float("inf"), float("-inf")
    got = _run(bad, w, b, y)
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[5:8] = False
    assert bool(got["lse"][~rest].isnan().all()) and bool(got["row_loss"][~rest].isnan().all()) and bool(got["dfeatures"][~rest].isnan().any(1).all())
    _compare({k: got[k][rest] for k in ("lse", "row_loss", "dfeatures")}, {k: (want[k][0][rest], want[k][1][rest]) for k in ("lse", "row_loss", "dfeatures")}, "beside infinities")


@pytest.mark.parametrize("dtype,n,c,v", [("bf16", 950, 8, 94619), ("f32", 6, 8, 1059975)])
def test_pieces_one_gradient_at_a_time_and_replayed(dtype, n, c, v):
    """Each gradient alone gives the bits that it has beside the others, and so does a captured pass, replayed with eager ones between."""
    import torch
    from paper_2112_05387_amd import binding as B
    from paper_2112_05387_amd import ops
    d = B.lp_linear_ce_desc(n, c, v, B.LP_BF16 if dtype == "bf16" else B.LP_F32, 0, 0, 0)
    assert B.lp_debug_linear_ce_plan(d, True)[2] > 1
    x, w, b, y = _inputs(n, c, v, dtype, ignored=0.1, seed=3)
    x = (x.float() + 16 * w.float()[y.clamp(min=0).long()] * (torch.arange(n, device="cuda") % 2 == 0)[:, None]).to(x.dtype)      # half of the rows all but certain
    lse = ops.linear_ce_forward(x, w, y, bias=b)[2]
    both = ops.linear_ce_backward(x, w, y, lse, bias=b)
    size = B.lp_linear_ce_workspace_bytes(d, True)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for k, t in enumerate(both):
        out = torch.full_like(t, 7.0)
        ws.fill_(255)
        B.lp_linear_ce_backward(d, torch.cuda.current_stream().cuda_stream, x.data_ptr(), w.data_ptr(), b.data_ptr(), y.data_ptr(), lse.data_ptr(), 1.0,
                                *[out.data_ptr() if k == i else None for i in range(3)], ws.data_ptr(), size)
        assert torch.equal(out, t), k
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.linear_ce_backward(x, w, y, lse, bias=b)
    for turn in range(3):
        x.copy_(_inputs(n, c, v, dtype, ignored=0.1, seed=3 + turn)[0])
        lse.copy_(ops.linear_ce_forward(x, w, y, bias=b)[2])
        graph.replay()
        eager = ops.linear_ce_backward(x, w, y, lse, bias=b)
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(out, eager)), turn


@pytest.mark.parametrize("dtype,n,c,v", [("bf16", 700, 64, 9000), ("f32", 300, 40, 9000), ("bf16", 64, 512, 1000)])
def test_whatever_the_workspace_holds(dtype, n, c, v):
    """Nothing is read from the workspace that the call has not written: the same bits over zeros and over NaN."""
    import torch
    from paper_2112_05387_amd import binding as B
    x, w, b, y = _inputs(n, c, v, dtype, ignored=0.2, seed=5)
    d = B.lp_linear_ce_desc(n, c, v, B.LP_BF16 if dtype == "bf16" else B.LP_F32, 0, 0, 0)
    results = []
    for fill in (0, 255):
        loss, rows, lse = (torch.empty(k, device="cuda") for k in (1, n, n))
        dx, dw, db = torch.empty_like(x), torch.empty(v, c, device="cuda"), torch.empty(v, device="cuda")
        s = torch.cuda.current_stream().cuda_stream
        for backward in (False, True):
            ws = torch.full((B.lp_linear_ce_workspace_bytes(d, backward),), fill, dtype=torch.uint8, device="cuda")
            if backward:
                B.lp_linear_ce_backward(d, s, x.data_ptr(), w.data_ptr(), b.data_ptr(), y.data_ptr(), lse.data_ptr(), 1.0, dx.data_ptr(), dw.data_ptr(), db.data_ptr(), ws.data_ptr(), ws.numel())
            else:
                B.lp_linear_ce_forward(d, s, x.data_ptr(), w.data_ptr(), b.data_ptr(), y.data_ptr(), loss.data_ptr(), rows.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel())
            torch.cuda.synchronize()
        results.append((loss, rows, lse, dx, dw, db))
    for a, e in zip(*results):
        assert torch.equal(a, e) and bool(a.isfinite().all())
