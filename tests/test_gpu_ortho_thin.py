"""Orthogonalisation of long thin matrices, whose Gram matrix is a sum over the longer side."""
import pytest

from tests.gpu_common import say
from tests.test_gpu_ortho import A, B_, C, _polynomial

pytestmark = pytest.mark.gpu


def _in_fp32(u):
    """The same products in fp32."""
    import torch
    tall = u.shape[0] > u.shape[1]
    x = (u / u.norm()).t().contiguous() if tall else u / u.norm()
    for _ in range(5):
        s = x @ x.t()
        x = A * x + (B_ * s + C * (s @ s)) @ x
    return x.t() if tall else x


@pytest.mark.parametrize("m,n", [(64, 5000), (5000, 64), (64, 50000), (10, 10000), (128, 20000), (20000, 128), (10, 100000), (300, 30000)])
def test_as_exact_as_fp32(m, n):
    """Operands are held to 2^-23 where fp32 holds them to 2^-24, so a result may be twice as far off as the same products in fp32 are (matrices of
    noise and a part of low rank, the sum of six): were the Gram matrix one long sum on the matrix cores, which cut every addend
    to the sum's last bit, it would be two to five times as far off as those."""
    import torch
    from paper_2112_05387_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m + n)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    k = min(m, n) // 4
    us = [1e-3 * (r(m, k) @ r(k, n) / k ** 0.5 + 0.5 * r(m, n)) for _ in range(6)]
    here = plain = 0.0
    for u, o in zip(us, ops.orthogonalize(us)):
        want = _polynomial(u)
        here += float((o.double() - want).norm() / want.norm())
        plain += float((_in_fp32(u).double() - want).norm() / want.norm())
    say(f"{m} x {n}: off by {here / 6:.2e}, fp32 by {plain / 6:.2e}")
    assert here <= 2 * plain


def test_thin_beside_large():
    """In a list with matrices that alone take the largest tiles, which have no room for a second sum."""
    import torch
    from paper_2112_05387_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")
    thin = [1e-3 * (r(64, 16) @ r(16, 50000) / 4 + 0.5 * r(64, 50000)) for _ in range(6)]
    here = plain = 0.0
    for u, o in zip(thin, ops.orthogonalize(thin + [r(4090, 4100)])):
        want = _polynomial(u)
        here += float((o.double() - want).norm() / want.norm())
        plain += float((_in_fp32(u).double() - want).norm() / want.norm())
    say(f"beside 4090 x 4100: off by {here / 6:.2e}, fp32 by {plain / 6:.2e}")
    assert here <= 2 * plain
