"""Gradients of the linear layer in 8 bits against differences of the layer itself, along the
gradient, where the slope is as large as it can be: a sign or a factor would not pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def rnd(seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


@pytest.mark.parametrize("M,K,N", [(200, 256, 192), (40, 1152, 640), (515, 144, 1168)])
@pytest.mark.parametrize("which", ["x", "weight"])
def test_slopes(mw, M, K, N, which):
    """sum(dy y) is linear in x and in W but for their rounding to 8 bits: uniform within 2^-4 of
    the power of two below, 2.6% of a value on average and of either sign, in x + p, x - p and dy.
    Steps p are half as large as x, so that each rounding is 5% of a step and less; some 10^4 of
    them, unrelated, add up to less than 5% * 3 / 100 of the slope along the gradient, three
    standard deviations to less than 5e-3."""
    x, w, dy = rnd(1, M, K), rnd(2, N, K), rnd(3, M, N)
    lx, lw = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    dx, dw = torch.autograd.grad(mw.Fp8Linear.apply(lx, lw), (lx, lw), dy)

    def total(x, w):
        return float((mw.Fp8Linear.apply(x, w).double() * dy).sum())

    if which == "x":
        p = dy @ w
        p *= 0.5 * x.norm() / p.norm()
        slope, difference = float((dx.double() * p).sum()), (total(x + p, w) - total(x - p, w)) / 2
    else:
        p = dy.T @ x
        p *= 0.5 * w.norm() / p.norm()
        slope, difference = float((dw.double() * p).sum()), (total(x, w + p) - total(x, w - p)) / 2
    assert slope > 0.9 * float((dx if which == "x" else dw).double().norm() * p.double().norm())
    assert abs(slope - difference) < 5e-3 * abs(difference)
