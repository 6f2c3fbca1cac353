"""Gradients that autograd delivers as views which start at any element (the backward of a
concatenation cuts them out of one array): the same as of a gradient of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    assert pkg._native is not None
    return pkg


@pytest.fixture(params=["native", "python"])
def way(request, mw, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(mw, "_native", None)
    return request.param


def rnd(seed, *shape, dtype=BF16):
    return torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).to(dtype)


def check(call, inputs, elements=1):
    """The result's gradient starts `elements` behind a boundary."""
    leaves = [t.clone().requires_grad_(True) for t in inputs]
    y = call(*leaves)
    seen = []
    y.register_hook(lambda g: seen.append((g.data_ptr() % 16, g.is_contiguous())))
    dy = rnd(9, *y.shape, dtype=y.dtype)
    want = torch.autograd.grad(y, leaves, dy, retain_graph=True)
    front = torch.zeros(elements, dtype=y.dtype, device="cuda", requires_grad=True)
    whole = torch.cat([front, y.flatten()])
    got = torch.autograd.grad(whole, leaves, torch.cat([front.detach(), dy.flatten()]))
    assert seen[0][0] == 0 and seen[1] == (elements * y.element_size() % 16, True)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("needs", [(True, True), (True, False), (False, True)])
def test_linear(mw, way, dtype, needs):
    x, w = rnd(1, 5, 7, 64, dtype=dtype), rnd(2, 48, 64, dtype=torch.float32)
    if needs == (True, True):
        check(mw.Fp8Linear.apply, (x, w))
    elif needs[0]:
        check(lambda t: mw.Fp8Linear.apply(t, w), (x,), 3)
    else:
        check(lambda t: mw.Fp8Linear.apply(x, t), (w,), 7 if dtype == BF16 else 2)


def test_norms(mw, way):
    """(Read element by element then, with sums in another order: fp32's rounding, 2^-24 for
    each of the 96 terms at most, and the result's.)"""
    for call in (lambda x, w: mw.LayerNorm.apply(x, w), lambda x, w: mw.RMSNorm.apply(x, w)):
        x, w = (t.requires_grad_(True) for t in (rnd(1, 30, 96), rnd(2, 96, dtype=torch.float32)))
        y = call(x, w)
        dy = rnd(3, 30, 96)
        want = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
        whole = torch.cat([torch.zeros(1, dtype=BF16, device="cuda", requires_grad=True), y.flatten()])
        got = torch.autograd.grad(whole, (x, w), torch.cat([torch.zeros(1, dtype=BF16, device="cuda"), dy.flatten()]))
        for a, b, last in zip(got, want, (2.0 ** -7, 0.0)):
            size = b.double().abs().max()
            assert bool(((a.double() - b.double()).abs() <= last * b.double().abs() + 96 * 2.0 ** -24 * size).all())
