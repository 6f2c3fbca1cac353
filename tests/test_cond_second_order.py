"""The autograd functions have first derivatives only: a second one is refused, by the
native nodes and by the Python functions, and never silently left out."""
import pytest
import torch

pytestmark = pytest.mark.gpu


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


def bf(seed, *shape):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(torch.bfloat16)


def functions(mw):
    x, w, b = torch.randn(6, 32, device="cuda"), torch.randn(32, device="cuda"), torch.randn(32, device="cuda")
    q, k, v = bf(1, 2, 4, 90, 64), bf(2, 2, 2, 70, 64), bf(3, 2, 2, 70, 64)
    c = [bf(4 + i, 1, 2, 64, 64) for i in range(3)]
    return {"cross": (lambda *t: mw.CrossAttention.apply(*t), (q, k, v)),
            "norm": (lambda *t: mw.LayerNorm.apply(*t), (x, w, b)),
            "causal": (lambda *t: mw.BlockCausalAttention.apply(*t, 32), c)}


@pytest.mark.parametrize("name", ["cross", "norm", "causal"])
@pytest.mark.parametrize("which", [0, 1])
def test_a_penalty_on_a_gradient(mw, way, name, which):
    """The gradient of the output is constant, so that only the inputs tie the first
    derivative to the graph; beside it a term that has a gradient of its own."""
    f, inputs = functions(mw)[name]
    leaves = [t.clone().requires_grad_() for t in inputs]
    y = f(*leaves)
    (g,) = torch.autograd.grad(y.float().sum(), leaves[which], create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        (g.float().pow(2).sum() + y.float().pow(2).sum()).backward()


@pytest.mark.parametrize("name", ["cross", "norm", "causal"])
def test_through_the_gradient_of_the_output(mw, way, name):
    f, inputs = functions(mw)[name]
    leaves = [t.clone().requires_grad_() for t in inputs]
    y = f(*leaves)
    dy = torch.ones_like(y).requires_grad_()
    grads = torch.autograd.grad(y, leaves, dy, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        torch.autograd.grad(grads[0].float().sum(), dy)


@pytest.mark.parametrize("name", ["cross", "norm", "causal"])
def test_first_derivatives_are_the_same(mw, way, name):
    f, inputs = functions(mw)[name]
    leaves = [t.clone().requires_grad_() for t in inputs]
    dy = torch.ones_like(f(*leaves))
    plain = torch.autograd.grad(f(*leaves), leaves, dy)
    for a, b in zip(plain, torch.autograd.grad(f(*leaves), leaves, dy, create_graph=True)):
        assert not a.requires_grad and b.requires_grad and torch.equal(a, b.detach())
    # what no input asks for needs no graph either
    (only,) = torch.autograd.grad(f(leaves[0], *inputs[1:]), leaves[:1], dy)
    assert torch.equal(only, plain[0]) and not only.requires_grad
