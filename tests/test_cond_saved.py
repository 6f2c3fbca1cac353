"""Saved tensors of the autograd functions that a hook puts others in the place of: on the
CPU, of another type, shape or layout.  The native nodes refuse them before anything is
launched, as the Python functions refuse those that do not fit together."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    assert pkg._native is not None
    return pkg


def bf(seed, *shape):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(torch.bfloat16)


def attention(mw):
    """A call whose saved tensors are told apart by shape and type."""
    t = [bf(1, 2, 4, 90, 64), bf(2, 2, 2, 70, 64), bf(3, 2, 2, 70, 64)]
    lens = torch.tensor([70, 9], dtype=torch.int32, device="cuda")
    return lambda *x: mw.CrossAttention.apply(*x, lens), t


def norm(mw, groups=None, x_type=torch.float32):
    shape = (32,) if groups is None else (groups, 32)
    t = [torch.randn(3, 4, 32, device="cuda").to(x_type), torch.randn(*shape, device="cuda"), torch.randn(*shape, device="cuda")]
    return lambda *x: mw.LayerNorm.apply(*x), t


IS = {
    "q": lambda t: t.shape == (2, 4, 90, 64),
    "k": lambda t: t.shape == (2, 2, 70, 64),
    "lse": lambda t: t.shape == (2, 4, 90),
    "kv_len": lambda t: t.dtype == torch.int32,
    "x": lambda t: t.shape == (3, 4, 32),
    "stats": lambda t: t.shape == (3, 4),
    "weight": lambda t: t.shape in ((32,), (2, 32)),
}
CPU = lambda t: t.cpu()  # noqa: E731
DOUBLE = lambda t: t.double() if t.is_floating_point() else t.long()  # noqa: E731
OTHER = lambda t: t.float() if t.dtype == torch.bfloat16 else t.to(torch.bfloat16)  # noqa: E731
SHORT = lambda t: t[..., :t.shape[-1] // 2].contiguous()  # noqa: E731
STRIDED = lambda t: torch.stack([t, t], -1)[..., 0]  # noqa: E731


def refused(f, inputs, which, change, errors):
    leaves = [t.clone().requires_grad_() for t in inputs]
    changed = []

    def unpack(t):
        if not IS[which](t):
            return t
        changed.append(t.shape)
        return change(t)

    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        y = f(*leaves)
    with pytest.raises(errors):
        y.float().sum().backward()
    assert changed
    torch.cuda.synchronize()


@pytest.mark.parametrize("which", ["q", "k", "lse", "kv_len"])
@pytest.mark.parametrize("change", [CPU, DOUBLE, SHORT, STRIDED], ids=["cpu", "type", "shape", "strided"])
def test_attention(mw, which, change):
    refused(*attention(mw), which, change, RuntimeError)


@pytest.mark.parametrize("groups", [None, 2])
@pytest.mark.parametrize("which", ["x", "stats", "weight"])
@pytest.mark.parametrize("change", [CPU, OTHER, SHORT, STRIDED], ids=["cpu", "type", "shape", "strided"])
def test_norm(mw, which, change, groups):
    refused(*norm(mw, groups), which, change, RuntimeError)


@pytest.mark.parametrize("change", [CPU, DOUBLE, SHORT, STRIDED], ids=["cpu", "type", "shape", "strided"])
def test_python_functions(mw, change, monkeypatch):
    monkeypatch.setattr(mw, "_native", None)
    for which in ("q", "k", "lse", "kv_len"):
        refused(*attention(mw), which, change, (ValueError, TypeError))
    for which in ("x", "stats", "weight"):
        refused(*norm(mw, 2), which, change, (ValueError, TypeError))


@pytest.mark.parametrize("name", ["attention", "norm"])
def test_the_same_values_elsewhere_are_taken(mw, name):
    """A round trip over the host, lengths and weights too."""
    f, inputs = attention(mw) if name == "attention" else norm(mw, 2)
    leaves = [t.clone().requires_grad_() for t in inputs]
    plain = torch.autograd.grad(f(*leaves).float().sum(), leaves)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.cuda()):
        y = f(*leaves)
    for a, b in zip(plain, torch.autograd.grad(y.float().sum(), leaves)):
        assert torch.equal(a, b)
