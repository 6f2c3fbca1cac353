"""CrossAttention and LayerNorm in PyTorch's graph: the native nodes and the Python
functions behind them give the same gradients, refusals and bookkeeping."""
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


def attention(mw, leaves, lens=None):
    return mw.CrossAttention.apply(*leaves, lens, 0.2)


def inputs():
    return [bf(1, 2, 4, 90, 64), bf(2, 2, 2, 70, 64), bf(3, 2, 2, 70, 64)]


@pytest.fixture(params=["native", "python"])
def way(request, mw, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(mw, "_native", None)
    return request.param


def test_both_ways_give_the_same(mw, monkeypatch):
    lens = torch.tensor([70, 9], dtype=torch.int32, device="cuda")
    x, w, b = torch.randn(2, 15, 96, device="cuda"), torch.randn(2, 96, device="cuda"), torch.randn(2, 96, device="cuda")
    do, dy = bf(4, 2, 4, 90, 64), bf(5, 2, 15, 96)

    def run():
        a = [t.clone().requires_grad_() for t in inputs()]
        attention(mw, a, lens).backward(do)
        n = [t.clone().requires_grad_() for t in (x, w, b)]
        y = mw.LayerNorm.apply(*n, 1e-6, torch.bfloat16)
        y.backward(dy)
        return [t.grad for t in a + n] + [y.detach()]

    first = run()
    assert type(attention(mw, [t.requires_grad_() for t in inputs()]).grad_fn).__name__ != "CrossAttentionBackward"
    monkeypatch.setattr(mw, "_native", None)
    for p, q in zip(first, run()):
        assert p.dtype == q.dtype and torch.equal(p, q)


def test_only_what_is_asked_for(mw, way):
    q, k, v = inputs()
    o = attention(mw, (q.requires_grad_(), k, v))
    (dq,) = torch.autograd.grad(o, (q,), torch.ones_like(o))
    assert dq.shape == q.shape
    o = attention(mw, (q.detach(), k, v.requires_grad_()))
    o.sum().backward()
    assert v.grad is not None and q.grad is None and k.grad is None
    x = torch.randn(6, 32, device="cuda")
    w = torch.randn(32, device="cuda", requires_grad=True)
    mw.LayerNorm.apply(x, w, None).sum().backward()
    assert w.grad.shape == (32,)


def test_modes(mw, way):
    q, k, v = (t.requires_grad_() for t in inputs())
    with torch.no_grad():
        assert not attention(mw, (q, k, v)).requires_grad
    with torch.inference_mode():
        assert attention(mw, (q, k, v)).is_inference()
    assert not attention(mw, [t.detach() for t in (q, k, v)]).requires_grad
    o = attention(mw, (q, k, v))
    assert o.requires_grad and o.grad_fn is not None and not o.is_leaf


def test_graph_kept_and_freed(mw, way):
    q, k, v = (t.requires_grad_() for t in inputs())
    o = attention(mw, (q, k, v))
    do = torch.ones_like(o)
    first = torch.autograd.grad(o, (q, k, v), do, retain_graph=True)
    again = torch.autograd.grad(o, (q, k, v), do)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    with pytest.raises(RuntimeError, match="second time|freed"):
        torch.autograd.grad(o, (q, k, v), do)


def test_changed_inputs_are_noticed(mw, way):
    q, k, v = inputs()
    k2 = k.clone()
    o = attention(mw, (q.requires_grad_(), k2, v))
    k2.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


def test_saved_tensor_hooks(mw, way):
    packed = []

    def pack(t):
        packed.append(t.shape)
        return t.cpu()

    q, k, v = (t.requires_grad_() for t in inputs())
    plain = torch.autograd.grad(attention(mw, (q, k, v)).sum(), (q, k, v))
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        o = attention(mw, (q, k, v))
    for a, b in zip(plain, torch.autograd.grad(o.sum(), (q, k, v))):
        assert torch.equal(a, b)
    assert len(packed) == 5


def test_a_refusal_in_the_backward_pass(mw, way):
    """A gradient that does not start at 16 bytes: the library's refusal, raised
    through the autograd engine."""
    q, k, v = (t.requires_grad_() for t in inputs())
    o = attention(mw, (q, k, v))
    odd = torch.zeros(o.numel() + 8, dtype=torch.bfloat16, device="cuda")[1:1 + o.numel()].view(o.shape)
    with pytest.raises(mw.MWError, match="dout is not 16-byte aligned"):
        torch.autograd.grad(o, (q, k, v), odd)


def test_refusals_in_the_forward_pass(mw, way):
    q, k, v = inputs()
    with pytest.raises(mw.MWError, match="scale must be > 0"):
        mw.CrossAttention.apply(q, k, v, None, -1.0)
    with pytest.raises(TypeError):
        mw.CrossAttention.apply(q.float(), k, v)
    with pytest.raises(mw.MWError, match="eps must be"):
        mw.LayerNorm.apply(torch.randn(4, 8, device="cuda"), None, None, -1.0)


def test_gradients_on_another_stream(mw, way):
    q, k, v = (t.requires_grad_() for t in inputs())
    ref = torch.autograd.grad(attention(mw, (q, k, v)).sum(), (q, k, v))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o = attention(mw, (q, k, v))
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(ref, torch.autograd.grad(o.sum(), (q, k, v))):
        assert torch.equal(a, b)
