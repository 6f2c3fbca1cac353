"""RMSNorm and Fp8Linear in PyTorch's graph: the native nodes and the Python functions behind
them give the same gradients, refusals and bookkeeping."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

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


def rnd(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).to(dtype)


def leaves(*ts):
    return [t.clone().requires_grad_(True) for t in ts]


def test_both_ways_give_the_same(mw, monkeypatch):
    x, r, dy, dh = (rnd(s, 2, 15, 96, dtype=BF16) for s in range(4))
    w2, w1, lin = rnd(5, 2, 96), rnd(6, 96, dtype=BF16), rnd(7, 48, 96)
    dz = rnd(8, 2, 15, 48, dtype=BF16)
    out = {}

    def same(name, *ts):
        for i, t in enumerate(ts):
            t = None if t is None else t.detach().view(torch.uint8) if t.element_size() == 1 else t.detach()
            if (name, i) not in out:
                out[name, i] = t
            else:
                a = out[name, i]
                assert (a is None) == (t is None) and (a is None or (a.dtype == t.dtype and torch.equal(a, t))), name

    def run():
        for k, (w, dt) in enumerate(((w2, None), (w1, None), (None, None))):
            same(f"fwd{k}", *mw.mw_rmsnorm_fwd(x, w, r, 1e-6), *mw.mw_rmsnorm_fwd(x, w, None, need_stats=False))
            same(f"fp8{k}", *mw.mw_rmsnorm_quantize(x, w, r), *mw.mw_rmsnorm_quantize(x, w, need_stats=False))
        h, rs = mw.mw_rmsnorm_fwd(x, w2, r)[1:]
        same("bwd", *mw.mw_rmsnorm_bwd(dy, h, rs, w2, dh), *mw.mw_rmsnorm_bwd(dy, h, rs))
        f = x.float()
        same("f32", *mw.mw_rmsnorm_fwd(f, w1, None, out_dtype=BF16), *mw.mw_rmsnorm_fwd(f, w1, f))
        for block in ((1, 128), (128, 1), (128, 128)):
            same(f"form{block}", *mw.mw_quantize(x, block), *mw.mw_quantize(f, block))
        same("both", *mw.mw_quantize_both(x))
        q, s, qc, sc = mw.mw_quantize_both(x.view(30, 96))
        lq, ls = mw.mw_quantize(lin, (128, 128))
        same("product", mw.mw_scaled_matmul(q, s, lq, ls), mw.mw_scaled_matmul(q, s, lq, ls, torch.float32))
        g, gs = mw.mw_quantize(dz.view(30, 48))
        same("across", mw.mw_scaled_matmul(g, gs, lq, ls, b_transposed=True),
             mw.mw_scaled_matmul(qc, sc, qc, sc, torch.float32, True, True))
        a = leaves(x, w2, r)
        y, hh = mw.RMSNorm.apply(*a, 1e-6)
        torch.autograd.backward((y, hh), (dy, dh))
        same("norm", y, hh, *(t.grad for t in a))
        a = leaves(f, w1)
        y = mw.RMSNorm.apply(*a, None, 1e-5, BF16)
        y.backward(dy)
        same("norm32", y, *(t.grad for t in a))
        for k, (t, lw) in enumerate(((x, lin), (x, lin.to(BF16)), (f, lin))):
            a = leaves(t, lw)
            y = mw.Fp8Linear.apply(*a)
            y.backward(dz.to(t.dtype))
            same(f"linear{k}", y, *(t.grad for t in a))
        same("linear out", mw.Fp8Linear.apply(x, lin, torch.float32))

    run()
    y, _ = mw.RMSNorm.apply(*leaves(x, w2, r))
    assert type(y.grad_fn).__name__ != "RMSNormBackward"
    assert type(mw.Fp8Linear.apply(*leaves(x, lin)).grad_fn).__name__ != "Fp8LinearBackward"
    monkeypatch.setattr(mw, "_native", None)
    run()


def test_only_what_is_asked_for(mw, way):
    x, r, w, lin = rnd(1, 6, 32, dtype=BF16), rnd(2, 6, 32, dtype=BF16), rnd(3, 32), rnd(4, 16, 32)
    for i in range(3):
        ts = [x, w, r]
        ts[i] = ts[i].clone().requires_grad_(True)
        y, h = mw.RMSNorm.apply(*ts)
        (g,) = torch.autograd.grad((y, h), ts[i], (torch.ones_like(y), torch.ones_like(h)), allow_unused=True)
        assert g.shape == ts[i].shape
    lx, lw = leaves(x, lin)
    for a, b, t in ((lx, lin, lx), (x, lw, lw)):
        (g,) = torch.autograd.grad(mw.Fp8Linear.apply(a, b).float().sum(), t)
        assert g.shape == t.shape and g.dtype == t.dtype


def test_modes(mw, way):
    x, w, lin = leaves(rnd(1, 6, 32, dtype=BF16), rnd(3, 32), rnd(4, 16, 32))
    calls = (lambda: mw.RMSNorm.apply(x, w), lambda: mw.RMSNorm.apply(x, w, x)[1], lambda: mw.Fp8Linear.apply(x, lin))
    for call in calls:
        with torch.no_grad():
            assert not call().requires_grad
        with torch.inference_mode():
            assert call().is_inference()
        y = call()
        assert y.requires_grad and not y.is_leaf
        y.float().sum().backward(retain_graph=True)
        y.float().sum().backward()
        with pytest.raises(RuntimeError):  # (what it had saved is gone)
            y.float().sum().backward()


def test_gradients_add_up_over_calls(mw, way):
    x, w, lin = leaves(rnd(1, 6, 32), rnd(3, 32), rnd(4, 32, 32))
    for _ in range(2):
        y, h = mw.RMSNorm.apply(x, w, x)
        (mw.Fp8Linear.apply(y, lin) + h).sum().backward()
    twice = [t.grad.clone() for t in (x, w, lin)]
    for t in (x, w, lin):
        t.grad = None
    y, h = mw.RMSNorm.apply(x, w, x)
    (mw.Fp8Linear.apply(y, lin) + h).sum().backward()
    for t, g in zip((x, w, lin), twice):
        assert torch.equal(g, t.grad + t.grad)


def test_inputs_changed_in_between(mw, way):
    """The norm's backward reads x: a change is told.  The linear layer keeps its own."""
    x, w = leaves(rnd(1, 6, 32), rnd(3, 32))
    y = mw.RMSNorm.apply(x, w)
    with torch.no_grad():
        x.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    x, lin = leaves(rnd(1, 6, 32), rnd(4, 16, 32))
    dy = rnd(5, 6, 16)
    want = torch.autograd.grad(mw.Fp8Linear.apply(x, lin), (x, lin), dy)
    y = mw.Fp8Linear.apply(x, lin)
    with torch.no_grad():
        x.add_(1)
        lin.mul_(2)
    for a, b in zip(torch.autograd.grad(y, (x, lin), dy), want):
        assert torch.equal(a, b)


CPU = lambda t: t.cpu()  # noqa: E731
SHORT = lambda t: t[..., :t.shape[-1] // 2].contiguous()  # noqa: E731
STRIDED = lambda t: torch.stack([t, t], -1)[..., 0]  # noqa: E731
OTHER = lambda t: t.view(torch.int8) if t.dtype == torch.uint8 else t.half()  # noqa: E731


@pytest.mark.parametrize("change", [CPU, SHORT, STRIDED, OTHER], ids=["cpu", "shape", "strided", "type"])
@pytest.mark.parametrize("which", ["h", "rstd", "weight", "linear"])
def test_saved_tensors_that_a_hook_changes(mw, which, change):
    x, w, r, lin = rnd(1, 3, 4, 32), rnd(2, 32), rnd(3, 3, 4, 32), rnd(4, 48, 32)
    is_it = {"h": lambda t: t.shape == (3, 4, 32), "rstd": lambda t: t.shape == (3, 4),
             "weight": lambda t: t.shape == (32,), "linear": lambda t: t.dtype == torch.uint8}[which]
    changed = []

    def unpack(t):
        if not is_it(t):
            return t
        changed.append(t.shape)
        return change(t)

    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
        if which == "linear":
            y = mw.Fp8Linear.apply(*leaves(x, lin))
        else:
            y, _ = mw.RMSNorm.apply(*leaves(x, w, r))
    with pytest.raises(RuntimeError, match="is not the plain CUDA tensor"):
        y.float().sum().backward()
    assert changed
    torch.cuda.synchronize()


def test_saved_tensors_kept_elsewhere(mw, way):
    """Hooks that put the saved tensors away on the host and bring the same back."""
    x, w, r, lin = rnd(1, 12, 64, dtype=BF16), rnd(2, 64), rnd(3, 12, 64, dtype=BF16), rnd(4, 48, 64)

    def run():
        a = leaves(x, w, r, lin)
        y, h = mw.RMSNorm.apply(*a[:3])
        return torch.autograd.grad((mw.Fp8Linear.apply(y, a[3]).float().square().sum() + h.float().sum()), a)

    want = run()
    with torch.autograd.graph.save_on_cpu():
        got = run()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_a_gradient_of_another_type_or_layout(mw, way):
    x, w, lin = leaves(rnd(1, 8, 32), rnd(2, 32), rnd(3, 16, 32))
    y = mw.Fp8Linear.apply(x, lin)
    dy = rnd(4, 16, 8).T  # (columns lie together)
    got = torch.autograd.grad(y, (x, lin), dy, retain_graph=True)
    for a, b in zip(got, torch.autograd.grad(y, (x, lin), dy.contiguous())):
        assert torch.equal(a, b)
    y, h = mw.RMSNorm.apply(x, w, x)
    dy, dh = rnd(5, 32, 8).T, torch.ones(1, 1, device="cuda").expand(8, 32)
    got = torch.autograd.grad((y, h), (x, w), (dy, dh), retain_graph=True)
    for a, b in zip(got, torch.autograd.grad((y, h), (x, w), (dy.contiguous(), dh.contiguous()))):
        assert torch.equal(a, b)


def test_a_training_step_captured_and_replayed(mw, way):
    """Forward and backward captured as one graph, replayed with other inputs, with the same
    bits as eager calls; two graphs at once."""
    x, r, dy = (rnd(s, 40, 64, dtype=BF16) for s in range(3))
    w, lin = leaves(rnd(3, 64), rnd(4, 64, 64))

    def step():
        y, h = mw.RMSNorm.apply(x, w, r)
        z = mw.Fp8Linear.apply(y, lin)
        return (z.detach(), h.detach(), *torch.autograd.grad((z, h), (w, lin), (dy, dy)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    x.copy_(rnd(9, 40, 64))
    with torch.no_grad():
        lin.mul_(0.5)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    want = step()
    for out in outs:
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_wrapped_and_fake_tensors_are_left_to_the_checks(mw):
    x, w, lin = rnd(1, 8, 32, dtype=BF16), rnd(2, 32), rnd(3, 16, 32)
    n = mw._native
    q, s = mw.mw_quantize(x)
    with FakeTensorMode(allow_non_fake_inputs=True) as mode:
        f = mode.from_tensor(x)
        for call in (lambda: n.rms_fwd(f, w, None, 1e-5, None, True), lambda: n.rms_quantize(f, w, None, 1e-5, True),
                     lambda: n.rms_apply(f, w, None, 1e-5, None), lambda: n.linear_apply(f, lin, None),
                     lambda: n.quantize(f, (1, 128)), lambda: n.quantize(x, None),
                     lambda: n.scaled_matmul(q, s, q, s, BF16, False, False)):
            assert call() is None
    assert n.rms_fwd(x.cpu(), w, None, 1e-5, None, True) is None and n.rms_fwd(x) is None
    assert n.quantize(x, (1, 64)) is None and n.quantize(x.T, (1, 128)) is None and n.quantize(x, 3) is None
    assert n.scaled_matmul(q, s, q, s[:3], BF16, False, False) is None
    assert n.scaled_matmul(q, s, q, s, torch.float16, False, False) is None
    assert n.scaled_matmul(q, s, q, s, BF16, 0, False) is None
    assert n.linear_apply(x, lin[:, :16], None) is None and n.rms_bwd(x, x, w, None, None) is None


def test_operands_that_do_not_start_at_16_bytes(mw, way):
    """Told, not read: 16-byte accesses and copies need it."""
    whole = torch.zeros(8 * 32 + 1, dtype=BF16, device="cuda")
    x = whole[1:].view(8, 32)
    lin = rnd(3, 16, 32)
    for call in (lambda: mw.mw_quantize(x), lambda: mw.mw_quantize_both(x), lambda: mw.mw_rmsnorm_quantize(x),
                 lambda: mw.Fp8Linear.apply(x, lin)):
        with pytest.raises(mw.MWError, match="16-byte aligned"):
            call()
    q, s = mw.mw_quantize(torch.zeros(8, 32, device="cuda"))
    off = torch.zeros(8 * 32 + 1, dtype=torch.uint8, device="cuda")[1:].view(8, 32).view(torch.float8_e4m3fn)
    with pytest.raises(mw.MWError, match="16-byte aligned"):
        mw.mw_scaled_matmul(off, s, q, s)
    odd = torch.zeros(9, dtype=torch.uint8, device="cuda")[1:].view(8, 1).view(torch.float8_e8m0fnu)
    odd.view(torch.uint8).copy_(s.view(torch.uint8))
    ones = mw.mw_quantize(torch.ones(8, 32, device="cuda"))
    odd.view(torch.uint8).copy_(ones[1].view(torch.uint8))
    assert bool((mw.mw_scaled_matmul(ones[0], odd, *ones) == 32).all())  # scales may start anywhere
