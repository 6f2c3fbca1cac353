"""Layer norm (mw_layernorm_fwd, mw_layernorm_bwd): refusals on the CPU, results on
the GPU against the 64-bit definition.

Tolerances, from the number formats: a result rounded to bf16 is off by at most
2^-8 of itself.  Before that, fp32: a row's sums of C <= 8192 terms are added in a
tree (at most 16 terms a thread, then at most 5 + 16 steps), so that mean and
variance are off by some 40 ulp (2^-18 of their terms' mean size), and with them
the normalised value; 2^-17 of the terms of y or dx is allowed.  Gradients of weight
and bias are sums of n rows in some order: n 2^-24 of the sum of their terms' sizes
at most, on top of the terms' own 2^-17."""
import math

import pytest
import torch

import oracle

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 5
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def rnd(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def test_refusals_before_the_device(mw):
    x, w = rnd(0, 6, 16), rnd(1, 16)
    m = torch.zeros(6)
    cases = [
        (lambda: mw.mw_layernorm_fwd(rnd(0, 16, 6).T, w, w), "contiguous"),
        (lambda: mw.mw_layernorm_fwd(x, rnd(1, 15), None), "weight must be"),
        (lambda: mw.mw_layernorm_fwd(x, w, rnd(1, 2, 16)), "one shape and type"),
        (lambda: mw.mw_layernorm_fwd(x, w, w.to(BF16)), "one shape and type"),
        (lambda: mw.mw_layernorm_fwd(x, rnd(1, 4, 16)), "not a multiple of the 4 groups"),
        (lambda: mw.mw_layernorm_fwd(x, rnd(1, 0, 16)), "not a multiple of the 0 groups"),
        (lambda: mw.mw_layernorm_fwd(x, w, out=torch.zeros(6, 15)), "out must be"),
        (lambda: mw.mw_layernorm_bwd(rnd(2, 6, 15), x, m, m, w), "dy must be"),
        (lambda: mw.mw_layernorm_bwd(x, x, m[:5], m, w), "mean must be"),
        (lambda: mw.mw_layernorm_bwd(x, x, m, m.double(), w), "rstd must be"),
        (lambda: mw.mw_layernorm_fwd(x, w, w), "CUDA tensors"),
        (lambda: mw.mw_layernorm_bwd(x, x, m, m, w, w), "CUDA tensors"),
    ]
    for call, message in cases:
        with pytest.raises(ValueError, match=message):
            call()
    for call in (lambda: mw.mw_layernorm_fwd(x.half(), w.half()), lambda: mw.mw_layernorm_fwd(x, w.half()),
                 lambda: mw.mw_layernorm_fwd(x, w, out_dtype=torch.float16), lambda: mw.mw_layernorm_fwd([1.0])):
        with pytest.raises(TypeError):
            call()


def test_c_refusals(mw):
    lib = mw.library()
    P = 0x10000

    def fwd(x=P, w=P, b=P, y=P, mean=None, rstd=None, rows=6, C=16, groups=1, eps=1e-5, xt=1, yt=1, pt=1):
        return lib.mw_layernorm_fwd(x, w, b, y, mean, rstd, rows, C, groups, eps, xt, yt, pt, None)

    for bad in (dict(x=None), dict(y=None), dict(x=P + 2), dict(w=P + 2), dict(mean=P + 2), dict(rows=-1),
                dict(rows=1 << 31), dict(groups=0), dict(groups=4), dict(eps=-1.0), dict(eps=math.nan), dict(xt=2),
                dict(yt=-1), dict(pt=7)):
        assert fwd(**bad) == INVALID, bad
        assert lib.mw_last_error()
    for bad in (dict(C=0), dict(C=8193), dict(xt=0, yt=1)):
        assert fwd(**bad) == UNSUPPORTED, bad

    def bwd(dy=P, x=P, mean=P, rstd=P, dx=P, dw=P, ws=None, n=0, rows=6, groups=1):
        return lib.mw_layernorm_bwd(dy, x, mean, rstd, P, dx, dw, P, ws, n, rows, 16, groups, 1, 1, 1, None)

    need = mw.mw_layernorm_bwd_workspace_size(6, 16, 1)
    assert need >= 6 * 2 * 16 * 4
    assert bwd() == WORKSPACE and bwd(ws=P, n=need - 1) == WORKSPACE and bwd(ws=P + 4, n=need) == INVALID
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=P + 1), dict(dx=P + 2), dict(dw=P + 2),
                dict(groups=5)):
        assert bwd(ws=P, n=need, **bad) == INVALID, bad
    assert mw.mw_layernorm_bwd_workspace_size(6, 16, 6) == 0  # a group a row: no partial sums
    assert mw.mw_layernorm_bwd_workspace_size(0, 16, 1) == 0


def close(got, ref, terms, bf16, n=1):
    """|got - ref| within the bounds above; terms: the size of what was added up."""
    bound = 2.0 ** -17 * terms + n * 2.0 ** -24 * terms + (2.0 ** -8 * ref.abs() if bf16 else 0.0) + 1e-30
    err = (got.double().cpu() - ref).abs()
    assert bool(torch.isfinite(got.float()).all())
    assert float((err / bound).max()) <= 1.0, float((err / bound).max())


def run(mw, R, C, groups=1, x_dtype=BF16, y_dtype=BF16, p_dtype=F32, params="wb", eps=1e-5, offset=0.0, spread=1.0,
        shift=0, seed=0):
    """One call and its gradients; shift: elements by which arrays start off 16 bytes."""
    def place(t):
        t = t.contiguous()
        whole = torch.zeros(t.numel() + 32, dtype=t.dtype, device="cuda")
        view = whole[shift:shift + t.numel()].view(t.shape)
        view.copy_(t)
        return view

    x = (rnd(seed, R, C) * spread + offset).to(x_dtype)
    dy = rnd(seed + 1, R, C, dtype=y_dtype)
    ps = (groups, C) if groups > 1 else (C,)
    w = (1.0 + 0.3 * rnd(seed + 2, *ps)).to(p_dtype) if "w" in params else None
    b = (0.3 * rnd(seed + 3, *ps)).to(p_dtype) if "b" in params else None
    xc, dyc = place(x), place(dy)
    wc, bc = (None if t is None else place(t) for t in (w, b))
    y, mean, rstd = mw.mw_layernorm_fwd(xc, wc, bc, eps, y_dtype)
    y2, m2, r2 = mw.mw_layernorm_fwd(xc, wc, bc, eps, y_dtype, need_stats=False)
    assert m2 is None and r2 is None and torch.equal(y, y2) and y.dtype == y_dtype
    dx, dw, db = mw.mw_layernorm_bwd(dyc, xc, mean, rstd, wc, bc)
    again = mw.mw_layernorm_bwd(dyc, xc, mean, rstd, wc, bc)
    torch.cuda.synchronize()
    for a, c in zip((dx, dw, db), again):
        assert (a is None) == (c is None) and (a is None or torch.equal(a, c))  # a fixed order of sums
    y_ref, mean_ref, rstd_ref = oracle.norm_fwd(x, w, b, eps)
    x64 = x.double()
    size = x64.abs().mean(1)
    assert float(((mean.double().cpu() - mean_ref).abs() / (2.0 ** -18 * size + 1e-30)).max()) <= 1.0
    # a mean that is off by e moves the normalised values by e rstd and the variance by e^2
    slack = 1.0 + (x64.abs().amax(1) * rstd_ref)[:, None]
    assert float(((rstd.double().cpu() / rstd_ref - 1.0).abs()).max()) <= float(2.0 ** -16 * slack.max())
    one = torch.ones(1, dtype=torch.float64)
    wr = one if w is None else w.double().view(groups, -1).repeat_interleave(R // groups, 0)
    br = one * 0 if b is None else b.double().view(groups, -1).repeat_interleave(R // groups, 0)
    xh = (x64 - mean_ref[:, None]) * rstd_ref[:, None]
    close(y, y_ref, (xh.abs() + slack) * wr.abs() + br.abs(), y_dtype == BF16)
    dx_ref, dw_ref, db_ref = oracle.norm_bwd(dy, x, w, eps, groups)
    g = (dy.double() * wr).abs()
    terms = rstd_ref[:, None] * slack * (g + g.mean(1, keepdim=True) + xh.abs() * (g * xh.abs()).mean(1, keepdim=True))
    assert dx.dtype == x_dtype
    close(dx, dx_ref, terms, x_dtype == BF16)
    n = R // groups
    for got, ref, parts in ((dw, dw_ref, dy.double().abs() * (xh.abs() + slack)), (db, db_ref, dy.double().abs())):
        if got is not None:
            assert got.dtype == p_dtype and got.shape == ps
            close(got.view(groups, C), ref, parts.view(groups, n, C).sum(1), p_dtype == BF16, n)


@pytest.mark.gpu
@pytest.mark.parametrize("R,C", [(1, 1), (1, 8), (3, 64), (7, 33), (5, 255), (9, 256), (300, 768), (11, 1024),
                                 (13, 1152), (17, 1155), (64, 1536), (5, 2048), (19, 2560), (3, 4097), (2, 6000),
                                 (5, 8192), (3, 8191), (1000, 40), (4001, 96), (700, 301)])
def test_sizes(mw, R, C):
    run(mw, R, C)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [2047, 2049, 2305, 3001, 4095, 4097, 6143, 8191])
@pytest.mark.parametrize("R", [3, 1300])
def test_wide_rows_of_odd_width(mw, R, C):
    run(mw, R, C)
    run(mw, R, C, x_dtype=F32, y_dtype=F32)


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("p_dtype", [F32, BF16])
@pytest.mark.parametrize("C", [768, 771, 2560, 8192, 7001])
def test_types(mw, types, p_dtype, C):
    run(mw, 37, C, 1, *types, p_dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("R,C,groups", [(6, 64, 2), (6, 65, 3), (40, 1152, 4), (320, 96, 160), (500, 72, 500),
                                        (2000, 128, 2), (352, 2560, 32), (1000, 33, 1000)])
@pytest.mark.parametrize("params", ["wb", "w", "b", ""])
def test_groups_and_missing_parameters(mw, R, C, groups, params):
    run(mw, R, C, groups if params else 1, params=params)


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [1, 4, 8])
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16)])
def test_arrays_that_start_off_16_bytes(mw, shift, types):
    run(mw, 21, 768, 3, *types, shift=shift)


@pytest.mark.gpu
@pytest.mark.parametrize("offset,spread", [(100.0, 1.0), (-1000.0, 0.1), (0.0, 1e-6), (0.0, 1e6), (3.0, 0.0)])
def test_rows_far_from_zero_and_constant_rows(mw, offset, spread):
    run(mw, 30, 1024, x_dtype=F32, y_dtype=F32, offset=offset, spread=spread)


@pytest.mark.gpu
def test_shapes_and_no_rows(mw):
    x = rnd(0, 2, 3, 5, 64, dtype=BF16).cuda()
    w = rnd(1, 6, 64).cuda()
    y, mean, rstd = mw.mw_layernorm_fwd(x, w, w)
    assert y.shape == x.shape and mean.shape == rstd.shape == (2, 3, 5)
    flat, _, _ = mw.mw_layernorm_fwd(x.view(30, 64), w, w)
    assert torch.equal(y.view(30, 64), flat)
    one, m1, _ = mw.mw_layernorm_fwd(x[0, 0, 0].contiguous())
    assert one.shape == (64,) and m1.shape == ()
    e = torch.zeros(0, 64, dtype=BF16, device="cuda")
    y, mean, rstd = mw.mw_layernorm_fwd(e, w[0].contiguous(), w[0].contiguous())
    dx, dw, db = mw.mw_layernorm_bwd(e, e, mean, rstd, w[0].contiguous(), w[0].contiguous())
    assert y.shape == dx.shape == (0, 64) and torch.count_nonzero(dw) == 0 and torch.count_nonzero(db) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("C", [2056, 2049])
def test_arrays_past_32_bits(mw, C):
    """More than 2^31 elements, rows in pieces of 16 bytes and single elements: the last rows,
    and the parameters' gradients over all of them.  An element is rounded to bf16 once
    (2^-8 of itself; dx is a difference of terms up to 4 times its size in fp32); the sums
    over a million rows by sqrt(R / blocks) 2^-24 of sqrt(R) terms: far below 1e-4."""
    R = (1 << 20) + 3
    x, dy = (torch.empty(R, C, dtype=BF16, device="cuda") for _ in range(2))
    assert x.numel() > 1 << 31
    for i, t in enumerate((x, dy)):
        t.normal_(generator=torch.Generator("cuda").manual_seed(40 + i))
    w, b = rnd(42, C).cuda(), rnd(43, C).cuda()
    y, mean, rstd = mw.mw_layernorm_fwd(x, w, b)
    dx, dw, db = mw.mw_layernorm_bwd(dy, x, mean, rstd, w, b)
    ref_w, ref_b = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2))
    for i in range(0, R, 1 << 16):
        v, g = x[i:i + (1 << 16)].double(), dy[i:i + (1 << 16)].double()
        var, mu = torch.var_mean(v, -1, correction=0, keepdim=True)
        xh = (v - mu) / (var + 1e-5).sqrt()
        ref_w += (g * xh).sum(0)
        ref_b += g.sum(0)
    gw = g * w.double()
    last = (gw - gw.mean(-1, keepdim=True) - xh * (gw * xh).mean(-1, keepdim=True)) / (var + 1e-5).sqrt()
    want = xh * w.double() + b.double()
    n = xh.shape[0]
    assert float(((y[-n:].double() - want).abs() - 2.0 ** -8 * want.abs()).max()) <= 1e-4
    assert float(((dx[-n:].double() - last).abs() - 2.0 ** -8 * last.abs()).max()) <= 1e-4
    for got, ref in ((dw, ref_w), (db, ref_b)):
        assert float((got.double() - ref).norm()) <= 1e-4 * float(ref.norm())


@pytest.mark.gpu
def test_autograd_by_differences(mw):
    """The gradients in fp32 against central differences of the function itself."""
    x, w, b, dy = (t.cuda() for t in (rnd(0, 4, 24), 1 + 0.2 * rnd(1, 2, 24), rnd(2, 2, 24), rnd(3, 4, 24)))
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    mw.LayerNorm.apply(*leaves, 1e-2).backward(dy)

    def loss(*t):
        return float((mw.mw_layernorm_fwd(*t, 1e-2)[0].double() * dy.double()).sum())

    step = 2.0 ** -6
    for which, leaf in enumerate(leaves):
        for i in range(0, leaf.numel(), 5):
            ends = []
            for sign in (1, -1):
                t = [a.detach().clone() for a in leaves]
                t[which].view(-1)[i] += sign * step
                ends.append(loss(*t))
            got = (ends[0] - ends[1]) / (2 * step)
            # second order of the step (third derivatives of size ~ 10), fp32 rounding over the step
            assert abs(got - float(leaf.grad.view(-1)[i])) <= 10 * step ** 2 + 96 * 2.0 ** -22 / step


@pytest.mark.gpu
def test_autograd_types_and_missing_parameters(mw):
    x = rnd(0, 6, 64, dtype=F32).cuda().requires_grad_()
    y = mw.LayerNorm.apply(x, None, None, 1e-5, BF16)
    assert y.dtype == BF16
    y.float().sum().backward()
    assert x.grad.dtype == F32 and float(x.grad.abs().max()) <= 1e-4  # sum of y does not depend on x
    w = torch.ones(64, device="cuda", dtype=BF16, requires_grad=True)
    z = mw.LayerNorm.apply(x.detach().to(BF16), w)
    z.backward(torch.ones_like(z).view(64, 6).T.contiguous().T.reshape(6, 64))
    assert w.grad.dtype == BF16


@pytest.mark.gpu
def test_out_streams_and_graphs(mw):
    x, w = rnd(0, 50, 768, dtype=BF16).cuda(), rnd(1, 768).cuda()
    y, mean, rstd = mw.mw_layernorm_fwd(x, w, w)
    buf = torch.full((52, 768), math.nan, dtype=BF16, device="cuda")
    mw.mw_layernorm_fwd(x, w, w, out=buf[1:51])
    assert torch.equal(buf[1:51], y) and bool(torch.isnan(buf[0].float()).all() & torch.isnan(buf[51].float()).all())
    with pytest.raises(ValueError, match="overlaps"):
        mw.mw_layernorm_fwd(x, w, w, out=x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, m2, r2 = mw.mw_layernorm_fwd(x, w, w)
        grads = mw.mw_layernorm_bwd(x, x, m2, r2, w, w)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y3, m3, r3 = mw.mw_layernorm_fwd(x, w, w)
        grads3 = mw.mw_layernorm_bwd(x, x, m3, r3, w, w)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip((y, mean, rstd, *grads), (y3, m3, r3, *grads3)):
        assert torch.equal(a, b)
    assert torch.equal(y, y2)


@pytest.mark.gpu
def test_binding_and_native_agree(mw, monkeypatch):
    x, w, dy = rnd(0, 2, 15, 768, dtype=F32).cuda(), rnd(1, 2, 768).cuda(), rnd(2, 2, 15, 768, dtype=BF16).cuda()

    def step():
        y, mean, rstd = mw.mw_layernorm_fwd(x, w, w, 1e-6, BF16)
        return (y, mean, rstd, *mw.mw_layernorm_bwd(dy, x, mean, rstd, w, w), *mw.mw_layernorm_bwd(dy, x, mean, rstd)[:1])

    assert mw._native.norm_fwd(x, w, None, 1e-5, None, False) is not None
    assert mw._native.norm_fwd(x, w, None, 1e-5, torch.float16, False) is None
    assert mw._native.norm_fwd(x.half(), None, None, 1e-5, None, False) is None
    y, mean, rstd = mw.mw_layernorm_fwd(x, w, w)
    assert mw._native.norm_bwd(dy, x, mean, rstd, w, w) is not None
    native = step()
    monkeypatch.setattr(mw, "_native", None)
    for a, b in zip(native, step()):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)
