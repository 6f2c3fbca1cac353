"""RMS norm (mw_rmsnorm_fwd, mw_rmsnorm_quantize, mw_rmsnorm_bwd, RMSNorm): refusals on the CPU,
results on the GPU against the 64-bit definition.

Tolerances, from the number formats: a result rounded to bf16 is off by at most 2^-8 of
itself.  Before that, fp32: a row's sum of C <= 8192 squares is added in a tree (at most 80
terms a thread, then at most 5 + 16 steps), all of one sign, so that it is off by at most 100
times 2^-24 of itself, rstd by half of that and a few ulp (2^-18 in all); y and dx are products
of a handful of such factors: 2^-17 of the terms is allowed.  A gradient of the weight is a sum
of n rows in some order: n 2^-24 of the sum of its terms' sizes at most, on top of the terms'
own 2^-17.  An output in 8 bits is off by at most 2^-4 of itself, or half a step of the
smallest codes (2^-10 of its scale), from the y that it stands for."""
import math

import pytest
import torch

from oracle import fp8

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
    x, w, s = rnd(0, 6, 16), rnd(1, 16), torch.zeros(6)
    cases = [
        (lambda: mw.mw_rmsnorm_fwd(rnd(0, 16, 6).T, w), "contiguous"),
        (lambda: mw.mw_rmsnorm_fwd(x, rnd(1, 15)), "weight must be"),
        (lambda: mw.mw_rmsnorm_fwd(x, rnd(1, 4, 16)), "not a multiple of the 4 groups"),
        (lambda: mw.mw_rmsnorm_fwd(x, w, rnd(2, 6, 15)), "residual must be"),
        (lambda: mw.mw_rmsnorm_fwd(x, w, x.to(BF16)), "residual must be"),
        (lambda: mw.mw_rmsnorm_fwd(x, w, out=torch.zeros(6, 15)), "out must be"),
        (lambda: mw.mw_rmsnorm_quantize(rnd(0, 6, 24), None), "multiples of 16"),
        (lambda: mw.mw_rmsnorm_bwd(rnd(2, 6, 15), x, s, w), "dy must be"),
        (lambda: mw.mw_rmsnorm_bwd(x, x, s[:5], w), "rstd must be"),
        (lambda: mw.mw_rmsnorm_bwd(x, x, s, w, x.to(BF16)), "dh must be"),
        (lambda: mw.mw_rmsnorm_fwd(x, w), "CUDA tensors"),
        (lambda: mw.mw_rmsnorm_quantize(x, w), "CUDA tensors"),
        (lambda: mw.mw_rmsnorm_bwd(x, x, s, w), "CUDA tensors"),
        (lambda: mw.RMSNorm.apply(x, w, x), "CUDA tensors"),
    ]
    for call, message in cases:
        with pytest.raises(ValueError, match=message):
            call()
    for call in (lambda: mw.mw_rmsnorm_fwd(x.half(), w.half()), lambda: mw.mw_rmsnorm_fwd(x, w.half()),
                 lambda: mw.mw_rmsnorm_fwd(x, w, out_dtype=torch.float16), lambda: mw.mw_rmsnorm_fwd([1.0]),
                 lambda: mw.mw_rmsnorm_quantize(x.half())):
        with pytest.raises(TypeError):
            call()


def test_c_refusals(mw):
    lib = mw.library()
    P = 0x10000

    def fwd(x=P, r=P, w=P, y=P, ys=P, h=P, rstd=None, rows=6, C=16, groups=1, eps=1e-5, xt=1, yt=1, pt=1):
        return lib.mw_rmsnorm_fwd(x, r, w, y, ys, h, rstd, rows, C, groups, eps, xt, yt, pt, None)

    for bad in (dict(x=None), dict(y=None), dict(h=None), dict(x=P + 2), dict(r=P + 2), dict(w=P + 2),
                dict(rstd=P + 2), dict(rows=-1), dict(rows=1 << 31), dict(groups=0), dict(groups=4), dict(eps=-1.0),
                dict(eps=math.nan), dict(xt=2), dict(yt=3), dict(pt=2), dict(yt=2, ys=None), dict(yt=2, x=P + 8),
                dict(yt=2, r=P + 8), dict(yt=2, w=P + 8), dict(yt=2, y=P + 8), dict(yt=2, h=P + 8)):
        assert fwd(**bad) == INVALID, bad
        assert lib.mw_last_error()
    for bad in (dict(C=0), dict(C=8193), dict(xt=0, yt=1), dict(C=24, yt=2)):
        assert fwd(**bad) == UNSUPPORTED, bad

    def bwd(dy=P, h=P, rstd=P, dh=P, dx=P, dw=P, ws=None, n=0, rows=6, groups=1, yt=1):
        return lib.mw_rmsnorm_bwd(dy, h, rstd, P, dh, dx, dw, ws, n, rows, 16, groups, 1, yt, 1, None)

    need = mw.mw_rmsnorm_bwd_workspace_size(6, 16, 1)
    assert need >= 6 * 16 * 4
    assert bwd() == WORKSPACE and bwd(ws=P, n=need - 1) == WORKSPACE and bwd(ws=P + 4, n=need) == INVALID
    for bad in (dict(dy=None), dict(h=None), dict(rstd=None), dict(rstd=P + 1), dict(dh=P + 2), dict(dx=P + 2),
                dict(dw=P + 2), dict(groups=5), dict(yt=2)):
        assert bwd(ws=P, n=need, **bad) == INVALID, bad
    assert mw.mw_rmsnorm_bwd_workspace_size(6, 16, 6) == 0  # a group a row: no partial sums
    assert mw.mw_rmsnorm_bwd_workspace_size(0, 16, 1) == 0


def close(got, ref, terms, bf16, n=1):
    """|got - ref| within the bounds above; terms: the size of what was added up."""
    bound = 2.0 ** -17 * terms + n * 2.0 ** -24 * terms + (2.0 ** -8 * ref.abs() if bf16 else 0.0) + 1e-30
    err = (got.double().cpu() - ref).abs()
    assert bool(torch.isfinite(got.float()).all())
    assert float((err / bound).max()) <= 1.0, float((err / bound).max())


def place(t, shift):
    """On the GPU, `shift` elements off 16 bytes."""
    if t is None:
        return None
    whole = torch.zeros(t.numel() + 32, dtype=t.dtype, device="cuda")
    view = whole[shift:shift + t.numel()].view(t.shape)
    view.copy_(t)
    return view


def run(mw, R, C, groups=1, x_dtype=BF16, y_dtype=BF16, p_dtype=F32, weighted=True, residual=True, eps=1e-5,
        spread=1.0, shift=0, seed=0):
    x = (rnd(seed, R, C) * spread).to(x_dtype)
    r = (rnd(seed + 1, R, C) * spread * 2).to(x_dtype) if residual else None
    dh = rnd(seed + 4, R, C, dtype=x_dtype) if residual else None
    dy = rnd(seed + 2, R, C, dtype=y_dtype)
    ps = (groups, C) if groups > 1 else (C,)
    w = (1.0 + 0.3 * rnd(seed + 3, *ps)).to(p_dtype) if weighted else None
    xc, rc, wc, dyc, dhc = (place(t, shift) for t in (x, r, w, dy, dh))
    y, h, rstd = mw.mw_rmsnorm_fwd(xc, wc, rc, eps, y_dtype)
    y2, h2, none = mw.mw_rmsnorm_fwd(xc, wc, rc, eps, y_dtype, need_stats=False)
    assert none is None and torch.equal(y, y2) and y.dtype == y_dtype and (h is None) == (r is None)
    rows = xc if h is None else h
    dx, dw = mw.mw_rmsnorm_bwd(dyc, place(rows, shift), rstd, wc, dhc)
    again = mw.mw_rmsnorm_bwd(dyc, place(rows, shift), rstd, wc, dhc)
    torch.cuda.synchronize()
    for a, c in zip((dx, dw), again):
        assert (a is None) == (c is None) and (a is None or torch.equal(a, c))  # a fixed order of sums
    y_ref, h_ref, rstd_ref = fp8.rms_fwd(x, r, w, eps)
    if h is not None:
        assert torch.equal(h, h2) and torch.equal(h.double().cpu(), h_ref)
    assert float((rstd.double().cpu() / rstd_ref - 1).abs().max()) <= 2.0 ** -18
    close(y, y_ref, y_ref.abs(), y_dtype == BF16)
    dx_ref, dw_ref = fp8.rms_bwd(dy, h_ref, w, eps, dh, groups)
    xh = (h_ref * rstd_ref[:, None]).abs()
    wr = 1.0 if w is None else w.double().view(groups, -1).repeat_interleave(R // groups, 0).abs()
    g = dy.double().abs() * wr
    terms = rstd_ref[:, None] * (g + xh * (g * xh).mean(1, keepdim=True))
    assert dx.dtype == x_dtype
    close(dx, dx_ref, terms + (0 if dh is None else dh.double().abs()), x_dtype == BF16)
    if w is not None:
        n = R // groups
        assert dw.dtype == p_dtype and dw.shape == ps
        close(dw.view(groups, C), dw_ref, (dy.double().abs() * xh).view(groups, n, C).sum(1), p_dtype == BF16, n)


def run_codes(mw, R, C, groups=1, x_dtype=BF16, p_dtype=F32, weighted=True, residual=True, spread=1.0, seed=0):
    x = (rnd(seed, R, C) * spread).to(x_dtype)
    r = (rnd(seed + 1, R, C) * spread * 2).to(x_dtype) if residual else None
    ps = (groups, C) if groups > 1 else (C,)
    w = (1.0 + 0.3 * rnd(seed + 3, *ps)).to(p_dtype) if weighted else None
    xc, rc, wc = (place(t, 0) for t in (x, r, w))
    q, scale, h, rstd = mw.mw_rmsnorm_quantize(xc, wc, rc)
    y, h2, rstd2 = mw.mw_rmsnorm_fwd(xc, wc, rc, out_dtype=x_dtype)
    torch.cuda.synchronize()
    assert torch.equal(rstd, rstd2) and (h is None) == (r is None) and (h is None or torch.equal(h, h2))
    assert q.shape == x.shape and scale.shape == (R, math.ceil(C / 128))
    if x_dtype == F32:  # y in fp32 is what goes into 8 bits
        want, ws = mw.mw_quantize(y)
        assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))
        assert torch.equal(scale.view(torch.uint8), ws.view(torch.uint8))
    y_ref, _, _ = fp8.rms_fwd(x, r, w, 1e-5)
    got = fp8.values(q.cpu(), scale.cpu(), 1, 128)
    s = scale.cpu().float().double().repeat_interleave(128, 1)[:, :C]
    bound = y_ref.abs() * (2.0 ** -4 + 2.0 ** -16) + s * 2.0 ** -10
    assert bool(((got - y_ref).abs() <= bound).all())
    top = y_ref.abs()
    blocks = fp8.blocks(top, 1, 128).amax((2, 3))
    sizes = scale.cpu().float().double()
    assert bool((blocks <= 448 * sizes * (1 + 2.0 ** -16)).all())
    assert bool((blocks > 224 * sizes * (1 - 2.0 ** -16))[blocks > 0].all())


SIZES = [(1, 1), (1, 8), (3, 64), (7, 33), (5, 255), (9, 256), (300, 768), (11, 1024), (13, 1152), (17, 1155),
         (64, 1536), (5, 2048), (19, 2560), (3, 4097), (2, 6000), (5, 8192), (3, 8191), (1000, 40), (4001, 96),
         (700, 301), (1300, 2049), (1300, 4095)]


@pytest.mark.gpu
@pytest.mark.parametrize("R,C", SIZES)
def test_sizes(mw, R, C):
    run(mw, R, C)
    run(mw, R, C, residual=False)


@pytest.mark.gpu
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("p_dtype", [F32, BF16])
@pytest.mark.parametrize("C", [768, 771, 2560, 8192, 7001])
@pytest.mark.parametrize("residual", [True, False])
def test_types(mw, types, p_dtype, C, residual):
    run(mw, 37, C, 1, *types, p_dtype, residual=residual)


@pytest.mark.gpu
@pytest.mark.parametrize("R,C,groups", [(6, 64, 2), (6, 65, 3), (40, 1152, 4), (320, 96, 160), (500, 72, 500),
                                        (2000, 128, 2), (352, 2560, 32), (1000, 33, 1000)])
@pytest.mark.parametrize("weighted", [True, False])
def test_groups(mw, R, C, groups, weighted):
    run(mw, R, C, groups if weighted else 1, weighted=weighted)


@pytest.mark.gpu
@pytest.mark.parametrize("shift", [1, 4, 8])
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16)])
def test_arrays_that_start_off_16_bytes(mw, shift, types):
    run(mw, 21, 768, 3, *types, shift=shift)


@pytest.mark.gpu
@pytest.mark.parametrize("spread", [1e-6, 1e6, 0.0])
def test_small_large_and_zero_rows(mw, spread):
    run(mw, 30, 1024, x_dtype=F32, y_dtype=F32, spread=spread)
    run_codes(mw, 30, 1024, x_dtype=F32, spread=spread)


@pytest.mark.gpu
@pytest.mark.parametrize("R,C", [(1, 16), (3, 128), (2, 144), (300, 768), (5, 1168), (13, 1152), (64, 1536),
                                 (1400, 2560), (3, 4112), (5, 8192), (1300, 6000), (4001, 112)])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
@pytest.mark.parametrize("residual", [True, False])
def test_output_in_8_bits(mw, R, C, x_dtype, residual):
    run_codes(mw, R, C, x_dtype=x_dtype, residual=residual)


@pytest.mark.gpu
@pytest.mark.parametrize("R,C,groups", [(6, 64, 2), (40, 1152, 4), (500, 80, 500), (352, 2560, 32)])
def test_output_in_8_bits_of_groups(mw, R, C, groups):
    run_codes(mw, R, C, groups)
    run_codes(mw, R, C, groups, p_dtype=BF16)
    run_codes(mw, R, C, weighted=False)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_a_value_that_is_not_finite_stays_in_its_row(mw, value):
    x = rnd(0, 5, 400, dtype=BF16)
    x[2, 130] = value
    y, _, _ = mw.mw_rmsnorm_fwd(x.cuda())
    q, scale, _, _ = mw.mw_rmsnorm_quantize(x.cuda())
    got = fp8.values(q.cpu(), scale.cpu(), 1, 128)
    others = torch.tensor([0, 1, 3, 4])
    clean = x.clone()
    clean[2] = 1.0
    want, _, _ = mw.mw_rmsnorm_fwd(clean.cuda())
    assert torch.equal(y[others], want[others]) and bool(torch.isfinite(got[others]).all())
    # 0 times an infinity, or NaN, where the value is; an infinite row's other values are 0
    assert bool(torch.isnan(y[2, 130])) and bool(torch.isnan(got[2, 128:256]).all())
    rest = got[2, :128]
    assert bool(torch.isnan(rest).all()) if math.isnan(value) else bool((rest == 0).all())


@pytest.mark.gpu
def test_shapes_and_no_rows(mw):
    x = rnd(0, 2, 3, 5, 64, dtype=BF16).cuda()
    w = rnd(1, 6, 64).cuda()
    y, h, rstd = mw.mw_rmsnorm_fwd(x, w, x)
    assert y.shape == h.shape == x.shape and rstd.shape == (2, 3, 5)
    flat, _, _ = mw.mw_rmsnorm_fwd(x.view(30, 64), w, x.view(30, 64))
    assert torch.equal(y.view(30, 64), flat)
    q, scale, _, _ = mw.mw_rmsnorm_quantize(x, w)
    assert q.shape == x.shape and scale.shape == (30, 1)
    one, _, r1 = mw.mw_rmsnorm_fwd(x[0, 0, 0].contiguous())
    assert one.shape == (64,) and r1.shape == ()
    e = torch.zeros(0, 64, dtype=BF16, device="cuda")
    y, h, rstd = mw.mw_rmsnorm_fwd(e, w[0].contiguous(), e)
    dx, dw = mw.mw_rmsnorm_bwd(e, e, rstd, w[0].contiguous(), e)
    assert y.shape == h.shape == dx.shape == (0, 64) and torch.count_nonzero(dw) == 0
    q, scale, _, _ = mw.mw_rmsnorm_quantize(e)
    assert q.shape == (0, 64) and scale.shape == (0, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("x_dtype,y_dtype", [(BF16, None), (F32, BF16), (F32, None)])
def test_autograd_is_the_two_calls(mw, residual, x_dtype, y_dtype):
    x, r, dy, dh = (rnd(s, 4, 10, 272, dtype=x_dtype).cuda() for s in range(4))
    w = rnd(5, 4, 272).cuda()
    dy = dy.to(x_dtype if y_dtype is None else y_dtype)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, r)]
    lx, lw, lr = leaves
    if residual:
        y, h = mw.RMSNorm.apply(lx, lw, lr, 1e-6, y_dtype)
        gx, gw, gr = torch.autograd.grad((y, h), (lx, lw, lr), (dy, dh))
    else:
        y = mw.RMSNorm.apply(lx, lw, None, 1e-6, y_dtype)
        gx, gw = torch.autograd.grad(y, (lx, lw), dy)
    ry, rh, rstd = mw.mw_rmsnorm_fwd(x, w, r if residual else None, 1e-6, y_dtype)
    dx, dw = mw.mw_rmsnorm_bwd(dy, rh if residual else x, rstd, w, dh if residual else None)
    assert torch.equal(y, ry) and torch.equal(gx, dx) and torch.equal(gw, dw)
    if residual:
        assert torch.equal(h, rh) and torch.equal(gr, dx)


@pytest.mark.gpu
def test_autograd_of_one_output(mw):
    """Only y, or only h, is used further on; one tensor is x and the residual."""
    x, r, dy = (rnd(s, 6, 64, dtype=BF16).cuda() for s in range(3))
    w = rnd(5, 64).cuda()
    lx, lr, lw = (t.clone().requires_grad_(True) for t in (x, r, w))
    y, h = mw.RMSNorm.apply(lx, lw, lr)
    gx, gr, gw = torch.autograd.grad(y, (lx, lr, lw), dy, retain_graph=True)
    _, rh, rstd = mw.mw_rmsnorm_fwd(x, w, r)
    dx, dw = mw.mw_rmsnorm_bwd(dy, rh, rstd, w)
    assert torch.equal(gx, dx) and torch.equal(gr, dx) and torch.equal(gw, dw)
    gx, gr, gw = torch.autograd.grad(h, (lx, lr, lw), dy, allow_unused=True)
    assert torch.equal(gx, dy) and torch.equal(gr, dy) and (gw is None or torch.count_nonzero(gw) == 0)
    lx = x.clone().requires_grad_(True)
    y, h = mw.RMSNorm.apply(lx, w, lx)
    (y.float().sum() + h.float().sum()).backward()
    _, rh, rstd = mw.mw_rmsnorm_fwd(x, w, x)
    dx, _ = mw.mw_rmsnorm_bwd(torch.ones_like(x), rh, rstd, w, torch.ones_like(x))
    assert torch.equal(lx.grad, dx + dx)


@pytest.mark.gpu
def test_second_derivatives_are_refused(mw):
    x = rnd(0, 6, 64).cuda().requires_grad_(True)
    y, h = mw.RMSNorm.apply(x, rnd(1, 64).cuda(), x)
    (g,) = torch.autograd.grad(y.square().sum() + h.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="no second derivative"):
        g.sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("C", [2056, 2049])
def test_arrays_past_32_bits(mw, C):
    """More than 2^31 elements, in pieces of 16 bytes and single elements: the last rows, and
    the weight's gradient over all of them.  An element is rounded to bf16 once (2^-8 of
    itself); the sums over a million rows by sqrt(R / blocks) 2^-24 of sqrt(R) terms: far
    below 1e-4."""
    R = (1 << 20) + 3
    x, dy = (torch.empty(R, C, dtype=BF16, device="cuda") for _ in range(2))
    assert x.numel() > 1 << 31
    for i, t in enumerate((x, dy)):
        t.normal_(generator=torch.Generator("cuda").manual_seed(40 + i))
    w = rnd(42, C).cuda()
    y, h, rstd = mw.mw_rmsnorm_fwd(x, w, dy)
    dx, dw = mw.mw_rmsnorm_bwd(dy, h, rstd, w, x)
    ref_w = torch.zeros(C, dtype=torch.float64, device="cuda")
    for a in range(0, R, 1 << 15):
        hs, g = h[a:a + (1 << 15)].double(), dy[a:a + (1 << 15)].double()
        ref_w += (g * hs * torch.rsqrt(hs.square().mean(1, keepdim=True) + 1e-5)).sum(0)
    assert float((dw.double() - ref_w).norm() / ref_w.norm()) < 1e-4
    tail = slice(R - 5, R)
    y_ref, h_ref, _ = fp8.rms_fwd(x[tail].cpu(), dy[tail].cpu(), w.cpu(), 1e-5)
    assert torch.equal(h[tail].double().cpu(), h_ref)
    close(y[tail], y_ref, y_ref.abs(), True)
    dx_ref, _ = fp8.rms_bwd(dy[tail].cpu(), h_ref, w.cpu(), 1e-5, x[tail].cpu())
    close(dx[tail], dx_ref, 4 * dy[tail].double().abs().cpu() * (1 + w.abs().max().double().cpu()) + 20, True)


@pytest.mark.gpu
def test_streams_and_graphs(mw):
    """A call on another stream, and captured and replayed with other inputs."""
    x, r = rnd(0, 64, 768, dtype=BF16).cuda(), rnd(1, 64, 768, dtype=BF16).cuda()
    w = rnd(2, 768).cuda()
    dy = rnd(3, 64, 768, dtype=BF16).cuda()

    def all_of_it():
        y, h, rstd = mw.mw_rmsnorm_fwd(x, w, r)
        q, scale, _, _ = mw.mw_rmsnorm_quantize(x, w, r)
        dx, dw = mw.mw_rmsnorm_bwd(dy, h, rstd, w, dy)
        return y, h, rstd, q.view(torch.uint8), scale.view(torch.uint8), dx, dw

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = all_of_it()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(all_of_it(), other):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = all_of_it()
    x.copy_(rnd(7, 64, 768))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(all_of_it(), captured):
        assert torch.equal(a, b)
