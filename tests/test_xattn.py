"""Cross attention to an encoder's states (mw_xattn_fwd, mw_xattn_bwd): refusals on
the CPU, results on the GPU against the 64-bit definition.

Tolerances, from the number formats: bf16 rounds by at most 2^-8 of a value, 1.7e-3
in the mean square.  P and dS are rounded before their products and outputs once
more, so O is off by sqrt(2) 1.7e-3 = 2.4e-3 in relative L2 and the gradients,
behind a second such pair (D comes from the rounded O), by some 3.4e-3; 5e-3 and
1e-2 allow for short sums, where rounding errors do not average.  An element of
O, a mean of values with weights off by 2^-8 at most, is off by 2^-8 of itself and of
the values' spread.  LSE: the weights' rounding shifts it by 2^-8 at most, where
there are few of them, and by far less than 1e-3 max(1, |LSE|) over many."""
import math

import pytest
import torch

import oracle

OK, INVALID, UNSUPPORTED = 0, 1, 2


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def bf(seed, *shape, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * gain).to(torch.bfloat16)


# ------------------------------------------------------------------ refusals

def test_refusals_before_the_device(mw):
    q, k = bf(0, 2, 4, 8, 64), bf(1, 2, 2, 5, 64)
    lens = torch.tensor([5, 3], dtype=torch.int32)
    o, lse = torch.zeros_like(q), torch.zeros(2, 4, 8)
    strided = bf(2, 2, 2, 64, 5).transpose(2, 3)
    cases = [
        (lambda: mw.mw_xattn_fwd(q, strided, k), "contiguous"),
        (lambda: mw.mw_xattn_fwd(q, k, bf(3, 2, 2, 6, 64)), "v shape"),
        (lambda: mw.mw_xattn_fwd(q, k[:1].contiguous(), k[:1].contiguous()), "does not match q"),
        (lambda: mw.mw_xattn_fwd(q, bf(4, 2, 3, 5, 64), bf(4, 2, 3, 5, 64)), "not a multiple"),
        (lambda: mw.mw_xattn_fwd(q, k, k, lens.long()), "kv_len must be"),
        (lambda: mw.mw_xattn_fwd(q, k, k, lens[:1]), "kv_len must be"),
        (lambda: mw.mw_xattn_fwd(q, k, k, lens, out=(o[:, :, :4].contiguous(), None)), "o must be"),
        (lambda: mw.mw_xattn_fwd(q, k, k, lens, out=(o, lse.double())), "lse must be"),
        (lambda: mw.mw_xattn_bwd(q, k, k, o, lse[:1], o, lens), "lse must be"),
        (lambda: mw.mw_xattn_bwd(q, k, k, o, lse, o[:, :2].contiguous(), lens), "dout shape"),
        (lambda: mw.mw_xattn_bwd(q, k, k, o, lse, o, lens, out=(o, k, o)), "dv must be"),
        (lambda: mw.mw_xattn_fwd(q, k, k, lens), "CUDA tensors"),
        (lambda: mw.mw_xattn_bwd(q, k, k, o, lse, o, lens), "CUDA tensors"),
    ]
    for call, message in cases:
        with pytest.raises(ValueError, match=message):
            call()
    with pytest.raises(TypeError, match="bfloat16"):
        mw.mw_xattn_fwd(q, k.float(), k, lens)


def test_c_refusals(mw):
    lib = mw.library()
    P, odd = 0x10000, 0x10004

    def fwd(q=P, k=P, v=P, lens=None, o=P, lse=None, B=1, H=4, Hkv=2, M=8, S=5, d=64, scale=0.1):
        return lib.mw_xattn_fwd(q, k, v, lens, o, lse, None, 0, B, H, Hkv, M, S, d, scale, None)

    for bad in (dict(B=0), dict(H=0), dict(Hkv=0), dict(Hkv=3), dict(M=-1), dict(S=-1), dict(S=(1 << 24) + 1),
                dict(M=1 << 24), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
                dict(q=None), dict(k=None), dict(v=odd), dict(o=odd), dict(lse=0x10002), dict(lens=0x10002),
                dict(B=1 << 10, H=1 << 10, Hkv=1 << 10, M=1 << 12)):
        assert fwd(**bad) == INVALID, bad
        assert lib.mw_last_error()
    for d in (32, 60, 65, 136):
        assert fwd(d=d) == UNSUPPORTED

    def bwd(q=P, lse=P, dq=P, dk=P, dv=P, o=P, dout=P, M=8, S=5, scale=0.1):
        return lib.mw_xattn_bwd(q, P, P, None, o, lse, dout, dq, dk, dv, None, 0, 1, 4, 2, M, S, 64, scale, None)

    for bad in (dict(q=None), dict(lse=None), dict(dq=odd), dict(dk=None), dict(dv=odd), dict(o=None),
                dict(dout=None), dict(M=-1), dict(S=-1), dict(scale=0.0)):
        assert bwd(**bad) == INVALID, bad
    assert mw.mw_xattn_workspace_size(1, 4, 3, 8, 5, 64) == 0
    assert mw.mw_xattn_bwd_workspace_size(1, 4, 2, 8, 5, 60) == 0


# ------------------------------------------------------------------ results

def rel(a, b):
    a = a.double().cpu()
    n = float(b.norm())
    return float((a - b).norm()) / n if n > 0 else float(a.norm())


def check_lse(lse, ref):
    lse = lse.double().cpu()
    none = ref == -math.inf
    assert torch.equal(lse == -math.inf, none)
    if not bool(none.all()):
        a, r = lse[~none], ref[~none]
        assert float(((a - r).abs() / (1e-3 * r.abs().clamp(min=1.0)).clamp(min=2.0 ** -8)).max()) <= 1.0


def run(mw, B, H, Hkv, M, S, d, lens, gain=1.0, scale=None, seed=0, padding=math.nan, train=True):
    """One call and its gradients against the definition; what lies in padded places
    is `padding`."""
    q, k, v = bf(seed, B, H, M, d, gain=gain), bf(seed + 1, B, Hkv, S, d, gain=gain), bf(seed + 2, B, Hkv, S, d)
    do = bf(seed + 3, B, H, M, d)
    if lens is not None:
        for b, n in enumerate(lens):
            k[b, :, max(n, 0):] = padding
            v[b, :, max(n, 0):] = -padding
    sc = 1.0 / math.sqrt(d) if scale is None else scale
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    qc, kc, vc, doc = (t.cuda() for t in (q, k, v, do))
    o, lse = mw.mw_xattn_fwd(qc, kc, vc, kv_len, scale)
    o2, none = mw.mw_xattn_fwd(qc, kc, vc, kv_len, scale, need_lse=False)
    torch.cuda.synchronize()
    assert mw.mw_device_status() == OK
    assert none is None and torch.equal(o, o2)
    o_ref, lse_ref = oracle.xattn_fwd(q, k, v, lens, sc)
    assert bool(torch.isfinite(o.float()).all())
    for b in range(B):
        for h in range(H):
            assert rel(o[b, h], o_ref[b, h]) <= 5e-3, (b, h)
    for b in range(B):
        for h in range(H):
            n = S if lens is None else lens[b]
            top = float(v[b, h * Hkv // H, :n].abs().max()) if n else 0.0
            err = (o[b, h].double().cpu() - o_ref[b, h]).abs()
            assert float((err - 2.0 ** -8 * o_ref[b, h].abs()).max()) <= 2.0 ** -8 * 2 * top, (b, h)
    check_lse(lse, lse_ref)
    if not train:
        return
    dq, dk, dv = mw.mw_xattn_bwd(qc, kc, vc, o, lse, doc, kv_len, scale)
    torch.cuda.synchronize()
    assert mw.mw_device_status() == OK
    refs = oracle.xattn_bwd(q, k, v, do, lens, sc)
    for name, got, ref in zip(("dq", "dk", "dv"), (dq, dk, dv), refs):
        assert got.shape == ref.shape and bool(torch.isfinite(got.float()).all()), name
        # a gradient that cancels (one state: dS = 0) has only rounding left, which the
        # products' scale bounds: |dS| <= 2^-8 |dO| |V| and its sums with K or Q
        floor = 1e-2 * gain * math.sqrt(ref.numel()) * sc
        err = float((got.double().cpu() - ref).norm())
        assert err <= 1e-2 * float(ref.norm()) + (floor if float(ref.norm()) < 10 * floor else 0.0), (name, err)
        if lens is not None and name != "dq":
            for b, n in enumerate(lens):
                assert torch.count_nonzero(got[b, :, max(n, 0):]) == 0, name


SIZES = [  # B, H, Hkv, M, S, d, lens
    (1, 1, 1, 1, 1, 64, None),
    (1, 2, 2, 1, 77, 64, None),
    (2, 4, 4, 1, 300, 128, [300, 17]),
    (2, 5, 1, 1, 513, 128, [1, 513]),
    (1, 8, 2, 1, 2000, 72, None),
    (3, 4, 2, 3, 129, 64, [0, 129, 128]),
    (1, 6, 2, 5, 1000, 128, [999]),
    (1, 16, 1, 1, 640, 80, [511]),
    (2, 3, 3, 7, 64, 96, [64, 0]),
    (1, 2, 2, 128, 128, 64, None),
    (1, 2, 2, 129, 127, 64, None),
    (2, 2, 1, 255, 257, 64, [257, 130]),
    (1, 3, 3, 257, 77, 128, None),
    (2, 2, 2, 300, 256, 72, [3, 256]),
    (2, 4, 2, 200, 385, 128, [385, 128]),
    (1, 2, 2, 640, 640, 64, [633]),
    (4, 2, 2, 130, 200, 88, [0, 1, 127, 200]),
    (1, 20, 4, 66, 301, 128, [301]),
    (1, 1, 1, 1100, 33, 64, None),
    (1, 1, 1, 40, 1500, 64, None),
    (1, 1, 1, 40, 1500, 128, [1400]),
    (1, 12, 12, 17, 20, 112, None),
    (2, 12, 12, 640, 200, 64, [200, 60]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hkv,M,S,d,lens", SIZES)
def test_against_the_definition(mw, B, H, Hkv, M, S, d, lens):
    run(mw, B, H, Hkv, M, S, d, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("padding", [math.inf, -math.inf, 3.0e38, 0.0])
@pytest.mark.parametrize("M", [1, 6, 150])
def test_what_padded_places_hold_does_not_matter(mw, padding, M):
    run(mw, 2, 4, 2, M, 150, 64, [150, 70], padding=padding)
    run(mw, 2, 2, 2, M, 150, 128, [0, 129], padding=padding)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 150])
def test_lengths_outside_the_states_are_clamped(mw, M):
    q, k, v = bf(0, 2, 2, M, 64).cuda(), bf(1, 2, 2, 40, 64).cuda(), bf(2, 2, 2, 40, 64).cuda()
    low_high = torch.tensor([-5, 41], dtype=torch.int32, device="cuda")
    inside = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    do = bf(3, 2, 2, M, 64).cuda()
    outs = []
    for lens in (low_high, inside):
        o, lse = mw.mw_xattn_fwd(q, k, v, lens)
        outs.append((o, lse, *mw.mw_xattn_bwd(q, k, v, o, lse, do, lens)))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("gain,scale", [(4.0, None), (1.0, 1.0), (0.05, None)])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_flat_and_peaky_rows(mw, gain, scale, d):
    run(mw, 1, 2, 1, 200, 300, d, None, gain=gain, scale=scale)
    run(mw, 1, 2, 2, 1, 900, d, None, gain=gain, scale=scale, train=False)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M", [1, 140])
def test_maxima_that_rise_and_fall(mw, d, M):
    """Keys that grow or shrink along the states: the running maximum moves with
    every tile, or never after the first."""
    for order in (1, -1):
        q, v, do = bf(1, 1, 1, M, d).abs(), bf(2, 1, 1, 700, d), bf(3, 1, 1, M, d)
        ramp = torch.linspace(0.0, 6.0, 700)[::order].contiguous() if order == 1 else torch.linspace(6.0, 0.0, 700)
        k = (bf(4, 1, 1, 700, d).float().abs() * 0.2 + ramp.view(1, 1, 700, 1) * 0.2).to(torch.bfloat16)
        sc = 1.0 / math.sqrt(d)
        qc, kc, vc, doc = (t.cuda() for t in (q, k, v, do))
        o, lse = mw.mw_xattn_fwd(qc, kc, vc)
        o_ref, lse_ref = oracle.xattn_fwd(q, k, v, None, sc)
        assert rel(o, o_ref) <= 5e-3
        check_lse(lse, lse_ref)
        dq, dk, dv = mw.mw_xattn_bwd(qc, kc, vc, o, lse, doc)
        dq_ref, dk_ref, dv_ref = oracle.xattn_bwd(q, k, v, do, None, sc)
        assert rel(dk, dk_ref) <= 1e-2 and rel(dv, dv_ref) <= 1e-2
        # these keys have a common part several times their spread, which dQ = scale dS K
        # multiplies by the rounding errors of dS: that of D = <dO, O> (O in bf16), which
        # is -dD P_ij over a row's keys, and each element's own
        qf, kf, vf, g = (t[0, 0].double() for t in (q, k, v, do))
        p = torch.exp(sc * (qf @ kf.T) - lse_ref[0, 0][:, None])
        ds = (p * (g @ vf.T - (g * o_ref[0, 0]).sum(1, keepdim=True))).abs()
        dD = 2.0 ** -8 * (g * o_ref[0, 0]).abs().sum(1, keepdim=True)
        bound = sc * (dD * (p @ kf).abs() + 2.0 ** -7 * (ds @ kf.abs())) + 2.0 ** -8 * dq_ref[0, 0].abs()
        assert float(((dq[0, 0].double().cpu() - dq_ref[0, 0]).abs() / bound).max()) <= 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("M,S", [(0, 5), (5, 0), (0, 0), (200, 0)])
def test_no_rows_and_no_states(mw, M, S):
    q, k = bf(0, 2, 4, M, 64).cuda(), bf(1, 2, 2, S, 64).cuda()
    o, lse = mw.mw_xattn_fwd(q, k, k)
    assert o.shape == q.shape and torch.count_nonzero(o) == 0 and bool((lse == -math.inf).all())
    dq, dk, dv = mw.mw_xattn_bwd(q, k, k, o, lse, q)
    for g, t in ((dq, q), (dk, k), (dv, k)):
        assert g.shape == t.shape and torch.count_nonzero(g) == 0
    torch.cuda.synchronize()
    assert mw.mw_device_status() == OK


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("lens", [[200, 0, 130], [0, 0, 40], [129, 0, 0], [1, 0, 300]])
def test_long_runs_of_blocks_without_states(mw, d, lens):
    """A dropped sample between others, with more blocks than the launch has CTAs times
    the blocks announced ahead: the result of every sample alone."""
    B, H, M, S = 3, 6, 256 * 152 + 77, 300
    g = torch.Generator("cuda").manual_seed(1)
    q, do = (torch.randn(B, H, M, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    k, v = (torch.randn(B, H, S, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    torch.cuda.synchronize()
    assert mw.mw_device_status() == OK
    for b, n in enumerate(lens):
        one = [t[b:b + 1] for t in (q, k[:, :, :n].contiguous(), v[:, :, :n].contiguous())]
        ob, lb = mw.mw_xattn_fwd(*one)
        assert torch.equal(o[b:b + 1], ob) and torch.equal(lse[b:b + 1], lb)
        grads = mw.mw_xattn_bwd(*one, ob, lb, do[b:b + 1])
        for got, ref in zip((dq[b:b + 1], dk[b:b + 1], dv[b:b + 1]), grads):
            rows = ref.shape[2]
            assert rel(got[:, :, :rows], ref.double().cpu()) <= 2e-3  # the order of fp32 sums
            assert torch.count_nonzero(got[:, :, rows:]) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M", [1, 9, 150, 700])
@pytest.mark.parametrize("S", [1, 77, 301, 1500])
def test_lse_is_of_the_weights_before_their_rounding(mw, M, S, d):
    """LSE in 32 bits.  S sums d / 16 partial products in fp32, each addition off by 2^-23
    of sum |q_i k_i| <= 0.64 d in the mean: 1e-5 after the scale; exponentials by 2^-22,
    sums of 64 by 4e-6 at most, the logarithm by 2^-22.  2e-5 (and of |LSE|, where that is
    above 1) holds all; sums of weights in bf16 are off by 1e-3 and more where they are few
    and by 1e-4 over hundreds."""
    q, k, v = bf(20, 2, 3, M, d), bf(21, 2, 3, S, d), bf(22, 2, 3, S, d)
    lens = [S, (S + 1) // 2]
    _, ref = oracle.xattn_fwd(q, k, v, lens, 1 / math.sqrt(d))
    _, lse = mw.mw_xattn_fwd(q.cuda(), k.cuda(), v.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    err = (lse.double().cpu() - ref).abs() / ref.abs().clamp(min=1)
    assert float(err.max()) <= 2e-5


def reference(q, k, v, do, scale):
    """(O, LSE, dQ, dK, dV) of one head in 64 bits, on the inputs' device."""
    q, k, v, do = (t.double() for t in (q, k, v, do))
    s = q @ k.T * scale
    lse = torch.logsumexp(s, -1)
    p = (s - lse[:, None]).exp()
    o = p @ v
    ds = p * (do @ v.T - (do * o).sum(-1, keepdim=True))
    return o, lse, scale * ds @ k, scale * ds.T @ q, p.T @ do


def near(got, ref, tol):
    return float((got.double() - ref).norm()) <= tol * float(ref.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("M,S", [(4000, 200), (8000, 300)])
def test_many_rows_and_few_states(mw, M, S):
    """d = 64, enough tiles of rows that the backward takes them through two and three key
    tiles a run at a time: dK and dV in accumulators."""
    B, H, d = 4, 12, 64
    lens = [S, 130, 0, 7]
    q, k, v, do = (bf(30 + i, B, H, n, d).cuda() for i, n in enumerate((M, S, S, M)))
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    padded = [-(-n // 128) * 128 for n in (M, S)]
    assert mw.mw_xattn_bwd_workspace_size(B, H, H, M, S, d) >= B * H * (padded[0] + 2 * padded[1]) * d * 4
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    for b, n in enumerate(lens):
        if n == 0:
            for t in (o, dq, dk, dv):
                assert torch.count_nonzero(t[b]) == 0
            continue
        assert torch.count_nonzero(dk[b, :, n:]) == 0 and torch.count_nonzero(dv[b, :, n:]) == 0
        for h in (0, 5, 11):
            ref = reference(q[b, h], k[b, h, :n], v[b, h, :n], do[b, h], 0.125)
            assert near(o[b, h], ref[0], 5e-3)
            assert float((lse[b, h].double() - ref[1]).abs().max()) <= 1e-3
            for got, r in ((dq[b, h], ref[2]), (dk[b, h, :n], ref[3]), (dv[b, h, :n], ref[4])):
                assert near(got, r, 1e-2), (b, h)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,lens", [(900, [700, 1, 300, 0]), (2500, [0, 640, 0, 129]), (1100, [0, 0, 0, 5]),
                                    (600, [0, 0, 0, 0])])
def test_ragged_lengths_over_many_tiles(mw, d, M, lens):
    """The backward divides key tiles that are there among the SMs, in ranges of rows."""
    B, H, Hkv, S = 4, 4, 2, 700
    q, k, v, do = (bf(50 + i, B, h, n, d).cuda() for i, (h, n) in enumerate(((H, M), (Hkv, S), (Hkv, S), (H, M))))
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    for b, n in enumerate(lens):
        if n == 0:
            for t in (o, dq, dk, dv):
                assert torch.count_nonzero(t[b]) == 0
            continue
        assert torch.count_nonzero(dk[b, :, n:]) == 0 and torch.count_nonzero(dv[b, :, n:]) == 0
        for h in range(Hkv):
            rows = lambda t: t[b, 2 * h:2 * h + 2].reshape(2 * M, d)  # noqa: E731
            ref = reference(rows(q), k[b, h, :n], v[b, h, :n], rows(do), d ** -0.5)
            assert near(rows(o), ref[0], 5e-3)
            assert near(dv[b, h, :n], ref[4], 1e-2)
            if n > 1:  # (one state: dS = 0)
                assert near(rows(dq), ref[2], 1e-2) and near(dk[b, h, :n], ref[3], 1e-2)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("S,lens", [(2, None), (3, [3, 2]), (8, [8, 5]), (300, [4, 300]), (200, [1, 7])])
def test_gradients_of_few_and_peaked_states(mw, d, S, lens):
    """Rows that put nearly all their weight on one of a few states: dS = P (dP - D) is a
    small difference, so D must not carry the rounding of O.  What is left are one rounding
    of dS (where two elements of opposite sign share it) and one of the result, 2.4e-3 in
    relative L2 at most; 4e-3 allows for sums too short to average."""
    B, H, M = 2, 3, 700
    q, k = bf(60, B, H, M, d, gain=2.0), bf(61, B, H, S, d, gain=2.0)
    v, do = bf(62, B, H, S, d), bf(63, B, H, M, d)
    q, k, v, do = (t.cuda() for t in (q, k, v, do))
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    for b in range(B):
        n = S if lens is None else lens[b]
        for h in range(H):
            ref = reference(q[b, h], k[b, h, :n], v[b, h, :n], do[b, h], d ** -0.5)
            tol = 4e-3 if n <= 8 else 1e-2
            assert near(dv[b, h, :n], ref[4], 1e-2)
            if n > 1:
                assert near(dq[b, h], ref[2], tol) and near(dk[b, h, :n], ref[3], tol), (b, h)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 40])
def test_states_past_32_bits(mw, M):
    """K and V of more than 2^31 elements: the last head's."""
    B, H, S, d = 1, 17, (1 << 20) + 5, 128
    k, v = (torch.empty(B, H, S, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 31
    for t in (k, v):
        t.normal_(generator=torch.Generator("cuda").manual_seed(4))
    q = bf(5, B, H, M, d).cuda()
    o, lse = mw.mw_xattn_fwd(q, k, v)
    ref = reference(q[0, -1], k[0, -1], v[0, -1], q[0, -1], d ** -0.5)
    # (a mean of a million states: its own size is 2^-8 of theirs)
    assert near(o[0, -1], ref[0], 1e-2)
    assert float((lse[0, -1].double() - ref[1]).abs().max()) <= 2e-5 * float(ref[1].abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("S", [100, 130])
def test_rows_past_32_bits(mw, S):
    """Q, O and their gradients of more than 2^31 elements."""
    B, H, M, d = 1, 16, (1 << 20) + 77, 128
    q, do = (torch.empty(B, H, M, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert q.numel() > 1 << 31
    for i, t in enumerate((q, do)):
        t.normal_(generator=torch.Generator("cuda").manual_seed(6 + i))
    k, v = bf(8, B, H, S, d).cuda(), bf(9, B, H, S, d).cuda()
    o, lse = mw.mw_xattn_fwd(q, k, v)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do)
    ref = reference(q[0, -1], k[0, -1], v[0, -1], do[0, -1], d ** -0.5)
    for got, r, tol in zip((o, dq, dk, dv), (ref[0],) + ref[2:], (5e-3, 1e-2, 1e-2, 1e-2)):
        assert near(got[0, -1], r, tol)
    assert float((lse[0, -1].double() - ref[1]).abs().max()) <= 1e-3


@pytest.mark.gpu
def test_autograd_and_shared_heads(mw):
    """The gradients of shared heads are the sums over the query heads that share
    them: the same as those of the heads repeated, added up."""
    q, k, v, do = (t.cuda() for t in (bf(1, 2, 6, 150, 64), bf(2, 2, 2, 90, 64), bf(3, 2, 2, 90, 64),
                                      bf(4, 2, 6, 150, 64)))
    lens = torch.tensor([90, 33], dtype=torch.int32, device="cuda")
    x = [t.clone().requires_grad_() for t in (q, k, v)]
    o = mw.CrossAttention.apply(*x, lens)
    o.backward(do)
    y = [q.clone().requires_grad_(), *(t.repeat_interleave(3, 1).requires_grad_() for t in (k, v))]
    o2 = mw.CrossAttention.apply(*y, lens, None)
    o2.backward(do)
    assert rel(o.detach(), o2.detach().double().cpu()) <= 1e-3
    for a, b, share in zip(x, y, (1, 3, 3)):
        g = b.grad.double().view(2, -1, share, *b.shape[2:]).sum(2).cpu()
        assert rel(a.grad, g) <= 1e-2
    # a gradient that is not contiguous
    z = [t.clone().requires_grad_() for t in (q, k, v)]
    mw.CrossAttention.apply(*z, lens).backward(do.transpose(2, 3).contiguous().transpose(2, 3))
    for a, b in zip(x, z):
        assert rel(b.grad, a.grad.double().cpu()) <= 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("M,d", [(1, 64), (300, 64), (300, 128)])
def test_buffers_stay_in_their_bounds(mw, M, d):
    """Outputs inside larger buffers of NaN: nothing outside is written, all inside is."""
    B, H, Hkv, S = 2, 4, 2, 190
    q, k, v, do = (t.cuda() for t in (bf(1, B, H, M, d), bf(2, B, Hkv, S, d), bf(3, B, Hkv, S, d), bf(4, B, H, M, d)))
    lens = torch.tensor([150, 0], dtype=torch.int32, device="cuda")

    def guarded(shape, dtype=torch.bfloat16):
        n = math.prod(shape)
        whole = torch.full((n + 512,), math.nan, dtype=dtype, device="cuda")
        return whole, whole[256:256 + n].view(shape)

    wo, o = guarded(q.shape)
    wl, lse = guarded(q.shape[:3], torch.float32)
    mw.mw_xattn_fwd(q, k, v, lens, out=(o, lse))
    grads = [guarded(t.shape) for t in (q, k, v)]
    mw.mw_xattn_bwd(q, k, v, o, lse, do, lens, out=tuple(g for _, g in grads))
    torch.cuda.synchronize()
    for whole, inner in ((wo, o), (wl, lse), *grads):
        assert bool(torch.isnan(whole[:256].float()).all()) and bool(torch.isnan(whole[-256:].float()).all())
        assert not bool(torch.isnan(inner.float()).any())


@pytest.mark.gpu
def test_workspace_of_the_caller_and_other_streams(mw):
    q, k, v = (t.cuda() for t in (bf(1, 1, 4, 1, 128), bf(2, 1, 2, 3000, 128), bf(3, 1, 2, 3000, 128)))
    o, lse = mw.mw_xattn_fwd(q, k, v)
    need = mw.mw_xattn_workspace_size(1, 4, 2, 1, 3000, 128)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    o2, lse2 = mw.mw_xattn_fwd(q, k, v, workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o3, lse3 = mw.mw_xattn_fwd(q, k, v)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    for a, b in ((o, o2), (lse, lse2), (o, o3), (lse, lse3)):
        assert torch.equal(a, b)
    with pytest.raises(ValueError, match="overlaps"):
        mw.mw_xattn_fwd(q, k, v, out=(q, None))


@pytest.mark.gpu
@pytest.mark.parametrize("M,S,d", [(1, 700, 64), (500, 300, 64), (500, 300, 128)])
def test_graph_replay_and_repeats(mw, M, S, d):
    """The same bits from every call and from a captured graph, whose lengths may
    change between replays (dQ of several key tiles: within its rounding)."""
    q, k, v, do = (t.cuda() for t in (bf(1, 2, 4, M, d), bf(2, 2, 2, S, d), bf(3, 2, 2, S, d), bf(4, 2, 4, M, d)))
    lens = torch.tensor([S, 100], dtype=torch.int32, device="cuda")

    def step():
        o, lse = mw.mw_xattn_fwd(q, k, v, lens)
        return (o, lse, *mw.mw_xattn_bwd(q, k, v, o, lse, do, lens))

    first = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    g.replay()
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(first, out)):
        assert torch.equal(a, b) if i < 2 else rel(a, b.double().cpu()) <= 2e-3
    lens.copy_(torch.tensor([S - 1, 0], dtype=torch.int32))
    g.replay()
    again = step()
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(again, out)):
        assert torch.equal(a, b) if i < 2 else rel(a, b.double().cpu()) <= 2e-3


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 200])
def test_binding_and_native_agree(mw, M, monkeypatch):
    q, k, v, do = (t.cuda() for t in (bf(1, 2, 4, M, 64), bf(2, 2, 2, 90, 64), bf(3, 2, 2, 90, 64), bf(4, 2, 4, M, 64)))
    lens = torch.tensor([90, 33], dtype=torch.int32, device="cuda")

    def step():
        o, lse = mw.mw_xattn_fwd(q, k, v, lens, 0.2)
        return (o, lse, mw.mw_xattn_fwd(q, k, v, need_lse=False)[0], *mw.mw_xattn_bwd(q, k, v, o, lse, do, lens, 0.2))

    assert mw._native is not None
    for args in ((q, k, v, lens, None, True, None), (q, k, v, None, 0.5, False, None)):
        assert mw._native.xattn_fwd(*args) is not None
    o, lse = mw.mw_xattn_fwd(q, k, v, lens)
    assert mw._native.xattn_bwd(q, k, v, o, lse, do, lens, None) is not None
    for args in ((q, k.float(), v, lens, None, True, None), (q, k, v, lens.long(), None, True, None),
                 (q, k[:, :, :50], v, lens, None, True, None), (q, k, v, lens.cpu(), None, True, None)):
        assert mw._native.xattn_fwd(*args) is None
    native = step()
    monkeypatch.setattr(mw, "_native", None)
    checked = step()
    for i, (a, b) in enumerate(zip(native, checked)):
        assert a.dtype == b.dtype and (torch.equal(a, b) if i < 3 else rel(a, b.double().cpu()) <= 2e-3)
