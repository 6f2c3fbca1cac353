"""Matrices in 8 bits with block scales (mw_quantize), their product (mw_scaled_matmul) and the
linear layer of them (Fp8Linear): refusals on the CPU, results on the GPU against the 64-bit
definitions.

The 8-bit form has no tolerance: dividing by a power of two is exact, and one rounding is left,
which is the definition's.  Of the product: a product of two codes is exact in fp32, scales
are powers of two; sums are fp32, 32 products an instruction, which cuts terms no lower than
2^-22 of the largest: K / 32 instructions (and 8 parts at most) leave (K / 32 + 8) 2^-22 of
the sum of the terms' sizes, and a result in bf16 another 2^-8 of itself."""
import math

import pytest
import torch

from oracle import fp8

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 5
BF16, F32, E4M3, E8M0 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCKS = [(1, 128), (128, 1), (128, 128)]


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def rnd(seed, *shape, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * torch.rand(shape[-1], generator=g) * 4).to(dtype)


def codes(*shape):
    return torch.zeros(shape, dtype=E4M3)


def scales(*shape):
    return torch.ones(shape).to(E8M0)


def bits(t):
    return t.view(torch.uint8)


# ------------------------------------------------------------------ refusals

def test_refusals_before_the_device(mw):
    x = rnd(0, 6, 32)
    a, sa, b, sb = codes(6, 32), scales(6, 1), codes(16, 32), scales(1, 1)
    cases = [
        (lambda: mw.mw_quantize(rnd(0, 32, 6).T), "contiguous"),
        (lambda: mw.mw_quantize(rnd(0, 6, 24)), "multiples of 16"),
        (lambda: mw.mw_quantize_both(rnd(0, 6, 24)), "multiples of 16"),
        (lambda: mw.mw_quantize(x, (1, 64)), "block must be"),
        (lambda: mw.mw_quantize(x, out=(codes(6, 16), scales(6, 1))), "q must be"),
        (lambda: mw.mw_quantize(x, out=(codes(6, 32), scales(1, 1))), "scale must be"),
        (lambda: mw.mw_quantize(x), "CUDA tensors"),
        (lambda: mw.mw_quantize_both(x), "CUDA tensors"),
        (lambda: mw.mw_scaled_matmul(a[None], sa, b, sb), "contiguous matrix"),
        (lambda: mw.mw_scaled_matmul(a.T, sa, b, sb), "contiguous matrix"),
        (lambda: mw.mw_scaled_matmul(codes(6, 24), sa, b, sb), "multiples of 16"),
        (lambda: mw.mw_scaled_matmul(a, scales(5, 1), b, sb), "does not fit a"),
        (lambda: mw.mw_scaled_matmul(a, scales(6, 2), b, sb), "does not fit a"),
        (lambda: mw.mw_scaled_matmul(a, sa, b, scales(2, 1)), "does not fit b"),
        (lambda: mw.mw_scaled_matmul(a, sa, codes(16, 48), scales(16, 1)), "contraction"),
        (lambda: mw.mw_scaled_matmul(a, sa, b, sb, a_transposed=True), "does not fit a"),
        (lambda: mw.mw_scaled_matmul(a, sa, b, sb, out=torch.zeros(6, 17, dtype=BF16)), "out must be"),
        (lambda: mw.mw_scaled_matmul(a, sa, b, sb), "CUDA tensors"),
        (lambda: mw.Fp8Linear.apply(x, rnd(1, 16, 48)), "weight"),
        (lambda: mw.Fp8Linear.apply(x, rnd(1, 17, 32)), "multiples of 16"),
        (lambda: mw.Fp8Linear.apply(x, rnd(1, 16, 32)), "CUDA tensors"),
    ]
    for call, message in cases:
        with pytest.raises(ValueError, match=message):
            call()
    for call in (lambda: mw.mw_quantize(x.half()), lambda: mw.mw_quantize([1.0]),
                 lambda: mw.mw_scaled_matmul(x, sa, b, sb), lambda: mw.mw_scaled_matmul(a, torch.ones(6, 1), b, sb),
                 lambda: mw.mw_scaled_matmul(a, sa, b, sb, torch.float16), lambda: mw.Fp8Linear.apply(x, x.half())):
        with pytest.raises(TypeError):
            call()


def test_c_refusals(mw):
    lib = mw.library()
    P = 0x10000

    def form(x=P, q=P, s=P, qc=P, sc=P, rows=6, C=32, form=3, t=1):
        return lib.mw_quantize(x, q, s, qc, sc, rows, C, form, t, None)

    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(qc=None), dict(sc=None), dict(x=P + 8), dict(q=P + 8),
                dict(qc=P + 8), dict(sc=P + 8), dict(rows=-1), dict(rows=1 << 31), dict(C=-16), dict(C=1 << 25),
                dict(form=-1), dict(form=4), dict(t=2), dict(rows=(1 << 31) - 1, C=1 << 24)):
        assert form(**bad) == INVALID, bad
        assert lib.mw_last_error()
    assert form(C=24) == UNSUPPORTED
    assert form(rows=0) == OK and form(C=0) == OK

    def mm(a=P, sa=P, at=0, aT=0, b=P, sb=P, bt=0, bT=0, c=P, M=32, N=32, K=32, t=0):
        return lib.mw_scaled_matmul(a, sa, at, aT, b, sb, bt, bT, c, M, N, K, t, None)

    for bad in (dict(a=None), dict(b=None), dict(sa=None), dict(sb=None), dict(c=None), dict(a=P + 8), dict(b=P + 8),
                dict(c=P + 1), dict(c=P + 2, t=1), dict(M=-1), dict(N=-1), dict(K=-16), dict(M=1 << 25),
                dict(M=1 << 24, N=1 << 24), dict(t=2)):
        assert mm(**bad) == INVALID, bad
        assert lib.mw_last_error()
    for bad in (dict(K=24), dict(K=24, aT=1), dict(K=24, bT=1), dict(M=24, aT=1), dict(N=24, bT=1)):
        assert mm(**bad) == UNSUPPORTED, bad
    assert mm(M=0) == OK and mm(N=0) == OK


# ------------------------------------------------------------------ the 8-bit form

def check_form(mw, x, block):
    q, scale = mw.mw_quantize(x.cuda(), block)
    torch.cuda.synchronize()
    flat = x.reshape(-1, x.shape[-1])
    v, e = fp8.form(flat, *block)
    assert q.shape == x.shape and q.dtype == E4M3 and scale.dtype == E8M0
    assert torch.equal(bits(scale.cpu()).int() - 127, e.int())
    got = fp8.values(q.cpu().reshape(flat.shape), scale.cpu(), *block)
    assert torch.equal(got.isnan(), v.isnan()) and torch.equal(got.nan_to_num(), v.nan_to_num())
    return q, scale


@pytest.mark.gpu
@pytest.mark.parametrize("rows,C", [(1, 16), (1, 128), (3, 48), (127, 144), (128, 128), (129, 256), (300, 1168),
                                    (1000, 768), (5, 8192), (2049, 32), (260, 2560)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_form(mw, rows, C, dtype):
    x = rnd(rows + C, rows, C, dtype=dtype)
    made = {block: check_form(mw, x, block) for block in BLOCKS}
    q, s, qc, sc = mw.mw_quantize_both(x.cuda())
    for got, want in ((q, made[1, 128][0]), (s, made[1, 128][1]), (qc, made[128, 1][0]), (sc, made[128, 1][1])):
        assert torch.equal(bits(got), bits(want))


@pytest.mark.gpu
@pytest.mark.parametrize("block", BLOCKS)
def test_form_of_limits(mw, block):
    x = torch.zeros(400, 272)
    x[0, 0], x[0, 128], x[130, 3], x[3, 140] = 448.0, 448.00003, 3.4e38, 2.0 ** -126
    x[131, 130:133] = torch.tensor([1e-40, -1e-44, 1e-39])
    x[260, 5], x[270, 135], x[280, 260] = math.inf, -math.inf, math.nan
    x[300, :] = torch.linspace(-500, 500, 272)
    check_form(mw, x, block)
    check_form(mw, x.to(BF16), block)


@pytest.mark.gpu
def test_form_of_all_codes_and_ties(mw):
    every = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
    every = torch.unique(every[torch.isfinite(every)])
    v = torch.cat([every, (every[1:] + every[:-1]) / 2])
    x = torch.zeros(1, 512)
    x[0, :v.numel()] = v
    x = x.view(4, 128).clone()
    x[:, 0] = 448.0
    for scale in (1.0, 2.0 ** -30, 2.0 ** 40):
        for block in BLOCKS:
            check_form(mw, x * scale, block)


@pytest.mark.gpu
def test_form_shapes_and_empty(mw):
    x = rnd(0, 2, 3, 5, 64, dtype=BF16)
    for block in BLOCKS:
        check_form(mw, x, block)
        q, s = mw.mw_quantize(torch.zeros(0, 64, device="cuda"), block)
        assert q.shape == (0, 64) and s.numel() == 0
    out = (torch.empty(30, 64, dtype=E4M3, device="cuda"), torch.empty(30, 1, dtype=E8M0, device="cuda"))
    got = mw.mw_quantize(x.view(30, 64).cuda(), out=out)
    assert got[0] is out[0] and torch.equal(bits(out[0]), bits(mw.mw_quantize(x.view(30, 64).cuda())[0]))
    with pytest.raises(ValueError, match="overlaps"):
        y = torch.zeros(2, 64, device="cuda")
        mw.mw_quantize(y, out=(y.view(torch.uint8).view(-1)[:128].view(2, 64).view(E4M3),
                               torch.empty(2, 1, dtype=E8M0, device="cuda")))


@pytest.mark.gpu
def test_form_past_32_bits(mw):
    """More than 2^31 elements: the last blocks."""
    R, C = (1 << 20) + 130, 2064
    x = torch.empty(R, C, dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    assert x.numel() > 1 << 31
    first = R // 128 * 128 - 128
    tail = x[first:].cpu()
    for block in BLOCKS:
        q, s = mw.mw_quantize(x, block)
        v, _ = fp8.form(tail, *block)
        got = fp8.values(q[first:].cpu(), s[first // block[0]:].cpu(), *block)
        assert torch.equal(got, v)


# ------------------------------------------------------------------ the product

def operand(mw, seed, rows, K, transposed, tiles):
    """(codes, scales, values [rows, K]) on the GPU."""
    x = rnd(seed, rows, K) * (0.1 + rnd(seed + 1, rows, 1).abs())
    x = x.T.contiguous() if transposed else x
    block = (128, 128) if tiles else (128, 1) if transposed else (1, 128)
    q, s = mw.mw_quantize(x.cuda(), block)
    v = q.double() * s.double().repeat_interleave(block[0], 0)[:q.shape[0]].repeat_interleave(block[1], 1)[:, :q.shape[1]]
    return q, s, v.T if transposed else v


def check_product(mw, M, N, K, aT=False, bT=False, a_tiles=False, b_tiles=True, dtype=BF16, out=None):
    a, sa, va = operand(mw, 10, M, K, aT, a_tiles)
    b, sb, vb = operand(mw, 20, N, K, bT, b_tiles)
    c = mw.mw_scaled_matmul(a, sa, b, sb, dtype, aT, bT, out=out)
    again = mw.mw_scaled_matmul(a, sa, b, sb, dtype, aT, bT)
    assert mw.mw_device_status() == 0
    assert c.shape == (M, N) and c.dtype == dtype and torch.equal(c, again)
    ref, terms = va @ vb.T, va.abs() @ vb.abs().T
    bound = (K / 32 + 8) * 2.0 ** -22 * terms + (2.0 ** -8 * ref.abs() if dtype == BF16 else 0.0) + 1e-30
    err = (c.double() - ref).abs() / bound
    assert float(err.max()) <= 1.0, float(err.max())


FEW = [(1, 128, 128), (1, 2304, 768), (2, 16, 16), (8, 2560, 2560), (16, 300, 272), (17, 129, 640), (33, 1000, 1168),
       (64, 4096, 1024), (300, 1, 256), (1000, 64, 2064), (20000, 48, 128)]
MANY = [(65, 96, 160), (128, 128, 16), (129, 257, 144), (301, 1152, 1152), (1000, 1000, 1008), (333, 777, 2064),
        (4403, 1152, 384), (2048, 2048, 2048), (260, 10000, 640), (13000, 200, 80)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", FEW + MANY)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_product(mw, M, N, K, dtype):
    check_product(mw, M, N, K, dtype=dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 128, 300 * 16), (9, 130, 272), (70, 90, 400), (1000, 512, 640), (300, 31, 1040)])
@pytest.mark.parametrize("a_tiles", [True, False])
@pytest.mark.parametrize("b_tiles", [True, False])
def test_product_of_all_scales(mw, M, N, K, a_tiles, b_tiles):
    check_product(mw, M, N, K, a_tiles=a_tiles, b_tiles=b_tiles, dtype=F32)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(16, 16, 1), (16, 48, 127), (128, 128, 128), (48, 2304, 77), (128, 256, 300),
                                   (304, 160, 4403), (1152, 1152, 1411), (2304, 768, 14080), (64, 64, 20000)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_product_of_columns(mw, M, N, K, dtype):
    """Both operands across the contraction, whose length is any: the weight's gradient."""
    check_product(mw, M, N, K, True, True, False, False, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,across", [(2560, 2562, 8320, False), (2561, 2560, 16640, False),
                                          (2560, 2560, 8300, True)])
def test_long_sums_in_fp32(mw, M, N, K, across):
    """More blocks than one part of a sum: the parts are added in the output, through copies or
    (rows that do not start at 16 bytes) element by element."""
    check_product(mw, M, N, K, across, across, False, not across, F32)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(5984, 4705, 16), (5984, 4705, 288), (6000, 4704, 128), (20000, 1300, 640),
                                   (12000, 2305, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_tiles_of_few_blocks(mw, M, N, K, dtype):
    """The tile at the edge leaves half of the warps that write results little or nothing to do, and
    the others fall behind them: by single elements, more than a tile's MMAs take."""
    check_product(mw, M, N, K, dtype=dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,aT,bT", [
    (1152, 1152, 14077, True, True), (2304, 768, 14080, True, True), (1104, 1104, 9000, True, True),
    (1536, 1280, 16000, True, True), (1024, 768, 14080, True, True), (512, 2560, 10240, False, False),
    (1100, 1101, 9008, False, False), (516, 2512, 12304, False, True), (1040, 1030, 9008, True, False)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_tiles_and_a_long_contraction(mw, M, N, K, aT, bT, dtype):
    """Two to four pairs of CTAs share the contraction of a tile of 256 x 256; tiles' second
    halves without rows; rows that start anywhere; what lies behind the results stays."""
    whole = torch.full((M * N + 64,), 7.0, dtype=dtype, device="cuda")
    check_product(mw, M, N, K, aT, bT, not aT and N % 2 == 0, not bT, dtype, out=whole[:M * N].view(M, N))
    assert bool((whole[M * N:] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 768, 2304), (31, 1152, 160), (65, 272, 144), (300, 1152, 1152), (4403, 64, 1152)])
@pytest.mark.parametrize("b_tiles", [True, False])
def test_product_with_b_across(mw, M, N, K, b_tiles):
    """The input's gradient; and the other way round."""
    check_product(mw, M, N, K, False, True, False, b_tiles)
    check_product(mw, N, M, K, True, False, b_tiles, False, F32)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [130, 129, 128])
@pytest.mark.parametrize("M", [5, 200])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_outputs_that_start_anywhere(mw, M, N, dtype):
    """A buffer that starts one element off; what lies around it stays."""
    whole = torch.full((M * N + 64,), 7.0, dtype=dtype, device="cuda")
    check_product(mw, M, N, 272, dtype=dtype, out=whole[1:1 + M * N].view(M, N))
    assert bool((whole[:1] == 7).all()) and bool((whole[1 + M * N:] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(3, 40), (200, 300)])
def test_values_that_are_not_finite(mw, M, N):
    """A block that is NaN makes its row of results NaN, and no other."""
    x, w = rnd(0, M, 400), rnd(1, N, 400)
    x[1, 130] = math.inf
    q, s = mw.mw_quantize(x.cuda())
    wq, ws = mw.mw_quantize(w.cuda(), (128, 128))
    c = mw.mw_scaled_matmul(q, s, wq, ws)
    nan = torch.isnan(c)
    assert bool(nan[1].all()) and int(nan.sum()) == N
    # codes alone, scales alone
    q2, s2 = mw.mw_quantize(rnd(0, M, 400).cuda())
    bits(q2)[2, 399] = 0x7f
    nan = torch.isnan(mw.mw_scaled_matmul(q2, s2, wq, ws))
    assert bool(nan[2].all()) and int(nan.sum()) == N
    q2, s2 = mw.mw_quantize(rnd(0, M, 400).cuda())
    bits(s2)[0, 3] = 0xff
    nan = torch.isnan(mw.mw_scaled_matmul(q2, s2, wq, ws))
    assert bool(nan[0].all()) and int(nan.sum()) == N


@pytest.mark.gpu
@pytest.mark.parametrize("e", [-100, -20, 40])
def test_scales_far_from_one(mw, e):
    """The scales' exponents add up where neither alone is near the result's."""
    M, N, K = 130, 140, 272
    x, w = rnd(0, M, K), rnd(1, N, K)
    q, s = mw.mw_quantize((x * 2.0 ** e).cuda())
    wq, ws = mw.mw_quantize((w * 2.0 ** -e).cuda(), (128, 128))
    near = mw.mw_scaled_matmul(*mw.mw_quantize(x.cuda()), *mw.mw_quantize(w.cuda(), (128, 128)), F32)
    assert torch.equal(mw.mw_scaled_matmul(q, s, wq, ws, F32), near)


@pytest.mark.gpu
def test_no_rows_and_no_contraction(mw):
    a, sa, b, sb = (t.cuda() for t in (codes(0, 64), scales(0, 1), codes(32, 64), scales(1, 1)))
    assert mw.mw_scaled_matmul(a, sa, b, sb).shape == (0, 32)
    assert mw.mw_scaled_matmul(b, sb, a, sa).shape == (32, 0)
    a, sa, b, sb = (t.cuda() for t in (codes(0, 64), scales(0, 64), codes(0, 32), scales(0, 32)))
    out = torch.full((64, 32), 3.0, device="cuda")
    mw.mw_scaled_matmul(a, sa, b, sb, F32, True, True, out=out)
    assert torch.count_nonzero(out) == 0


@pytest.mark.gpu
def test_results_past_32_bits(mw):
    """More than 2^31 results: the last rows and columns."""
    M, N, K = 70000, 32768, 32
    a, sa, va = operand(mw, 1, M, K, False, False)
    b, sb, vb = operand(mw, 2, N, K, False, True)
    c = mw.mw_scaled_matmul(a, sa, b, sb)
    assert c.numel() > 1 << 31
    for rows in (slice(0, 3), slice(M - 200, M)):
        ref = va[rows] @ vb.T
        bound = 9 * 2.0 ** -22 * (va[rows].abs() @ vb.abs().T) + 2.0 ** -8 * ref.abs() + 1e-30
        assert float(((c[rows].double() - ref).abs() / bound).max()) <= 1.0


@pytest.mark.gpu
def test_streams_graphs_and_the_same_operand_twice(mw):
    M, N, K = 200, 384, 640
    x, w = rnd(0, M, K).cuda(), rnd(1, N, K).cuda()

    def chain():
        q, s = mw.mw_quantize(x)
        wq, ws = mw.mw_quantize(w, (128, 128))
        return mw.mw_scaled_matmul(q, s, wq, ws), mw.mw_scaled_matmul(q[:5], s[:5], wq, ws), mw.mw_scaled_matmul(q, s, q, s)

    here = chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = chain()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(here, there):
        assert torch.equal(a, b)
    assert torch.equal(here[1], here[0][:5])
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(chain())
        graphs.append(g)
    x.copy_(rnd(5, M, K))
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    want = chain()
    for got in outs:
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 300])
def test_a_wait_that_runs_out_is_told(mw, M):
    a, sa, _ = operand(mw, 1, M, 640, False, False)
    b, sb, _ = operand(mw, 2, 512, 640, False, True)
    good = mw.mw_scaled_matmul(a, sa, b, sb)
    mw.mw_set_option("wait_budget_ms", 50)
    mw.mw_set_option("debug_skip_q_load", 1)
    try:
        mw.mw_scaled_matmul(a, sa, b, sb)
        assert mw.mw_device_status() == 4
    finally:
        mw.mw_set_option("debug_skip_q_load", 0)
        mw.mw_set_option("wait_budget_ms", 2000)
    assert torch.equal(mw.mw_scaled_matmul(a, sa, b, sb), good) and mw.mw_device_status() == 0


@pytest.mark.gpu
def test_a_wait_that_runs_out_in_joined_pairs(mw):
    a, sa, _ = operand(mw, 1, 1152, 8192, True, False)
    b, sb, _ = operand(mw, 2, 1152, 8192, True, False)
    good = mw.mw_scaled_matmul(a, sa, b, sb, F32, True, True)
    mw.mw_set_option("wait_budget_ms", 50)
    mw.mw_set_option("debug_skip_q_load", 1)
    try:
        mw.mw_scaled_matmul(a, sa, b, sb, F32, True, True)
        assert mw.mw_device_status() == 4
    finally:
        mw.mw_set_option("debug_skip_q_load", 0)
        mw.mw_set_option("wait_budget_ms", 2000)
    assert torch.equal(mw.mw_scaled_matmul(a, sa, b, sb, F32, True, True), good) and mw.mw_device_status() == 0


@pytest.mark.gpu
def test_products_on_streams_at_once(mw):
    """Every kind of product, and the 8-bit form, side by side on the device: as one after another."""
    jobs = []
    for i, (M, N, K, T) in enumerate([(1152, 1152, 9008, True), (3, 2304, 768, False), (64, 512, 4096, False),
                                      (4403, 768, 640, False), (700, 640, 2304, False)]):
        a, sa, _ = operand(mw, 10 + i, M, K, T, False)
        b, sb, _ = operand(mw, 30 + i, N, K, T, False)
        jobs.append(lambda a=a, sa=sa, b=b, sb=sb, T=T: mw.mw_scaled_matmul(a, sa, b, sb, F32, T, T))
    x = rnd(50, 4403, 2304, dtype=BF16).cuda()
    jobs.append(lambda: bits(mw.mw_quantize(x, (128, 128))[0]))
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for turn in range(12):
        got = []
        for i, job in enumerate(jobs):
            with torch.cuda.stream(streams[(i * 5 + turn) % 3]):
                got.append(job())
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert mw.mw_device_status() == 0


# ------------------------------------------------------------------ the linear layer

def linear_reference(x, w, dy):
    """(y, dx, dw) in 64 bits from the forms of x, w and dy, and the sizes of their terms."""
    xr, xc = fp8.form(x, 1, 128)[0], fp8.form(x, 128, 1)[0]
    wt = fp8.form(w, 128, 128)[0]
    gr, gc = fp8.form(dy, 1, 128)[0], fp8.form(dy, 128, 1)[0]
    pairs = ((xr, wt.T), (gr, wt), (gc.T, xc))
    return [(a @ b, a.abs() @ b.abs(), a.shape[1]) for a, b in pairs]


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(1, 16, 16), (5, 272, 160), (64, 128, 512), (77, 768, 304), (301, 1152, 400),
                                   (515, 144, 1168)])
@pytest.mark.parametrize("x_dtype,w_dtype", [(BF16, F32), (BF16, BF16), (F32, F32)])
def test_linear(mw, M, K, N, x_dtype, w_dtype):
    x, w, dy = rnd(1, M, K, dtype=x_dtype), rnd(2, N, K, dtype=w_dtype), rnd(3, M, N, dtype=x_dtype) * 1e-4
    lx, lw = x.cuda().requires_grad_(True), w.cuda().requires_grad_(True)
    y = mw.Fp8Linear.apply(lx, lw)
    dx, dw = torch.autograd.grad(y, (lx, lw), dy.cuda())
    assert mw.mw_device_status() == 0
    assert y.dtype == dx.dtype == x_dtype and dw.dtype == w_dtype
    for got, (ref, terms, n) in zip((y, dx, dw), linear_reference(x, w, dy)):
        bound = (n / 32 + 8) * 2.0 ** -22 * terms + (2.0 ** -8 * ref.abs() if got.dtype == BF16 else 0.0) + 1e-30
        assert got.shape == ref.shape and float(((got.detach().double().cpu() - ref).abs() / bound).max()) <= 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("x_dtype,out_dtype", [(F32, BF16), (BF16, F32)])
def test_linear_output_of_another_type(mw, x_dtype, out_dtype):
    M, K, N = 150, 272, 160
    x, w, dy = rnd(1, M, K, dtype=x_dtype), rnd(2, N, K), rnd(3, M, N, dtype=out_dtype)
    lx, lw = x.cuda().requires_grad_(True), w.cuda().requires_grad_(True)
    y = mw.Fp8Linear.apply(lx, lw, out_dtype)
    dx, dw = torch.autograd.grad(y, (lx, lw), dy.cuda())
    assert y.dtype == out_dtype and dx.dtype == x_dtype and dw.dtype == F32
    for got, (ref, terms, n) in zip((y, dx, dw), linear_reference(x, w, dy)):
        bound = (n / 32 + 8) * 2.0 ** -22 * terms + (2.0 ** -8 * ref.abs() if got.dtype == BF16 else 0.0) + 1e-30
        assert float(((got.detach().double().cpu() - ref).abs() / bound).max()) <= 1.0


@pytest.mark.gpu
def test_linear_gradients_by_differences(mw):
    """y is linear in each input but for the rounding of 8 bits, at most 2^-4 of a value and 3%
    on average: differences of the layer without it, over all inputs at once."""
    M, K, N = 200, 256, 192
    x, w, dy = (rnd(s, *shape).cuda() for s, shape in ((1, (M, K)), (2, (N, K)), (3, (M, N))))
    lx, lw = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    dx, dw = torch.autograd.grad(mw.Fp8Linear.apply(lx, lw), (lx, lw), dy)
    for got, exact in ((dx, dy.double() @ w.double()), (dw, dy.double().T @ x.double())):
        # two factors of 3% each
        assert float((got.double() - exact).norm() / exact.norm()) < 0.05
    px, pw = rnd(4, M, K).cuda().double(), rnd(5, N, K).cuda().double()
    plus = ((x + px) @ (w + pw).T * dy).sum()
    minus = ((x - px) @ (w - pw).T * dy).sum()
    slope = float((dx.double() * px).sum() + (dw.double() * pw).sum())
    size = float((dx.double().norm() * px.norm() + dw.double().norm() * pw.norm()))
    assert abs(slope - float(plus - minus) / 2) < 0.05 * size


@pytest.mark.gpu
def test_linear_shapes_and_partial_gradients(mw):
    x, w, dy = rnd(1, 2, 7, 64, dtype=BF16).cuda(), rnd(2, 48, 64).cuda(), rnd(3, 2, 7, 48, dtype=BF16).cuda()
    lx, lw = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    y = mw.Fp8Linear.apply(lx, lw)
    dx, dw = torch.autograd.grad(y, (lx, lw), dy)
    assert y.shape == (2, 7, 48) and dx.shape == x.shape and dw.shape == w.shape
    flat = mw.Fp8Linear.apply(x.view(14, 64), w)
    assert torch.equal(y.view(14, 48), flat) and not flat.requires_grad
    (only,) = torch.autograd.grad(mw.Fp8Linear.apply(lx, w), lx, dy)
    assert torch.equal(only, dx)
    (only,) = torch.autograd.grad(mw.Fp8Linear.apply(x, lw), lw, dy)
    assert torch.equal(only, dw)
    strided = x.transpose(0, 1).requires_grad_(True)  # neither operand need be contiguous
    y2 = mw.Fp8Linear.apply(strided, lw)
    assert torch.equal(y2, y.transpose(0, 1))
    (g2,) = torch.autograd.grad(y2, strided, dy.transpose(0, 1))
    assert torch.equal(g2, dx.transpose(0, 1))
    assert mw.Fp8Linear.apply(x[0, 0], w).shape == (48,)
    assert mw.Fp8Linear.apply(x, w, torch.float32).dtype == F32
    e = torch.zeros(0, 64, dtype=BF16, device="cuda").requires_grad_(True)
    y = mw.Fp8Linear.apply(e, lw)
    dx, dw = torch.autograd.grad(y, (e, lw), torch.zeros(0, 48, dtype=BF16, device="cuda"))
    assert y.shape == (0, 48) and dx.shape == (0, 64) and torch.count_nonzero(dw) == 0


@pytest.mark.gpu
def test_linear_has_no_second_derivative(mw):
    x, w = rnd(1, 8, 64).cuda().requires_grad_(True), rnd(2, 48, 64).cuda().requires_grad_(True)
    dx, dw = torch.autograd.grad(mw.Fp8Linear.apply(x, w).sum(), (x, w), create_graph=True)
    for g in (dx, dw):
        with pytest.raises(RuntimeError, match="no second derivative"):
            g.sum().backward(retain_graph=True)


# ------------------------------------------------------------------ a run of them together

@pytest.mark.gpu
def test_norm_product_split_attention_product(mw):
    """A sublayer as a streaming or validation program runs it: norm with the residual's
    addition into 8 bits, QKV product, split with RoPE, block-causal attention, its output
    into 8 bits, product; against the same steps with torch's products of what the forms
    stand for.  Each product is rounded to bf16 once on both sides (2^-8), attention in
    between is the same call on inputs that differ by that."""
    B, N, H, d, T = 2, 96, 3, 64, 32
    C = H * d
    x, r = rnd(1, B, N, C, dtype=BF16).cuda(), rnd(2, B, N, C, dtype=BF16).cuda()
    w = (1 + 0.1 * rnd(3, C)).cuda()
    qkv_w, out_w = rnd(4, 3 * C, C).cuda() / 14, rnd(5, C, C).cuda() / 14
    qkv_q, out_q = (mw.mw_quantize(t, (128, 128)) for t in (qkv_w, out_w))

    def values(q, s, rows):
        return fp8.values(q.cpu().reshape(-1, q.shape[-1]), s.cpu(), rows, 128).float().cuda()

    q, s, h, _ = mw.mw_rmsnorm_quantize(x, w, r)
    qkv = mw.mw_scaled_matmul(q.view(B * N, C), s, *qkv_q)
    ref = (values(q, s, 1) @ values(*qkv_q, 128).T)
    assert float((qkv.float() - ref).norm() / ref.norm()) < 2.0 ** -8
    heads = mw.mw_qkv_rope_split(qkv.view(B, N, 3, H, d), 32, 10000.0, 16)
    o, _ = mw.mw_bca_fwd(*heads, T, need_lse=False)
    o = o.transpose(1, 2).reshape(B * N, C)
    oq, os = mw.mw_quantize(o)
    y = mw.mw_scaled_matmul(oq, os, *out_q)
    ref = values(oq, os, 1) @ values(*out_q, 128).T
    assert float((y.float() - ref).norm() / ref.norm()) < 2.0 ** -8
    # The whole against 64-bit products.  A rounding to 8 bits is uniform within half a step,
    # 2^-4 of the power of two below: 2^-4 / sqrt(3) of that, 2.6% of a value from 1 to 2.  Two
    # of them make 3.6% of Q, K and V, Q and K 5.1% of the logits' spread, which is the error
    # of a weight against the others (less where one holds the row); the output's product adds
    # 3.6% to V's.
    y_ref, h_ref, _ = fp8.rms_fwd(x.cpu().view(-1, C), r.cpu().view(-1, C), w.cpu(), 1e-5)
    assert torch.equal(h.cpu().double().view(-1, C), h_ref)
    plain = (y_ref.cuda() @ qkv_w.double().T).to(BF16).view(B, N, 3, H, d)
    pq, pk, pv = mw.mw_qkv_rope_split(plain, 32, 10000.0, 16)
    o, _ = mw.mw_bca_fwd(pq, pk, pv, T, need_lse=False)
    whole = o.transpose(1, 2).reshape(B * N, C).double() @ out_w.double().T
    spread = float((pq.float() @ pk.float().transpose(-1, -2) / math.sqrt(d)).std())
    assert float((y.double() - whole).norm() / whole.norm()) < math.hypot(0.051 * spread, 0.036, 0.036)


@pytest.mark.gpu
def test_norm_and_linear_trained_together(mw):
    """RMSNorm with the residual and Fp8Linear one after another, twice: gradients against
    the same chain in fp32 with torch's norm and products; 8 bits in every product."""
    R, C = 256, 256
    x, r = rnd(1, R, C, dtype=BF16).cuda(), rnd(2, R, C, dtype=BF16).cuda()
    leaves = [(1 + 0.1 * rnd(3, C)).cuda(), (rnd(4, C, C) / 16).cuda(), (1 + 0.1 * rnd(5, C)).cuda(), (rnd(6, C, C) / 16).cuda()]
    dy, dh = rnd(7, R, C, dtype=BF16).cuda(), rnd(8, R, C, dtype=BF16).cuda()

    def ours(x, r, n1, w1, n2, w2):
        y, h = mw.RMSNorm.apply(x, n1, r)
        y, h = mw.RMSNorm.apply(mw.Fp8Linear.apply(y, w1), n2, h)
        return mw.Fp8Linear.apply(y, w2), h

    def plain(x, r, n1, w1, n2, w2):
        def norm(t, w):
            return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-5) * w

        h = x + r
        z = norm(h, n1) @ w1.T
        h = h + z
        return norm(h, n2) @ w2.T, h

    got_in = [t.clone().requires_grad_(True) for t in (x, r, *leaves)]
    ref_in = [t.double().requires_grad_(True) for t in (x, r, *leaves)]
    got = torch.autograd.grad(ours(*got_in), got_in, (dy, dh))
    ref = torch.autograd.grad(plain(*ref_in), ref_in, (dy.double(), dh.double()))
    for g, t in zip(got, ref):
        assert float((g.double() - t).norm() / t.norm()) < 0.1
    assert mw.mw_device_status() == 0
