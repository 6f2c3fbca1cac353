"""Long contractions of mw_scaled_matmul: what the tensor cores cut must not grow with the length.

An instruction adds 32 products to a sum and cuts, not rounds, what falls below the last places
of the larger: less than 2^-22 of the sum then, always towards zero.  Where all terms are
positive and alike, n instructions in a row lose less than n / 2 * 2^-22 of their part on
average (the sum grows from 0 to the part), at no element more than n * 2^-22; parts are added in
fp32, rounded, 2^-24 of the sum for each.  Whole numbers below 2^24 lose nothing at all."""
import pytest
import torch

BF16, F32, E4M3, E8M0 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
PART = 64 * 4  # instructions in a row of an fp32 result: 64 blocks
PART_BF16 = 2048 * 4


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


def positive(seed, rows, K):
    """Any positive codes, a power of two for every row: terms of all magnitudes, sums that need
    every place.  Rows end at codes of their own, so that their sums differ."""
    g = generator(seed)
    top = torch.randint(0x70, 0x7f, (rows, 1), device="cuda", generator=g)
    q = torch.empty(rows, K, dtype=torch.uint8, device="cuda")
    for r in range(0, rows, 256):
        u = torch.rand(min(256, rows - r), K, device="cuda", generator=g)
        q[r:r + 256] = (1 + u * (top[r:r + 256] - 1)).to(torch.uint8)
    s = torch.randint(120, 134, (rows, 1), dtype=torch.uint8, device="cuda", generator=g)
    return q.view(E4M3), s.expand(rows, -(-K // 128)).contiguous().view(E8M0)


def whole(seed, rows, K):
    """Whole numbers from -4 to 4 with scales of 1 and 2."""
    g = generator(seed)
    q = torch.randint(-4, 5, (rows, K), device="cuda", generator=g, dtype=torch.int8).float().to(E4M3)
    s = torch.randint(127, 129, (rows, -(-K // 128)), dtype=torch.uint8, device="cuda", generator=g)
    return q, s.view(E8M0)


def reference(a, sa, b, sb):
    """In 64 bits, a piece of the contraction at a time."""
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    step = 1 << 16
    for k in range(0, a.shape[1], step):
        def values(q, s):
            q = q[:, k:k + step].double()
            return q * s[:, k // 128:(k + step) // 128].double().repeat_interleave(128, 1)[:, :q.shape[1]]
        out += values(a, sa) @ values(b, sb).T
    return out


def deviations(mw, M, N, K, dtype, rounding=None, few=256):
    """(result - exact) / exact of up to `few` rows and columns; sizes less the last rounding's."""
    a, sa = positive(1, M, K)
    b, sb = positive(2, N, K)
    c = mw.mw_scaled_matmul(a, sa, b, sb, dtype)
    assert mw.mw_device_status() == 0
    ref = reference(a[-few:], sa[-few:], b[-few:], sb[-few:])
    off = c[-few:, -few:].double() - ref
    return off / ref if rounding is None else (off.abs() - rounding(ref)) / ref


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(16, 2560, 1 << 17), (16, 2560, 1 << 19), (1, 19456, 16384), (20, 4096, 1 << 18),
                                   (64, 7680, 1 << 17), (7680, 33, 1 << 17), (8, 128, 1 << 20), (300, 300, 1 << 16),
                                   (1024, 1024, 1 << 15), (2048, 2048, 1 << 17)])
def test_what_fp32_results_lose_does_not_grow(mw, M, N, K):
    off = deviations(mw, M, N, K, F32)
    parts = K / 128 / 64 + 8
    assert abs(float(off.mean())) <= PART / 2 * 2.0 ** -22 + parts * 2.0 ** -25
    assert float(off.abs().max()) <= PART * 2.0 ** -22 + parts * 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 19456, 16384), (3, 19450, 8208), (3, 20000, 8192 * 5 + 16), (16, 2560, 8192 * 13),
                                   (17, 6000, 8192 * 9 + 128), (33, 15000, 8192 * 3), (64, 2304, 8192 * 16 + 4096),
                                   (19456, 2, 8192 * 2 + 16), (15001, 48, 8192 * 3 + 400), (5, 16, 8192 * 33)])
def test_parts_of_whole_numbers_are_exact(mw, M, N, K):
    """Few rows and more blocks than one part, up to the last part's odd end; rows that start
    anywhere; what lies behind the results stays."""
    a, sa = whole(1, M, K)
    b, sb = whole(2, N, K)
    everything = torch.full((M * N + 64,), 7.0, device="cuda")
    c = mw.mw_scaled_matmul(a, sa, b, sb, F32, out=everything[:M * N].view(M, N))
    assert mw.mw_device_status() == 0
    assert torch.equal(c.double(), reference(a, sa, b, sb))
    assert bool((everything[M * N:] == 7).all())
    assert torch.equal(mw.mw_scaled_matmul(a, sa, b, sb, F32), c)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(16, 640, 1 << 22), (200, 40, 1 << 22), (300, 300, 1 << 22), (1024, 1024, 1 << 21),
                                   (2600, 2304, 1 << 19)])
def test_what_bf16_results_lose_does_not_grow(mw, M, N, K):
    """Less the last rounding, half a step at most.  Of thousands of instructions the sum grows
    evenly, within a twentieth, at every element: a half again, not at the mean alone."""
    off = deviations(mw, M, N, K, BF16, lambda ref: torch.exp2(torch.floor(torch.log2(ref)) - 8))
    assert float(off.max()) <= 1.05 * PART_BF16 / 2 * 2.0 ** -22


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(2, 19456, 1 << 18), (7, 2000, 262144 * 7 + 48), (300, 257, 262144 * 9 + 16),
                                   (1500, 1300, 262144 + 128), (1200, 1100, 262144 * 2 + 112)])
def test_bf16_parts_of_whole_numbers_are_exact(mw, M, N, K):
    a, sa = whole(1, M, K)
    b, sb = whole(2, N, K)
    c = mw.mw_scaled_matmul(a, sa, b, sb)
    assert mw.mw_device_status() == 0
    assert torch.equal(c, reference(a, sa, b, sb).float().to(BF16))


@pytest.mark.gpu
def test_columns_of_a_long_contraction(mw):
    """Both operands across it: the weight's gradient over half a million rows."""
    K = (1 << 19) + 3
    (a, sa), (b, sb) = whole(1, 640, K), whole(2, 512, K)
    ones = torch.full((-(-K // 128), 640), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    for dtype in (BF16, F32):
        c = mw.mw_scaled_matmul(a.T.contiguous(), ones, b.T.contiguous(), ones[:, :512].contiguous(), dtype, True, True)
        want = sum(a[:, k:k + 65536].double() @ b[:, k:k + 65536].double().T for k in range(0, K, 65536))
        assert torch.equal(c, want.float().to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 30, 60])
def test_a_wait_that_runs_out_with_parts_to_come(mw, M):
    a, sa = whole(1, M, 8192 * 5)
    b, sb = whole(2, 15000, 8192 * 5)
    good = mw.mw_scaled_matmul(a, sa, b, sb, F32)
    mw.mw_set_option("wait_budget_ms", 50)
    mw.mw_set_option("debug_skip_q_load", 1)
    try:
        mw.mw_scaled_matmul(a, sa, b, sb, F32)
        assert mw.mw_device_status() == 4
    finally:
        mw.mw_set_option("debug_skip_q_load", 0)
        mw.mw_set_option("wait_budget_ms", 2000)
    assert torch.equal(mw.mw_scaled_matmul(a, sa, b, sb, F32), good) and mw.mw_device_status() == 0


@pytest.mark.gpu
def test_a_wait_that_runs_out_with_bf16_parts_to_come(mw):
    a, sa = whole(1, 300, 1 << 22)
    b, sb = whole(2, 260, 1 << 22)
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
def test_parts_on_streams_at_once(mw):
    """Two CTAs an SM take turns with accumulators; other products beside them."""
    jobs = []
    for i, (M, N, K) in enumerate([(3, 19456, 16384), (64, 15000, 8192 * 3), (30, 8000, 8192 * 7), (300, 1152, 1152)]):
        (a, sa), (b, sb) = whole(10 + i, M, K), whole(20 + i, N, K)
        jobs.append(lambda a=a, sa=sa, b=b, sb=sb: mw.mw_scaled_matmul(a, sa, b, sb, F32))
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for turn in range(8):
        got = []
        for i, job in enumerate(jobs):
            with torch.cuda.stream(streams[(i + turn) % 3]):
                got.append(job())
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert mw.mw_device_status() == 0
