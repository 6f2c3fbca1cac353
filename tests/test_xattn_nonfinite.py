"""NaN and infinities in valid places of a cross attention: the results that depend on
them are NaN, as the definition has them, and never those of a row that sees no state;
everything else is what it is without them."""
import math

import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def bf(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


# rows a head of K and V: one, both sizes of the form for few rows, one block and several; key
# ranges that are joined in another kernel (40 rows of 1500 states), and several key tiles
SIZES = [(1, 300), (4, 130), (8, 700), (20, 1500), (150, 77), (700, 300)]


def check(mw, q, k, v, lens):
    """O and LSE against the definition: NaN in the same places, close in all others
    (bf16 weights and results: 5e-3 of a head's finite part; LSE in fp32)."""
    scale = q.shape[-1] ** -0.5
    o, lse = mw.mw_xattn_fwd(q.cuda(), k.cuda(), v.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert mw.mw_device_status() == 0
    o, lse = o.double().cpu(), lse.double().cpu()
    o_ref, lse_ref = oracle.xattn_fwd(q, k, v, lens, scale)
    assert torch.equal(o.isnan(), o_ref.isnan()) and torch.equal(lse.isnan(), lse_ref.isnan())
    rest = ~o_ref.isnan()
    assert float((o[rest] - o_ref[rest]).norm()) <= 5e-3 * float(o_ref[rest].norm()) + 1e-30
    some = ~lse_ref.isnan()
    none = lse_ref[some] == -INF
    assert torch.equal(lse[some] == -INF, none)
    assert bool(((lse[some] - lse_ref[some])[~none].abs() <= 1e-4 * lse_ref[some][~none].abs().clamp(min=1)).all())
    return o, lse


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,S", SIZES)
def test_a_row_of_q(mw, M, S, d):
    q, k, v = bf(0, 2, 4, M, d), bf(1, 2, 2, S, d), bf(2, 2, 2, S, d)
    q[0, 1, M // 2, 5] = NAN
    q[1, 2, 0, d - 1] = INF  # scores of both infinities
    o, lse = check(mw, q, k, v, [S, S // 2 + 1])
    assert bool(o[0, 1, M // 2].isnan().all()) and bool(lse[1, 2, 0].isnan())
    q[1] = NAN  # of a sample without states, nothing is asked
    o, lse = check(mw, q, k, v, [S, 0])
    assert torch.count_nonzero(o[1]) == 0 and bool((lse[1] == -INF).all())


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,S", SIZES)
@pytest.mark.parametrize("place", ["first", "last", "middle"])
def test_a_valid_key(mw, M, S, d, place):
    """One NaN among a head's keys: no row of the heads that share it has a weight."""
    q, k, v = bf(3, 2, 4, M, d), bf(4, 2, 2, S, d), bf(5, 2, 2, S, d)
    n = S - 1
    k[0, 1, {"first": 0, "last": n - 1, "middle": n // 2}[place], 3] = NAN
    o, lse = check(mw, q, k, v, [n, S])
    assert bool(o[0, 2:].isnan().all()) and bool(lse[0, 2:].isnan().all())
    assert not bool(o[0, :2].isnan().any()) and not bool(o[1].isnan().any())


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,S", SIZES)
def test_a_valid_value(mw, M, S, d):
    """NaN or an infinity in one channel of V: that channel of O, and no weight."""
    q, k, v = bf(6, 2, 4, M, d), bf(7, 2, 2, S, d), bf(8, 2, 2, S, d)
    v[0, 0, S // 3, 9] = NAN
    o, lse = check(mw, q, k, v, [S, S])
    assert bool(o[0, :2, :, 9].isnan().all()) and not bool(lse.isnan().any())


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,S", [(1, 100), (150, 77), (700, 300), (3000, 200)])
def test_scores_of_minus_infinity(mw, M, S, d):
    """A state whose score is -inf has weight 0; a row of nothing else sees no state."""
    q, k, v = bf(9, 1, 2, M, d).abs(), bf(10, 1, 2, S, d), bf(11, 1, 2, S, d)
    k[0, 0, S // 2] = -INF
    k[0, 1] = -INF
    o, lse = mw.mw_xattn_fwd(q.cuda(), k.cuda(), v.cuda())
    keep = [j for j in range(S) if j != S // 2]
    o_ref, lse_ref = oracle.xattn_fwd(q[:, :1], k[:, :1, keep], v[:, :1, keep], None, d ** -0.5)
    assert float((o[:, :1].double().cpu() - o_ref).norm()) <= 5e-3 * float(o_ref.norm())
    assert float((lse[:, :1].double().cpu() - lse_ref).abs().max()) <= 1e-4 * max(1.0, float(lse_ref.abs().max()))
    assert torch.count_nonzero(o[0, 1]) == 0 and bool((lse[0, 1] == -INF).all())


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,S,lens", [(40, 200, [130, 70]), (700, 700, [300, 650]), (9000, 300, [5, 290])])
def test_a_gradient_of_one_row(mw, M, S, lens, d):
    """A gradient with NaN in one row: it reaches that row's dQ and its heads' valid keys, and
    nothing in padded places, other rows or other heads."""
    B, H, Hkv = 2, 4, 2
    q, k, v, do = (t.cuda() for t in (bf(4, B, H, M, d), bf(5, B, Hkv, S, d), bf(6, B, Hkv, S, d), bf(7, B, H, M, d)))
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    good = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    bad = do.clone()
    bad[1, 3, M // 2, 4] = math.nan
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, bad, kv_len)
    torch.cuda.synchronize()
    assert mw.mw_device_status() == 0
    for b, n in enumerate(lens):
        assert torch.count_nonzero(dk[b, :, n:]) == 0 and torch.count_nonzero(dv[b, :, n:]) == 0
    n = lens[1]
    assert bool(dq[1, 3, M // 2].isnan().all())
    assert bool(dk[1, 1, :n].isnan().all()) and bool(dv[1, 1, :n, 4].isnan().all())
    dq[1, 3, M // 2] = good[0][1, 3, M // 2]
    for got, ref in zip((dq, dk, dv), good):
        got, ref = got.double(), ref.double()
        if got.shape[2] == S:  # but for the head that the row shares
            got, ref = (torch.cat([t[0].flatten(), t[1, 0].flatten()]) for t in (got, ref))
        # (sums of several tiles come in any order)
        assert bool(torch.isfinite(got).all()) and float((got - ref).norm()) <= 4e-3 * float(ref.norm())


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("M,S,lens", [(4, 90, [30, 90]), (40, 200, [130, 70]), (700, 700, [300, 650]), (9000, 300, [5, 290])])
@pytest.mark.parametrize("where", ["q", "key"])
def test_gradients_of_inputs_with_a_nan(mw, M, S, lens, d, where):
    """Forward and backward: a NaN in a row of Q reaches that row's dQ and its heads' valid
    keys, one in a key all rows of the heads that share it; padded places, and the heads and
    rows that do not see it, keep their gradients."""
    B, H, Hkv = 2, 4, 2
    q, k, v, do = (t.cuda() for t in (bf(20, B, H, M, d), bf(21, B, Hkv, S, d), bf(22, B, Hkv, S, d), bf(23, B, H, M, d)))
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    good = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    n = lens[1]
    lost = torch.zeros(B, H, M, dtype=torch.bool, device="cuda")
    if where == "q":
        q[1, 3, M // 2, 2] = NAN
        lost[1, 3, M // 2] = True
    else:
        k[1, 1, n - 1, 2] = NAN
        lost[1, 2:] = True
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    assert torch.equal(o.isnan(), lost[..., None].expand_as(o)) and torch.equal(lse.isnan(), lost)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    torch.cuda.synchronize()
    assert mw.mw_device_status() == 0
    for b, m in enumerate(lens):
        assert torch.count_nonzero(dk[b, :, m:]) == 0 and torch.count_nonzero(dv[b, :, m:]) == 0
    assert torch.equal(dq.isnan(), lost[..., None].expand_as(dq))
    assert bool(dk[1, 1, :n].isnan().all()) and bool(dv[1, 1, :n].isnan().all())
    for i, got in enumerate((dq, dk, dv)):
        keep = ~lost if i == 0 else torch.ones(B, Hkv, S, dtype=torch.bool, device="cuda")
        if i > 0:
            keep[1, 1] = False
        got, ref = got[keep].double(), good[i][keep].double()
        # (sums of several tiles come in any order)
        assert bool(torch.isfinite(got).all()) and float((got - ref).norm()) <= 4e-3 * float(ref.norm())
