"""NaN in Q or in a key of the block-causal forward and of its form against a ring: the
rows that see it are NaN in O and LSE, the others are what they are without it."""
import math

import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def bf(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def check(o, lse, o_ref, lse_ref, lost):
    """lost [B, H, rows]: the rows that are NaN; the tolerances of test_gpu_parity.py for the rest."""
    torch.cuda.synchronize()
    o, lse = o.double().cpu(), lse.double().cpu()
    assert bool(o[lost].isnan().all()) and bool(lse[lost].isnan().all())
    assert float((o[~lost] - o_ref[~lost]).norm()) <= 5e-3 * float(o_ref[~lost].norm())
    assert float(((lse - lse_ref)[~lost].abs() / lse_ref[~lost].abs().clamp_min(1.0)).max()) <= 1e-3


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("n,T", [(3, 100), (5, 64), (2, 440)])
def test_training_form(mw, n, T, d):
    q, k, v = (bf(i, 1, 2, n * T, d) for i in range(3))
    o_ref, lse_ref = oracle.fwd(q, k, v, T, d ** -0.5)
    q[0, 0, T + 3, 7] = math.nan
    k[0, 1, T + 5, d - 1] = math.nan  # of the second chunk, which the first does not see
    lost = torch.zeros(1, 2, n * T, dtype=torch.bool)
    lost[0, 0, T + 3] = lost[0, 1, T:] = True
    check(*mw.mw_bca_fwd(q.cuda(), k.cuda(), v.cuda(), T), o_ref, lse_ref, lost)


@pytest.mark.parametrize("d", [64, 72, 128])
@pytest.mark.parametrize("sink", [0, 50])
@pytest.mark.parametrize("n,T,cap,length", [(1, 64, 2048, 2000), (2, 200, 1000, 900), (2, 60, 8, 0)])
def test_ring_form(mw, n, T, cap, length, sink, d):
    """Long rings are split into ranges of keys, whose join has to keep the NaN; a sink's keys
    turn as they are read.  The reference is the call without the NaN."""
    q, kn, vn = (bf(10 + i, 1, 2, n * T, d) for i in range(3))
    ks, vs = (bf(13 + i, 1, 2, cap, d) for i in range(2))
    anchor = [bf(15 + i, 1, 2, sink, d).cuda() for i in range(2)] if sink else [None, None]

    def call(q, kn, kr):
        args = [t.cuda() for t in (q, kn, vn)] + anchor + [kr.cuda(), vs.cuda(), 0, length, T]
        if sink:
            return mw.mw_bca_cache_fwd_rope(*args, 16, 1e4, 3)
        return mw.mw_bca_cache_fwd(*args[:3], *args[5:])

    o_ref, lse_ref = (t.double().cpu() for t in call(q, kn, ks))
    for where, i in [("q", T // 2), ("new", 3)] + ([("ring", length // 2)] if length else []):
        qq, kk, kr = q.clone(), kn.clone(), ks.clone()
        lost = torch.zeros(1, 2, n * T, dtype=torch.bool)
        if where == "q":
            qq[0, 1, i, 0] = math.nan
            lost[0, 1, i] = True
        else:
            (kk if where == "new" else kr)[0, 1, i, 1] = math.nan
            lost[0, 1] = True
        check(*call(qq, kk, kr), o_ref, lse_ref, lost)
