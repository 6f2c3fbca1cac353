"""A forward against the ring in ranges of keys, of which some are given up: the rows get
O = 0 and LSE = -inf, not a softmax over the ranges that are left."""
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

OK, TIMEOUT = 0, 4


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    assert pkg.mw_device_status(clear=True) == OK
    return pkg


@pytest.mark.parametrize("hook", [1, 2])
@pytest.mark.parametrize("sink", [0, 40])
@pytest.mark.parametrize("d", [64, 72, 128])
def test_ranges_given_up(mw, d, sink, hook):
    T, cap = 64, 2000
    g = torch.Generator().manual_seed(3)
    q, kn, vn = (torch.randn(1, 2, T, d, generator=g).to(torch.bfloat16) for _ in range(3))
    k, v = (torch.randn(1, 2, cap, d, generator=g).to(torch.bfloat16) for _ in range(2))
    ks, vs = (torch.randn(1, 2, sink, d, generator=g).to(torch.bfloat16) for _ in range(2))
    assert mw.mw_bca_cache_workspace_size(1, 2, 1, T, d, cap + sink) > 0  # several ranges
    anchor = [t.cuda() for t in (ks, vs)] if sink else [None, None]
    args = [t.cuda() for t in (q, kn, vn)] + anchor + [t.cuda() for t in (k, v)]

    def call():
        return mw.mw_bca_cache_fwd_sink(*args, 0, cap, T) if sink else mw.mw_bca_cache_fwd(*args[:3], *args[5:], 0, cap, T)

    mw.mw_set_option("wait_budget_ms", 100)
    mw.mw_set_option("debug_skip_q_load", hook)
    try:
        o, lse = call()
        status = mw.mw_device_status(clear=True)
    finally:
        mw.mw_set_option("debug_skip_q_load", 0)
        mw.mw_set_option("wait_budget_ms", 2000)
    assert status == TIMEOUT
    assert torch.count_nonzero(o) == 0 and bool((lse == -float("inf")).all())
    o, lse = call()
    torch.cuda.synchronize()
    assert mw.mw_device_status() == OK
    ref, lse_ref = oracle.cache_fwd(q, kn, vn, k, v, cap, 0, cap, T, d ** -0.5, *((ks, vs) if sink else ()))
    assert float((o.double().cpu() - ref).norm()) <= 5e-3 * float(ref.norm())
    assert float((lse.double().cpu() - lse_ref).abs().max()) <= 1e-3 * max(1.0, float(lse_ref.abs().max()))
