"""Gradients of a cross attention sample by sample and head by head, few rows against many
states among them, whose dK and dV are small (P is about 1 / S) without cancelling.

Tolerances, from the number formats.  dV = P^T dO: P and the result are rounded to bf16
(1.7e-3 each in the mean square); 1e-2 of a head's norm allows for sums too short to
average.  dS = P (dP - D) is rounded likewise, so that dQ and dK have the same 1e-2; of more
than eight states D = <dO, O> carries besides what O lost in bf16, dD_i <= 2^-9 sum_c |dO_ic
O_ic|, and with it dS_ij is off by P_ij dD_i.  One state: dS is 0, and what is left is the
rounding of dP - D, 2^-8 of sum_c |dO_ic v_c| at most."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mw():
    import paper_2608_01127_gb300 as pkg
    pkg.library()
    return pkg


def bf(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


SIZES = [  # B, H, Hkv, M, S, d, lens
    (1, 8, 2, 1, 2000, 72, None),
    (1, 1, 1, 40, 1500, 64, None),
    (1, 1, 1, 40, 1500, 128, [1400]),
    (1, 6, 2, 5, 1000, 128, [999]),
    (2, 5, 1, 1, 513, 128, [1, 513]),
    (2, 4, 4, 1, 300, 128, [300, 17]),
    (3, 4, 2, 3, 129, 64, [0, 129, 128]),
    (4, 4, 2, 130, 200, 88, [0, 1, 127, 200]),
    (1, 16, 1, 1, 640, 80, [511]),
    (2, 4, 2, 200, 385, 128, [385, 128]),
    (2, 2, 2, 640, 640, 64, [633, 257]),
    (1, 20, 4, 66, 301, 128, [301]),
    (1, 1, 1, 1, 4097, 64, None),
    (1, 2, 1, 1100, 33, 72, [30]),
]


@pytest.mark.parametrize("B,H,Hkv,M,S,d,lens", SIZES)
def test_every_head_of_every_sample(mw, B, H, Hkv, M, S, d, lens):
    q, k, v, do = (t.cuda() for t in (bf(0, B, H, M, d), bf(1, B, Hkv, S, d), bf(2, B, Hkv, S, d), bf(3, B, H, M, d)))
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = mw.mw_xattn_fwd(q, k, v, kv_len)
    dq, dk, dv = mw.mw_xattn_bwd(q, k, v, o, lse, do, kv_len)
    scale, share = d ** -0.5, H // Hkv
    for b in range(B):
        n = S if lens is None else lens[b]
        assert torch.count_nonzero(dk[b, :, n:]) == 0 and torch.count_nonzero(dv[b, :, n:]) == 0
        if n == 0:
            assert torch.count_nonzero(dq[b]) == 0
            continue
        for h in range(Hkv):
            rows = lambda t: t[b, share * h:share * (h + 1)].reshape(share * M, d).double()  # noqa: E731
            qh, gh, kh, vh = rows(q), rows(do), k[b, h, :n].double(), v[b, h, :n].double()
            p = torch.softmax(scale * qh @ kh.T, -1)
            oh = p @ vh
            ds = p * (gh @ vh.T - (gh * oh).sum(1, keepdim=True))
            lost = 2.0 ** -9 * (gh * oh).abs().sum(1, keepdim=True) * p if n > 8 else torch.zeros_like(p)
            if n == 1:
                ds = torch.zeros_like(ds)
                lost = 2.0 ** -8 * (gh.abs() @ vh.abs().T)
            for name, got, ref, more in (("dv", dv[b, h, :n], p.T @ gh, None),
                                         ("dk", dk[b, h, :n], scale * ds.T @ qh, scale * lost.T @ qh.abs()),
                                         ("dq", rows(dq), scale * ds @ kh, scale * lost @ kh.abs())):
                err = float((got.double() - ref).norm())
                assert err <= 1e-2 * float(ref.norm()) + (0.0 if more is None else float(more.norm())), (name, b, h)
