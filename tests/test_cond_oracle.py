"""The 64-bit definitions of the conditioning path (oracle/cond.py), on the CPU:
against PyTorch's own functions, their gradients against central differences."""
import math

import pytest
import torch
import torch.nn.functional as F

import oracle

F64 = torch.float64


def gen(seed, *shapes):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g, dtype=F64) for s in shapes]


def differences(f, x, step=1e-6):
    """Central differences of the scalar f at x."""
    out = torch.zeros_like(x)
    flat, og = x.reshape(-1), out.reshape(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        flat[i] = keep + step
        up = f()
        flat[i] = keep - step
        og[i] = (up - f()) / (2 * step)
        flat[i] = keep
    return out


@pytest.mark.parametrize("H,Hkv,M,S,lens", [(2, 2, 3, 5, None), (4, 2, 3, 5, [5, 2]), (3, 1, 1, 4, [0, 1])])
def test_cross_attention_is_the_library_function(H, Hkv, M, S, lens):
    q, k, v = gen(1, (2, H, M, 8), (2, Hkv, S, 8), (2, Hkv, S, 8))
    o, lse = oracle.xattn_fwd(q, k, v, lens, 0.3)
    kk, vv = (t.repeat_interleave(H // Hkv, 1) for t in (k, v))
    for b in range(2):
        n = S if lens is None else lens[b]
        if n == 0:
            assert torch.count_nonzero(o[b]) == 0 and bool((lse[b] == -math.inf).all())
            continue
        ref = F.scaled_dot_product_attention(q[b:b + 1], kk[b:b + 1, :, :n], vv[b:b + 1, :, :n], scale=0.3)
        assert torch.allclose(o[b:b + 1], ref, atol=1e-12, rtol=0)
        s = 0.3 * (q[b] @ kk[b, :, :n].transpose(1, 2))
        assert torch.allclose(lse[b], torch.logsumexp(s, -1), atol=1e-12, rtol=0)


@pytest.mark.parametrize("H,Hkv,M,S,lens", [(2, 2, 3, 4, None), (4, 2, 2, 4, [3, 0]), (2, 1, 1, 1, [1, 1])])
def test_cross_attention_gradients_by_differences(H, Hkv, M, S, lens):
    q, k, v, do = gen(2, (2, H, M, 4), (2, Hkv, S, 4), (2, Hkv, S, 4), (2, H, M, 4))

    def loss():
        return float((oracle.xattn_fwd(q, k, v, lens, 0.4)[0] * do).sum())

    grads = oracle.xattn_bwd(q, k, v, do, lens, 0.4)
    for t, g in zip((q, k, v), grads):
        # second order of the step, and rounding of the loss over the step
        assert float((differences(loss, t) - g).abs().max()) < 1e-7


def test_padded_states_do_not_count():
    q, k, v, do = gen(3, (1, 2, 3, 4), (1, 2, 5, 4), (1, 2, 5, 4), (1, 2, 3, 4))
    whole = oracle.xattn_bwd(q, k[:, :, :3].clone(), v[:, :, :3].clone(), do, None, 0.5)
    k[:, :, 3:], v[:, :, 3:] = math.nan, math.inf
    padded = oracle.xattn_bwd(q, k, v, do, [3], 0.5)
    assert torch.equal(padded[0], whole[0])
    for a, b in zip(padded[1:], whole[1:]):
        assert torch.equal(a[:, :, :3], b) and torch.count_nonzero(a[:, :, 3:]) == 0


@pytest.mark.parametrize("groups", [1, 3])
def test_layer_norm_is_the_library_function(groups):
    x, w, b = gen(4, (6, 10), (groups, 10), (groups, 10))
    y, mean, rstd = oracle.norm_fwd(x, w, b, 1e-3)
    for g in range(groups):
        rows = slice(g * 6 // groups, (g + 1) * 6 // groups)
        assert torch.allclose(y[rows], F.layer_norm(x[rows], (10,), w[g], b[g], 1e-3), atol=1e-12, rtol=0)
    assert torch.allclose(mean, x.mean(1)) and torch.allclose(rstd, (x.var(1, correction=0) + 1e-3).rsqrt())


@pytest.mark.parametrize("groups", [1, 2])
def test_layer_norm_gradients_by_differences(groups):
    x, w, b, dy = gen(5, (4, 7), (groups, 7), (groups, 7), (4, 7))

    def loss():
        return float((oracle.norm_fwd(x, w, b, 1e-2)[0] * dy).sum())

    dx, dw, db = oracle.norm_bwd(dy, x, w, 1e-2, groups)
    for t, g in ((x, dx), (w, dw), (b, db)):
        assert float((differences(loss, t) - g).abs().max()) < 1e-7
