"""fp64 CPU definitions of the conditioning path: cross attention to an encoder's
states and layer norm, with their gradients (test infrastructure only).

Cross attention: q [B, H, M, d] against k, v [B, Hkv, S, d], H / Hkv query heads
to a head of K and V, the first lens[b] states of sample b valid:

    s_ij = scale * <q_i, k_j> for j < lens[b],  LSE_i = ln sum_j exp(s_ij)
    O_i  = sum_j exp(s_ij - LSE_i) v_j          (no state: O_i = 0, LSE_i = -inf)

Layer norm with a weight and bias for each of G equal groups of rows:

    xh = (x - mean) / sqrt(var + eps),  y = xh * w_g + b_g
"""
from __future__ import annotations

import math
from typing import List, Optional

import torch

from .bca import F64


def xattn_fwd(q, k, v, lens: Optional[List[int]], scale: float):
    """(O, LSE) in fp64, head by head."""
    B, H, M, d = q.shape
    share = H // k.shape[1]
    o = torch.zeros(B, H, M, d, dtype=F64)
    lse = torch.full((B, H, M), -math.inf, dtype=F64)
    for b in range(B):
        n = k.shape[2] if lens is None else min(max(int(lens[b]), 0), k.shape[2])
        if n == 0:
            continue
        for h in range(H):
            s = scale * (q[b, h].to(F64) @ k[b, h // share, :n].to(F64).T)
            top = s.max(1, keepdim=True).values
            e = torch.exp(s - top)
            total = e.sum(1, keepdim=True)
            o[b, h] = (e / total) @ v[b, h // share, :n].to(F64)
            lse[b, h] = (top + torch.log(total))[:, 0]
    return o, lse


def xattn_bwd(q, k, v, dout, lens: Optional[List[int]], scale: float):
    """(dQ, dK, dV) in fp64 of sum(O * dout)."""
    B, H, M, d = q.shape
    share = H // k.shape[1]
    dq = torch.zeros(q.shape, dtype=F64)
    dk, dv = torch.zeros(k.shape, dtype=F64), torch.zeros(v.shape, dtype=F64)
    o, lse = xattn_fwd(q, k, v, lens, scale)
    for b in range(B):
        n = k.shape[2] if lens is None else min(max(int(lens[b]), 0), k.shape[2])
        if n == 0 or M == 0:
            continue
        for h in range(H):
            c = h // share
            qf, kf, vf, g = (t.to(F64) for t in (q[b, h], k[b, c, :n], v[b, c, :n], dout[b, h]))
            p = torch.exp(scale * (qf @ kf.T) - lse[b, h][:, None])
            dv[b, c, :n] += p.T @ g
            ds = p * (g @ vf.T - (g * o[b, h]).sum(1, keepdim=True))
            dq[b, h] = scale * (ds @ kf)
            dk[b, c, :n] += scale * (ds.T @ qf)
    return dq, dk, dv


def norm_fwd(x, weight, bias, eps: float):
    """(y, mean, rstd) in fp64; x [R, C], weight and bias [C], [G, C] or None."""
    x = x.to(F64)
    R, C = x.shape
    mean = x.sum(1) / C
    rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).sum(1) / C + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * _per_row(weight, R)
    if bias is not None:
        y = y + _per_row(bias, R)
    return y, mean, rstd


def _per_row(t, R):
    t = t.to(F64).reshape(-1, t.shape[-1])
    return t.repeat_interleave(R // t.shape[0], 0)


def norm_bwd(dy, x, weight, eps: float, groups: int):
    """(dx, dweight [G, C], dbias [G, C]) in fp64 of sum(y * dy)."""
    x, dy = x.to(F64), dy.to(F64)
    R, C = x.shape
    _, mean, rstd = norm_fwd(x, None, None, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy if weight is None else dy * _per_row(weight, R)
    dx = rstd[:, None] * (g - g.sum(1, keepdim=True) / C - xh * ((g * xh).sum(1, keepdim=True) / C))
    return dx, (dy * xh).view(groups, -1, C).sum(1), dy.view(groups, -1, C).sum(1)
