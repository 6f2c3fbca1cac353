"""fp64 CPU definitions of the 8-bit projections: the 8-bit form with block scales, the product
of two forms, RMS norm (test infrastructure only).

8-bit form: blocks of r x c elements, s the least power of two with max |x| <= 448 s, at
least 2^-127, code = the e4m3 value next to x / s, ties to an even last place.  A block that
is not finite everywhere stands for NaN.

RMS norm with a weight for each of G equal groups of rows, of h = x + residual rounded to
x's type:

    y = h * w_g / sqrt(mean h^2 + eps)
"""
from __future__ import annotations

import torch

from .bca import F64
from .cond import _per_row


def e4m3(v):
    """The values of e4m3 next to v, |v| <= 448: three bits after the leading one down to
    2^-6, steps of 2^-9 below; ties to even."""
    _, exponent = torch.frexp(v)  # |v| in [2^(exponent - 1), 2^exponent)
    step = torch.pow(torch.tensor(2.0, dtype=F64), (exponent - 1).clamp(min=-6).to(F64) - 3)
    return torch.round(v / step) * step


def blocks(x, rows: int, columns: int):
    """[ceil(R / rows), ceil(C / columns), rows, columns] with zeros past the ends."""
    R, C = x.shape
    x = torch.nn.functional.pad(x, (0, -C % columns, 0, -R % rows))
    return x.view(x.shape[0] // rows, rows, x.shape[1] // columns, columns).transpose(1, 2)


def form(x, rows: int, columns: int):
    """(values that the form stands for [R, C], exponents of the scales; 128 for NaN)."""
    R, C = x.shape
    b = blocks(x.to(F64), rows, columns)
    top = b.abs().amax((2, 3))
    good = torch.isfinite(b).all(3).all(2)
    mantissa, exponent = torch.frexp(torch.where(good, top, 0.0))
    # top = mantissa 2^exponent, 448 = 0.875 2^9: the quotient's power, rounded up
    e = exponent - 9 + (mantissa > 0.875).int()
    e = torch.where(top == 0, -127, e).clamp(min=-127)
    s = torch.pow(torch.tensor(2.0, dtype=F64), e.to(F64))[:, :, None, None]
    v = torch.where(good[:, :, None, None], e4m3(torch.where(good[:, :, None, None], b, 0.0) / s) * s, float("nan"))
    v = v.transpose(1, 2).reshape(b.shape[0] * rows, b.shape[1] * columns)[:R, :C]
    return v, torch.where(good, e, 128)


def values(q, scale, rows: int, columns: int):
    """What codes and scales stand for, from torch's own types."""
    s = scale.float().to(F64).repeat_interleave(rows, 0)[:q.shape[0]].repeat_interleave(columns, 1)
    return q.float().to(F64) * s[:, :q.shape[1]]


def rms_fwd(x, residual, weight, eps: float):
    """(y, h, rstd) in fp64, h as it is rounded."""
    h = x if residual is None else (x.to(F64) + residual.to(F64)).to(x.dtype)
    h64 = h.to(F64)
    R, C = h.shape
    rstd = 1.0 / torch.sqrt((h64 * h64).sum(1) / C + eps)
    y = h64 * rstd[:, None]
    if weight is not None:
        y = y * _per_row(weight, R)
    return y, h64, rstd


def rms_bwd(dy, h, weight, eps: float, dh=None, groups: int = 1):
    """(dx, dweight [groups, C] or None) in fp64 of sum(y dy) + sum(h dh)."""
    h, g = h.to(F64), dy.to(F64)
    R, C = h.shape
    rstd = 1.0 / torch.sqrt((h * h).sum(1, keepdim=True) / C + eps)
    xh = h * rstd
    dw = None if weight is None else (g * xh).view(groups, R // groups, C).sum(1)
    if weight is not None:
        g = g * _per_row(weight, R)
    dx = rstd * (g - xh * ((g * xh).sum(1, keepdim=True) / C))
    return dx if dh is None else dx + dh.to(F64), dw
