"""The 64-bit definitions of the 8-bit projections, held to torch's own types, to brute force
over all codes and to differences."""
import math

import pytest
import torch

from oracle import fp8

F64 = torch.float64


def test_e4m3_is_the_nearest_code():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().to(F64)
    codes = torch.unique(codes[torch.isfinite(codes)])
    assert codes.max() == 448.0
    middles = (codes[1:] + codes[:-1]) / 2
    v = torch.cat([codes, middles, middles * (1 + 2.0 ** -40), middles * (1 - 2.0 ** -40),
                   torch.randn(2000, generator=torch.Generator().manual_seed(0), dtype=F64) * 50])
    v = v[v.abs() <= 448]
    got = fp8.e4m3(v)
    distance = (v[:, None] - codes[None]).abs()
    assert torch.equal((got - v).abs(), distance.min(1).values)
    # ties: the code with the even last place, as torch rounds
    assert torch.equal(fp8.e4m3(middles), middles.float().to(torch.float8_e4m3fn).float().to(F64))


@pytest.mark.parametrize("rows,columns", [(1, 128), (128, 1), (128, 128)])
def test_form_by_brute_force(rows, columns):
    x = torch.randn(130, 144, generator=torch.Generator().manual_seed(1)) * 7
    x[3, 5], x[40:, 20] = 1e4, 0.0
    v, e = fp8.form(x, rows, columns)
    assert e.shape == (math.ceil(130 / rows), math.ceil(144 / columns))
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            at = slice(i * rows, (i + 1) * rows), slice(j * columns, (j + 1) * columns)
            top = float(x[at].abs().max())
            s = 2.0 ** int(e[i, j])
            if top > 0:
                assert top <= 448 * s and top > 448 * s / 2
            q = (x[at].double() / s).float().to(torch.float8_e4m3fn)
            assert torch.equal(v[at], q.double() * s)


def test_form_of_limits():
    x = torch.zeros(6, 16)
    x[0, 0], x[1, 0], x[2, 0], x[3, 3], x[4, 1] = 448.0, 448.00003, 3.4e38, float("inf"), float("nan")
    x[5, 2] = 1e-40
    v, e = fp8.form(x, 1, 128)
    assert e[:, 0].tolist() == [0, 1, 120, 128, 128, -127]
    assert torch.isnan(v[3:5]).all() and torch.isfinite(v[[0, 1, 2, 5]]).all()


@pytest.mark.parametrize("groups", [1, 3])
def test_rms_gradients_by_differences(groups):
    g = torch.Generator().manual_seed(2)

    def randn(*shape):
        return torch.randn(*shape, generator=g, dtype=F64)

    R, C, eps = 6, 5, 1e-2
    x, w = randn(R, C), randn(*((C,) if groups == 1 else (groups, C)))
    dy, dh = randn(R, C), randn(R, C)

    def loss(x, w):
        y, h, _ = fp8.rms_fwd(x, None, w, eps)
        return float((y * dy).sum() + (h * dh).sum())

    dx, dw = fp8.rms_bwd(dy, x, w, eps, dh, groups)
    step = 1e-6
    for t, grad in ((x, dx), (w, dw.view(w.shape))):
        for i in range(t.numel()):
            moved = []
            for s in (step, -step):
                u = t.clone().view(-1)
                u[i] += s
                u = u.view(t.shape)
                moved.append(loss(u, w) if t is x else loss(x, u))
            assert abs((moved[0] - moved[1]) / (2 * step) - float(grad.reshape(-1)[i])) < 1e-7


def test_rms_adds_the_residual_as_it_is_stored():
    x = torch.tensor([[1.0, 256.0]], dtype=torch.bfloat16)
    r = torch.tensor([[2.0 ** -9, 1.0]], dtype=torch.bfloat16)
    y, h, rstd = fp8.rms_fwd(x, r, None, 0.0)
    assert h.tolist() == [[1.0, 256.0]]  # both sums are ties, to the even neighbour
    assert torch.allclose(y, h * rstd[:, None])
