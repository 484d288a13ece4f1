"""Gradients of the norms on rows far from zero. The values are 1000 + j / 16 with small whole j that cancel over every 256 columns, and the
widths powers of two, so every sum of values and the mean are exact in fp32: what is left of xhat = (v - mean) rstd is rstd's error and
a rounding, a few 2^-24 of it, where a product of the mean itself would leave 2^-24 of 1000 rstd."""
import pytest
import torch

import operators64 as R
from paper_2205_05632_b200.layers import dropout_add_layer_norm, layer_norm

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
E = R.E


def deviations(g, n, rows, h):
    """Multiples of 2^-4 from -1/2 to 1/2, not 0, the second half of every 256 columns the negatives of the first."""
    half = min(h, 256) // 2
    j = torch.randint(1, 9, (n, rows, h // (2 * half), 1, half), generator=g, device="cuda") * (
        1 - 2 * torch.randint(0, 2, (n, rows, h // (2 * half), 1, half), generator=g, device="cuda"))
    return (torch.cat((j, -j), dim=3).reshape(n, rows, h) / 16.0).float()


def wanted(dy, v, w, eps):
    """(value, tolerance) of dv and dw. rstd: the sum of squares is off by g, the root and the quotient by 2; xhat: 2 more roundings."""
    h, rows = v.shape[-1], v.shape[1]
    g, gr = (h / 512 + 64) * E, (rows + 64) * E
    mean = v.mean(-1, keepdim=True)
    rstd = ((v - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    xhat = (v - mean) * rstd
    er = g + 4 * E
    ex = er * xhat.abs()
    q = dy * w
    c1, c2 = q.mean(-1, keepdim=True), (q * xhat).mean(-1, keepdim=True)
    e1 = g * q.abs().mean(-1, keepdim=True)
    e2 = (g + er) * (q * xhat).abs().mean(-1, keepdim=True)
    dv = rstd * (q - c1 - xhat * c2)
    tol = rstd * (e1 + xhat.abs() * e2 + ex * c2.abs() + 8 * E * (q.abs() + c1.abs() + (xhat * c2).abs())) + dv.abs() * er
    return (dv, tol), ((dy * xhat).sum(1), (dy.abs() * ex).sum(1) + gr * (dy * xhat).abs().sum(1))


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("h", [64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384, 32768])
def test_gradients_of_rows_far_from_zero(h, shift):
    n, rows = 2, 5
    g = torch.Generator(device="cuda").manual_seed(h + shift)
    dev = deviations(g, n, rows, h)

    def placed(t):  # shift 1: rows that start off 16-byte boundaries
        q = torch.zeros(n, rows, h + 8, dtype=t.dtype, device="cuda")
        q[..., shift:shift + h] = t
        return q[..., shift:shift + h].detach().requires_grad_()

    w, b = (1 + 0.3 * torch.randn(h, generator=g, device="cuda")).expand(n, h).detach().requires_grad_(), torch.zeros(n, h, device="cuda")
    dy = torch.randn(n, rows, h, generator=g, device="cuda")
    x = placed(1000.0 + dev)
    dx, dw = torch.autograd.grad(layer_norm(x, w, b), (x, w), dy)
    (want, tol), (ww, tw) = wanted(R.d(dy), R.d(x), R.d(w)[:, None], 1e-5)
    R.check(dx, want, tol, "dx")
    R.check(dw, ww, tw, "dweight")
    # the residual far from zero, the branch's values small
    x, r = placed(dev.to(BF16)), placed(torch.full_like(dev, 1000.0))
    dy = dy.to(BF16)
    y, s = dropout_add_layer_norm(x, r, w, b)
    assert torch.equal(s, 1000.0 + dev)
    dx, dr, dw = torch.autograd.grad(y, (x, r, w), dy)
    (want, tol), (ww, tw) = wanted(R.d(dy), R.d(s), R.d(w)[:, None], 1e-5)
    R.check(dr, want, tol, "dresidual")
    R.check(dx, want, tol, "dx")
    R.check(dw, ww, tw, "dweight")
