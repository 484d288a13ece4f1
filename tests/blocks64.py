"""The head, the root-mean-square norms and the clipped gradients from their definitions in 64 bits, and how far their fp32 arithmetic with
one final rounding may be off. Shares no code with the library. Runs where its inputs are.

Tolerances. A rounding is off by at most half a step, U = finfo(t).eps / 2 relative. A sum of products by fp32 fused operations or by the
tensor cores, which cut what they add to 2^-23 of the largest, in stretches of at most 64 additions that join by rounded ones, is off by at
most g = (h / 512 + 64) 2^-23 of the sum of the terms' magnitudes. An exponential of a difference is off by 2^-21 and by the difference's
own error.

Head. z is off by dz = g sum |x w|, and lse by the largest dz and 2^-20; a loss by both. d = (p - [target]) g: by p (dz + that of lse + 2^-20),
and by the rounding of its planes, U of the result's type (three planes: 2^-24; two: 2^-17). dx and dW: the terms' errors, the sum's g, for
dx of a 16-bit type beside an fp32 weight the planes of W that are left out (bf16: 2^-17 of |d w|), and the final rounding."""
import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
E = 2.0 ** -24
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def check(got, want, tol, what):
    """Elementwise within tol and the result's own rounding; the two have infinities and NaNs at the same places."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g, u = got.detach().double(), U[got.dtype]
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), what + ": NaN elsewhere"
    assert torch.equal(g[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities"
    over = ((g - want).abs() - tol - u * (want.abs() + tol) - TINY[got.dtype])[fine]
    assert not (over > 0).any(), "%s: off by up to %.3g more than the tolerance, at %d of %d" % (what, over.max(), (over > 0).sum(), over.numel())


def near(got, want, most, what):
    """The 2-norm of the difference, relative; near zero each element may be off by a unit there."""
    off = float((got.detach().double() - want).norm()), float(want.norm())
    assert off[0] <= most * off[1] + TINY[got.dtype] * want.numel() ** 0.5, "%s: %.3g off, relative to its length" % (what, off[0] / max(off[1], 1e-300))


def head(x, weight, target, reduction, ignored=-100, dloss=None):
    """loss, its tolerance, and (dx, tolerance, dW, tolerance) where dloss is given: x [n, rows, h], weight [vocab, h] or [n, vocab, h];
    dW of a weight [n, ...] is apart."""
    n, rows, h = x.shape
    vocab, kind, wkind = weight.shape[-2], x.dtype, weight.dtype
    g = (h / 512 + 64) * 2 * E
    x64, together = x.double(), weight.dim() == 2
    losses, tols, dxs, txs, dws, tws = [], [], [], [], [], []
    counted = (target != ignored).reshape(n, rows)
    valid = counted & (target.reshape(n, rows) >= 0) & (target.reshape(n, rows) < vocab)
    for i in range(n):
        w = (weight if together else weight[i]).double()
        t = torch.where(valid[i], target.reshape(n, rows)[i], 0)
        z, dz = x64[i] @ w.T, g * (x64[i].abs() @ w.abs().T)
        lse = torch.logsumexp(z, -1)
        tz = dz.amax(-1) + 2.0 ** -20
        row = lse - z.gather(-1, t[:, None])[:, 0]
        row = torch.where(valid[i], row, torch.where(counted[i], float("nan"), 0.0))
        tol = torch.where(counted[i], 2 * tz + 4 * E * (lse.abs() + z.abs().amax(-1)), 0.0)
        count = max(1, int(counted[i].sum()))
        if reduction == "none":
            losses.append(row), tols.append(tol)
            gr = None if dloss is None else dloss.reshape(n, rows)[i].double()
        else:
            by = count if reduction == "mean" else 1
            losses.append(row.sum() / by), tols.append((tol.sum() + (rows / 256 + 16) * E * row.abs().sum()) / by)
            gr = None if dloss is None else (dloss[i].double() / by).expand(rows)
        if dloss is None:
            continue
        gr = torch.where(valid[i], gr, torch.where(counted[i], float("nan"), 0.0))
        p = torch.exp(z - lse[:, None])
        dp = p * (dz + tz[:, None] + 2.0 ** -19)
        delta = p.clone()
        delta[torch.arange(rows, device=x.device), t] -= 1.0
        d = delta * gr[:, None]
        dead = ~counted[i]
        d[dead] = 0.0
        size, err = d.abs(), dp * gr.abs()[:, None] + 4 * E * d.abs() + 2.0 ** -38 * gr.abs()[:, None]
        size[dead], err[dead] = 0.0, 0.0

        def product(left, left_err, right, planes, terms, lost):
            """left @ right and its error; planes: what the rounding of left to its planes leaves out."""
            s = left.abs() @ right.abs()
            return left @ right, left_err @ right.abs() + (planes + lost + (terms / 512 + 64) * 2 * E) * s

        px = {torch.bfloat16: U[torch.bfloat16], torch.float16: U[torch.float16] if wkind != torch.float32 else 2.0 ** -17, torch.float32: E}[kind]
        a, b = product(d, err, w, px, vocab, 2.0 ** -16 if wkind != kind else 3 * E)
        dxs.append(a), txs.append(b)
        pw = E if wkind == torch.float32 else U[wkind]
        a, b = product(d.T, err.T, x64[i], pw, rows, 3 * E)
        dws.append(a), tws.append(b)
    loss, tol = torch.stack(losses), torch.stack(tols)
    if reduction == "none":
        loss, tol = loss.reshape(target.shape), tol.reshape(target.shape)
    if dloss is None:
        return loss, tol
    dw, tw = torch.stack(dws), torch.stack(tws)
    return loss, tol, torch.stack(dxs), torch.stack(txs), dw.sum(0) if together else dw, tw.sum(0) if together else tw


# ---- norms -----------------------------------------------------------------------------------------------------------------


def _r(v, eps):
    return 1.0 / (v.square().mean(-1, keepdim=True) + eps).sqrt()


def rms(v, w, eps):
    """y and its tolerance before its rounding; w [n, 1, h] or 1."""
    y = v * _r(v, eps) * w
    return y, (v.shape[-1] / 512 + 64) * E * y.abs()


def gated(x, residual, w, g, alpha, eps):
    """s before its rounding, and its tolerance in fp32."""
    u, tol = rms(x, w, eps)
    return alpha * residual + g * u, g.abs() * tol + 4 * E * ((alpha * residual).abs() + (g * u).abs()) if torch.is_tensor(g) else tol + 4 * E * (
        (alpha * residual).abs() + u.abs())


def rms_gradients(dy, tdy, v, w, eps):
    """(dv, its tolerance, dw, its tolerance) of rms with a gradient dy that is off by tdy."""
    h = v.shape[-1]
    k = (h / 512 + 64) * E
    r = _r(v, eps)
    vhat, a = v * r, dy * w
    w_abs = w.abs() if torch.is_tensor(w) else abs(w)
    ta = tdy * w_abs + 2 * E * a.abs()
    mean = (a * vhat).mean(-1, keepdim=True)
    tmean = (ta * vhat.abs() + 2 * k * (a * vhat).abs()).mean(-1, keepdim=True)
    dv = r * (a - vhat * mean)
    tdv = r * (ta + vhat.abs() * tmean) + 2 * k * r * (a.abs() + (vhat * mean).abs())
    rows = v.shape[1]
    return dv, tdv, (dy * vhat).sum(1), (tdy * vhat.abs() + (2 * k + (rows / 4 + 64) * E) * (dy * vhat).abs()).sum(1)
