"""The operators of paper_2205_05632_b200.layers from their definitions in 64 bits, on the CPU, and how far fp32 arithmetic with one
final rounding may be from them. Shares no code with the library.

Tolerances. U[t] = finfo(t).eps / 2 is a rounding's largest relative error. A sum of k fp32 terms is off by at most g(k) times the sum
of their magnitudes; the kernels add at most h / 512 + 64 terms one after another (a thread's, then a tree over lanes and warps), so
g = (h / 512 + 64) 2^-24 covers them, products and the tensor cores' additions of exact products included. Where such a sum enters a
formula its error goes through the formula by the product rule; the few roundings of the formula itself count 8 2^-24."""
import numpy as np
import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
E = 2.0 ** -24
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}  # results near zero: one unit there


def philox(counter, key):
    """Philox4x32-10 on arrays of uint64 that hold 32-bit words."""
    mask, w = np.uint64(0xFFFFFFFF), np.uint64
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(10):
        p0, p1 = w(0xD2511F53) * c[0], w(0xCD9E8D57) * c[2]
        c = [(p1 >> w(32)) ^ c[1] ^ w(k[0]), p1 & mask, (p0 >> w(32)) ^ c[3] ^ w(k[1]), p0 & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def factor(n, rows, h, p, seed=0, call=0, worker=0):
    """[n, rows, h] float64: 0 where an element is dropped, the factor of the others elsewhere."""
    t = int(np.floor(65536.0 * p + 0.5))
    groups = (h + 7) // 8
    shape = (n, rows, groups)
    counter = [np.broadcast_to(np.arange(groups).reshape(1, 1, -1), shape), np.broadcast_to(np.arange(rows).reshape(1, -1, 1), shape),
               np.broadcast_to(worker + np.arange(n).reshape(-1, 1, 1), shape), np.full(shape, call)]
    words = philox([c.astype(np.uint64) for c in counter], (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([(w >> np.uint64(16 * half)) & np.uint64(0xFFFF) for w in words for half in (0, 1)], axis=-1)
    keep = u.reshape(n, rows, 8 * groups)[:, :, :h] >= t
    return torch.from_numpy(keep.astype(np.float64) * (65536.0 / (65536 - t) if t < 65536 else 0.0))


def d(t):
    return t.detach().cpu().double()


def flat(t):
    """[n, ..., h] as [n, rows, h]."""
    return t.reshape(t.shape[0], -1, t.shape[-1])


def masked(v, f):
    """v f, with zeros where f is 0, whatever v is there."""
    return torch.where(f == 0, torch.zeros_like(v), v * f)


def norm(v, w, b, eps):
    """y and the tolerance of y before its rounding; w, b: [n, 1, h] float64."""
    h = v.shape[-1]
    g = (h / 512 + 64) * E
    mean = v.mean(-1, keepdim=True)
    var = (v - mean).square().mean(-1, keepdim=True)
    rstd = (var + eps).rsqrt()
    xhat = (v - mean) * rstd
    # mean: g mean|v|; the differences from it carry that, and enter the variance to second order and by 2 mean(v - mean) = 0 to first
    dm = g * v.abs().mean(-1, keepdim=True) + 2 * E * (v.abs() + mean.abs())
    ex = rstd * dm + xhat.abs() * (g + 8 * E + (rstd * dm.amax(-1, keepdim=True)).square() + rstd * 2 * E * (v.abs() + mean.abs()).amax(-1, keepdim=True))
    y = xhat * w + b
    return y, ex * w.abs() + 8 * E * (y.abs() + (xhat * w).abs() + b.abs()), mean, rstd, xhat, ex


def norm_gradients(dy, v, w, eps, ds=None):
    """(dv, tol), (dw, tol), (db, tol) before roundings to the results' types."""
    n, rows, h = v.shape
    g, gr = (h / 512 + 64) * E, (rows + 64) * E
    _, _, mean, rstd, xhat, ex = norm(v, w, torch.zeros_like(w), eps)
    q = dy * w
    c1, c2 = q.mean(-1, keepdim=True), (q * xhat).mean(-1, keepdim=True)
    e1 = g * q.abs().mean(-1, keepdim=True)
    e2 = g * (q * xhat).abs().mean(-1, keepdim=True) + (q.abs() * ex).mean(-1, keepdim=True)
    inner = q - c1 - xhat * c2
    dv = rstd * inner
    er = (ex / xhat.abs().clamp_min(1e-30)).clamp_max(1.0).amin(-1, keepdim=True) + g  # rstd's own share of ex, relative
    tol = rstd * (e1 + xhat.abs() * e2 + ex * c2.abs() + 8 * E * (q.abs() + c1.abs() + (xhat * c2).abs())) + dv.abs() * er
    if ds is not None:
        dv = dv + ds
        tol = tol + 2 * E * (dv.abs() + ds.abs())
    dw, tw = (dy * xhat).sum(1), (dy.abs() * ex).sum(1) + gr * (dy * xhat).abs().sum(1)
    return (dv, tol), (dw, tw), (dy.sum(1), gr * dy.abs().sum(1))


def adapter(x, base, a, b, scale, f):
    """t, y and y's tolerance before its rounding, for a 16-bit and a 32-bit result: in the former the products of t and B may be
    of operands cut to 16 bits each (2^-16 per operand and for the product of what was cut: below 2^-14 together)."""
    rank, h = a.shape[1:]
    g, gr = (h / 64 + 64) * E, (rank + 64) * E
    xd = masked(x, f)
    t = xd @ a.transpose(1, 2)
    et = g * (xd.abs() @ a.abs().transpose(1, 2))
    y = scale * (t @ b.transpose(1, 2))
    bt = b.abs().transpose(1, 2)
    tol = abs(scale) * (et @ bt + gr * (t.abs() @ bt))
    cut = abs(scale) * 2.0 ** -14 * (t.abs() @ bt)
    if base is not None:
        y = y + base
    tol = tol + 4 * E * (y.abs() + (0 if base is None else base.abs()))
    return t, y, tol, tol + cut


def adapter_gradients(dy, x, a, b, scale, f):
    """(dx, tol32, tol16), (dA, tol), (dB, tol)."""
    rank, h = a.shape[1:]
    rows, out = dy.shape[1:]
    gi, go, gr, gk = ((k / 64 + 64) * E for k in (h, out, rows * 64, rank * 64))
    xd = masked(x, f)
    dt = scale * (dy @ b)
    edt = abs(scale) * go * (dy.abs() @ b.abs())
    t = xd @ a.transpose(1, 2)
    et = gi * (xd.abs() @ a.abs().transpose(1, 2))
    da = dt.transpose(1, 2) @ xd
    ta = (edt + gr * dt.abs()).transpose(1, 2) @ xd.abs()
    db = scale * (dy.transpose(1, 2) @ t)
    tb = abs(scale) * (dy.abs().transpose(1, 2) @ (et + gr * t.abs()))
    dx = masked(dt @ a, f)
    full = dt.abs() @ a.abs()
    tx = masked(edt @ a.abs() + gk * full, f)
    return (dx, tx, tx + masked(2.0 ** -14 * full, f)), (da, ta), (db, tb)


def check(got, want, tol, what, u=None):
    """got, in its own type, is want to the tolerance and one rounding to that type."""
    u = U[got.dtype] if u is None else u
    g = d(got).reshape(want.shape)
    bad = ~((g - want).abs() <= tol * (1 + u) + u * want.abs() + TINY[got.dtype])
    both = (torch.isnan(g) & torch.isnan(want)) | (g == want)
    bad &= ~both
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError("%s: %d of %d values off, first at %s: %r, want %r, tolerance %r" % (
            what, int(bad.sum()), bad.numel(), at, float(g[tuple(at)]), float(want[tuple(at)]),
            float((tol * (1 + u) + u * want.abs())[tuple(at)])))
