"""rms_norm and gated_add_rms_norm against 64 bits: types, widths around the rows' forms, strides, parameters given or not, rounding of the
residual stream, refusals on the device, graphs, streams."""
import pytest
import torch

import blocks64 as B
from paper_2205_05632_b200.layers import gated_add_rms_norm, rms_norm

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, F32)]
EPS = 1e-6


def rand(g, *shape, dtype=F32, sigma=1.0):
    return (sigma * torch.randn(*shape, generator=g, device="cuda")).to(dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def wide(p, n, h):
    """[n, 1, h] in 64 bits, or 1."""
    return 1.0 if p is None else p.detach().double().expand(n, h)[:, None] if p.dim() == 2 else p.detach().double().expand(n, h)[:, None]


def rows_of(t):
    return t.detach().double().reshape(t.shape[0], -1, t.shape[-1])


def parameter_check(got, p, want, tol, what):
    """want [n, h]; a parameter for all workers has the sum."""
    if p is None:
        return
    if p.dim() == 1:
        tol = tol.sum(0) + (want.shape[0] * B.E) * want.abs().sum(0)
        want = want.sum(0)
    B.check(got, want, tol, what)


def plain(x, w, dy, eps=EPS):
    leaves = [t.detach().requires_grad_() if t is not None else None for t in (x, w)]
    y = rms_norm(leaves[0], leaves[1], eps)
    n, h = x.shape[0], x.shape[-1]
    w64 = wide(w, n, h)
    want, tol = B.rms(rows_of(x), w64, eps)
    assert y.dtype == x.dtype and y.shape == x.shape
    B.check(y.reshape(want.shape), want, tol, "y")
    with torch.no_grad():
        assert torch.equal(rms_norm(x, w, eps), y)
    got = torch.autograd.grad(y, [t for t in leaves if t is not None], dy)
    wx, tx, ww, tw = B.rms_gradients(rows_of(dy), torch.zeros((), device="cuda", dtype=torch.float64), rows_of(x), w64, eps)
    B.check(got[0].reshape(wx.shape), wx, tx, "dx")
    if w is not None:
        parameter_check(got[1], w, ww, tw, "dweight")
    return y, got


def gated(x, residual, w, g, v, dy, ds, alpha=0.9, eps=EPS):
    leaves = [t.detach().requires_grad_() if t is not None else None for t in (x, residual, w, g, v)]
    y, s = gated_add_rms_norm(*leaves, residual_scale=alpha, eps=eps)
    n, h = x.shape[0], x.shape[-1]
    w64, g64, v64 = (wide(p, n, h) for p in (w, g, v))
    want, tol = B.gated(rows_of(x), rows_of(residual), w64, g64, alpha, eps)
    assert y.dtype == x.dtype and s.dtype == residual.dtype and y.shape == s.shape == x.shape
    kept = rows_of(s)
    if s.dtype == F32:
        B.check(s.reshape(want.shape), want, tol, "s")
    else:
        # the exact value, rounded to fp32 and then to the type, but for one in a million, which is the neighbour
        off = kept != want.float().to(s.dtype).double()
        assert int(off.sum()) <= 1e-6 * off.numel() + 1
        B.check(s.reshape(want.shape), want, 2.0 ** -40 * want.abs() + tol * off, "s")
    wy, ty = B.rms(kept, v64, eps)  # of s as it is kept
    B.check(y.reshape(wy.shape), wy, ty, "y")
    with torch.no_grad():
        again = gated_add_rms_norm(x, residual, w, g, v, alpha, eps)
        assert torch.equal(again[0], y) and torch.equal(again[1], s)
    outs, grads = ((y, s), (dy, ds)) if dy is not None and ds is not None else ((y,), (dy,)) if ds is None else ((s,), (ds,))
    got = torch.autograd.grad(outs, [t for t in leaves if t is not None], grads, allow_unused=True)
    zero = torch.zeros((), device="cuda", dtype=torch.float64)
    dy64 = rows_of(dy) if dy is not None else torch.zeros_like(kept)
    ds64 = rows_of(ds) if ds is not None else torch.zeros_like(kept)
    gs, ts, wv, tv = B.rms_gradients(dy64, zero, kept, v64, eps)
    gs, ts = gs + ds64, ts + B.E * (gs + ds64).abs()
    u = lambda t: t.abs() if torch.is_tensor(t) else t  # noqa: E731
    wx, tx, ww, tw = B.rms_gradients(gs * g64, ts * u(g64) + B.E * (gs * g64).abs(), rows_of(x), w64, eps)
    normed = rows_of(x) * B._r(rows_of(x), eps) * w64
    wg = (gs * normed).sum(1)
    tg = (ts * normed.abs() + ((h / 512 + 64) + x.shape[1] / 4 + 64) * 2 * B.E * (gs * normed).abs()).sum(1)
    found = iter(got)
    B.check(next(found).reshape(wx.shape), wx, tx, "dx")
    B.check(next(found).reshape(gs.shape), alpha * gs, abs(alpha) * ts + 2 * B.E * (alpha * gs).abs(), "dresidual")
    for p, a, b, what in ((w, ww, tw, "dweight"), (g, wg, tg, "dgate"), (v, wv, tv, "dnext")):
        if p is not None:
            parameter_check(next(found), p, a, b, what)
    return y, s, got


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("n,rows,h", [(1, 1, 1), (2, 3, 8), (3, 70, 57), (2, 33, 64), (2, 9, 72), (2, 40, 128), (1, 600, 136), (3, 5, 256), (2, 17, 264),
                                      (2, 12, 1000), (1, 7, 1001), (2, 90, 2048), (2, 6, 4096), (1, 3, 4097), (2, 5, 4104), (1, 4, 8192), (1, 5, 8193),
                                      (2, 3, 20000)])
def test_against_64_bits(n, rows, h, kinds):
    g = gen(rows + h)
    x, res = rand(g, n, rows, h, dtype=kinds[0]), rand(g, n, rows, h, dtype=kinds[1], sigma=2.0)
    dy, ds = rand(g, n, rows, h, dtype=kinds[0]), rand(g, n, rows, h, dtype=kinds[1])
    w, gate, v = (1.0 + 0.3 * rand(g, n, h) for _ in range(3))
    gated(x, res, w, gate, v, dy, ds)
    gated(x, res, w[0], gate[0], v[0], dy, ds)
    if kinds[0] == kinds[1]:
        plain(x, w, dy)
        plain(x, w[0], dy)
        plain(x, None, dy)


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("given", [(0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1)])
@pytest.mark.parametrize("h", [64, 333, 9000])
def test_parameters_given_or_not(h, given, kinds):
    g = gen(h)
    x, res = rand(g, 2, 11, h, dtype=kinds[0]), rand(g, 2, 11, h, dtype=kinds[1])
    dy, ds = rand(g, 2, 11, h, dtype=kinds[0]), rand(g, 2, 11, h, dtype=kinds[1])
    p = [1.0 + 0.3 * rand(g, 2, h) if there else None for there in given]
    gated(x, res, *p, dy, ds, alpha=1.0)
    gated(x, res, *p, dy, None, alpha=-0.5)
    if not given[2]:
        gated(x, res, *p, None, ds, alpha=0.0)


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("h", [40, 512, 8200])
def test_strides_and_axes(h, kinds):
    g = gen(3)
    x, res = rand(g, 3, 12, 2 * h + 8, dtype=kinds[0]), rand(g, 3, 12, 2 * h + 8, dtype=kinds[1])
    dy, ds = rand(g, 3, 12, 2 * h + 8, dtype=kinds[0]), rand(g, 3, 12, 2 * h + 8, dtype=kinds[1])
    w, gate, v = (1.0 + 0.3 * rand(g, 3, h) for _ in range(3))
    for cut in (lambda t: t[..., :h], lambda t: t[..., 1:h + 1], lambda t: t[:, ::3, :h], lambda t: t[:, 0, :h], lambda t: t[..., :h].reshape(3, 2, 6, h),
                lambda t: t[..., :h].transpose(1, 2).contiguous().transpose(1, 2), lambda t: t[:, :1, :h].expand(3, 5, h)):
        gated(cut(x), cut(res), w, gate, v, cut(dy), cut(ds))
        if kinds[0] == kinds[1]:
            plain(cut(x), w, cut(dy))
    few = [p.expand(3, h) for p in (w[:1], gate[:1], v[:1])]  # one parameter seen by all
    gated(x[..., :h], res[..., :h], *few, dy[..., :h], ds[..., :h])
    odd = [rand(g, 3, h + 1)[:, 1:] for _ in range(3)]  # parameters off 16-byte boundaries
    gated(x[..., :h], res[..., :h], *odd, dy[..., :h], ds[..., :h])


@pytest.mark.parametrize("kind", [BF16, F16])
def test_the_stream_is_rounded_as_the_exact_sum(kind):
    # sums that cancel, gates far apart, a scale that fp32 does not hold
    g = gen(4)
    x = rand(g, 4, 300, 2048, dtype=kind)
    gate = rand(g, 4, 2048) * 10.0 ** (4 * torch.rand(4, 2048, generator=g, device="cuda") - 3)
    w = 1.0 + 0.3 * rand(g, 4, 2048)
    u = B.rms(rows_of(x), wide(w, 4, 2048), EPS)[0] * wide(gate, 4, 2048)
    res = (-u / 0.7 * (1.0 + 0.01 * torch.randn(u.shape, generator=g, device="cuda"))).to(kind)
    _, s = gated_add_rms_norm(x, res, w, gate, None, residual_scale=0.7)
    want = 0.7 * rows_of(res) + u
    off = (rows_of(s) != want.float().to(kind).double()) & (want.abs() > B.TINY[F16] * 2 ** 14)  # (below, fp16 has fewer bits than the kernel's test assumes)
    assert int(off.sum()) <= 2 + 1e-6 * off.numel()


def test_values_that_are_not_finite_stay_in_their_rows():
    g = gen(5)
    for h in (100, 4096, 9000):
        x, res = rand(g, 2, 9, h, dtype=BF16), rand(g, 2, 9, h, dtype=BF16)
        y0, s0 = gated_add_rms_norm(x, res)
        p0 = rms_norm(x)
        x[1, 4, 7] = float("nan")
        y, s = gated_add_rms_norm(x, res)
        keep = torch.ones(2, 9, dtype=torch.bool, device="cuda")
        keep[1, 4] = False
        assert torch.isnan(y[1, 4]).all() and torch.equal(y[keep], y0[keep]) and torch.equal(s[keep], s0[keep])
        assert torch.isnan(rms_norm(x)[1, 4]).all() and torch.equal(rms_norm(x)[keep], p0[keep])
        x[1, 4] = 0.0
        assert not rms_norm(x)[1, 4].any()  # a row of zeros


def test_no_rows():
    x = torch.zeros(2, 0, 16, device="cuda", requires_grad=True)
    w = torch.ones(2, 16, device="cuda", requires_grad=True)
    dx, dw = torch.autograd.grad(rms_norm(x, w).sum(), (x, w))
    assert dx.shape == x.shape and not dw.any()
    y, s = gated_add_rms_norm(x, x, w, w, w)
    dx, dw = torch.autograd.grad((y.sum() + s.sum()), (x, w))
    assert y.shape == s.shape == x.shape and not dw.any()


@pytest.mark.parametrize("h", [96, 97])
def test_some_gradients_alone_are_the_same(h):
    g = gen(9)
    values = [rand(g, 3, 10, h, dtype=BF16), rand(g, 3, 10, h)] + [1 + 0.2 * rand(g, 3, h) for _ in range(3)]
    dy, ds = rand(g, 3, 10, h, dtype=BF16), rand(g, 3, 10, h)

    def gradients(wanted, given=(1, 1, 1, 1, 1)):
        leaves = [(v.clone().requires_grad_() if k in wanted else v) if given[k] else None for k, v in enumerate(values)]
        out = gated_add_rms_norm(*leaves)
        return torch.autograd.grad(out, [leaves[k] for k in wanted], (dy, ds))

    everything = gradients((0, 1, 2, 3, 4))
    for wanted in ((0,), (1,), (2,), (3,), (4,), (0, 4), (1, 3), (2, 3)):
        assert all(torch.equal(a, everything[k]) for a, k in zip(gradients(wanted), wanted))
    without = gradients((0, 1, 3), (1, 1, 0, 1, 1))  # a parameter that is not given in front of one that is
    assert all(torch.equal(a, b) for a, b in zip(gradients((3,), (1, 1, 0, 1, 1)), without[2:]))
    x, w = values[0].clone().requires_grad_(), values[2].clone().requires_grad_()
    dx, dw = torch.autograd.grad(rms_norm(x, w), (x, w), dy)
    assert torch.equal(torch.autograd.grad(rms_norm(x, values[2]), x, dy)[0], dx)
    assert torch.equal(torch.autograd.grad(rms_norm(values[0], w), w, dy)[0], dw)


def test_the_same_tensor_everywhere():
    g = gen(6)
    x, w = rand(g, 2, 6, 96).requires_grad_(), (1 + 0.2 * rand(g, 2, 96)).requires_grad_()
    y, s = gated_add_rms_norm(x, x, w, w, w, 0.5)
    dx, dw = torch.autograd.grad((y * y).sum() + s.sum(), (x, w))
    x64, w64 = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()

    def f(v):
        return v / (v.square().mean(-1, keepdim=True) + EPS).sqrt() * w64[:, None]

    s64 = 0.5 * x64 + w64[:, None] * f(x64)
    wx, ww = torch.autograd.grad((f(s64) ** 2).sum() + s64.sum(), (x64, w64))
    B.near(dx, wx, 1e-6, "dx"), B.near(dw, ww, 1e-6, "dw")


def test_captured_and_on_two_streams():
    g = gen(7)
    x, res = rand(g, 3, 50, 264, dtype=BF16).requires_grad_(), rand(g, 3, 50, 264).requires_grad_()
    w = [(1 + 0.2 * rand(g, 3, 264)).requires_grad_() for _ in range(3)]
    dy, ds = rand(g, 3, 50, 264, dtype=BF16), rand(g, 3, 50, 264)

    def both(*t):
        y, s = gated_add_rms_norm(*t)
        return (y.detach(), s.detach(), *torch.autograd.grad((y, s), t, (dy, ds)))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            both(x, res, *w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = both(x, res, *w)
    torch.cuda.current_stream().wait_stream(side)
    with torch.no_grad():
        x.copy_(rand(g, 3, 50, 264))
    graph.replay()
    torch.cuda.synchronize()
    fresh = [t.detach().clone().requires_grad_() for t in (x, res, *w)]
    want = both(*fresh)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    many = []
    for _ in range(6):
        for s in streams:
            with torch.cuda.stream(s):
                many.append(both(*[t.detach().requires_grad_() for t in fresh]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for m in many for a, b in zip(m, want))


@pytest.mark.parametrize("n,rows,h", [(65535, 1, 8), (1, 70000, 16), (3, 300000, 1)])
def test_many_rows_and_workers(n, rows, h):
    g = gen(8)
    x, res = rand(g, n, rows, h, dtype=BF16), rand(g, n, rows, h)
    gated(x, res, *(1.0 + 0.3 * rand(g, n, h) for _ in range(3)), rand(g, n, rows, h, dtype=BF16), rand(g, n, rows, h))
