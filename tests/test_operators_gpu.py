"""The operators on [n, ..., h] activations against their definitions in 64 bits, at sizes and layouts where they can go wrong."""
import pytest
import torch

import operators64 as R
from paper_2205_05632_b200.layers import dropout, dropout_add_layer_norm, layer_norm, low_rank_adapter

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, *shape, dtype=F32, sigma=1.0):
    return (sigma * torch.randn(*shape, generator=g, device="cuda")).to(dtype)


# (n, rows, h): one element, short and odd rows, the borders of spans of 256 and of the kernels' widths, beyond registers
SHAPES = [(1, 1, 1), (3, 5, 7), (2, 3, 8), (1, 17, 255), (2, 9, 256), (1, 4, 257), (5, 3, 520), (2, 7, 1001), (1, 33, 1024), (2, 2, 1032),
          (1, 3, 4096), (1, 2, 4104), (1, 2, 8191), (1, 2, 8200), (1, 2, 16384), (2, 2, 16392), (1, 1, 40001), (32, 1, 64), (1, 700, 48), (3, 3001, 64), (2, 45, 72), (1, 261, 128), (2, 19, 16),
          (1, 3, 4097), (1, 2, 6001)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", SHAPES)
def test_dropout(shape, dtype):
    g = gen(1)
    x = rand(g, *shape, dtype=dtype).requires_grad_()
    for p, seed, call, worker in ((0.1, 7, 0, 0), (0.5, (1 << 64) - 1, (1 << 32) - 1, (1 << 32) - 64), (0.0, 0, 1, 2), (1.0, 3, 1, 2), (2.0 ** -16, 5, 5, 5)):
        f = R.factor(*shape, p, seed, call, worker)
        y = dropout(x, p, seed=seed, call=call, worker=worker)
        R.check(y, R.d(x) * f, torch.zeros(()).double(), "y", u=R.U[dtype] + 2 * R.E)
        assert torch.equal(R.d(y) == 0, (f == 0) | (R.d(x) == 0))
        dy = rand(g, *shape, dtype=dtype)
        dx, = torch.autograd.grad(y, x, dy)
        R.check(dx, R.d(dy) * f, torch.zeros(()).double(), "dx", u=R.U[dtype] + 2 * R.E)
        assert torch.equal(dropout(x.detach(), p, seed=seed, call=call, worker=worker), y)


def test_dropout_zeroes_what_is_not_a_number_and_keeps_what_is_not_dropped():
    x = torch.full((2, 3, 40), float("nan"), device="cuda")
    x[:, 1] = float("inf")
    f = R.factor(2, 3, 40, 0.5, 11, 4)
    y = R.d(dropout(x, 0.5, seed=11, call=4))
    assert torch.equal(y == 0, f == 0)
    assert torch.isnan(y[:, 0][f[:, 0] != 0]).all() and torch.isinf(y[:, 1][f[:, 1] != 0]).all()
    assert torch.equal(R.d(dropout(x, 1.0)), torch.zeros(2, 3, 40).double())


def test_dropout_share_and_independence():
    x = torch.ones(4, 256, 1024, device="cuda")
    a, b, c = dropout(x, 0.3, seed=1), dropout(x, 0.3, seed=1, call=1), dropout(x, 0.3, seed=2)
    kept = [(t != 0) for t in (a, b, c)]
    n = x.numel()
    for k in kept:  # six standard deviations of a share
        assert abs(float(k.float().mean()) - 0.7) < 6 * (0.21 / n) ** 0.5
    for i in range(3):
        for j in range(i):
            assert abs(float((kept[i] & kept[j]).float().mean()) - 0.49) < 6 * (0.25 / n) ** 0.5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_layouts(dtype):
    g = gen(2)
    wide = rand(g, 3, 10, 96, dtype=dtype)
    cases = [wide[:, :, 3:67], wide[:, :, 8:72], wide[:, ::2, :64], wide.transpose(0, 1)[:, :, :40], wide[:, :1].expand(3, 10, 96),
             wide.transpose(1, 2), wide[:, 0], rand(g, 3, 2, 5, 24, dtype=dtype), rand(g, 3, 4, 2, 24, dtype=dtype).transpose(1, 2),
             wide[:1].expand(4, 10, 96), wide[:, :, :1]]
    for x in cases:
        y = dropout(x, 0.25, seed=9)
        v = R.flat(R.d(x))
        R.check(y, v * R.factor(*v.shape, 0.25, 9), torch.zeros(()).double(), str(x.stride()), u=R.U[dtype] + 2 * R.E)
        assert y.is_contiguous() and y.shape == x.shape


def test_a_worker_alone_draws_what_it_draws_in_the_batch():
    x = rand(gen(3), 5, 6, 100)
    y = dropout(x, 0.4, seed=8, call=3, worker=10)
    for i in range(5):
        assert torch.equal(dropout(x[i:i + 1], 0.4, seed=8, call=3, worker=10 + i), y[i:i + 1])


def test_call_on_the_device_and_in_a_graph():
    x = rand(gen(4), 2, 8, 136)
    res = rand(gen(5), 2, 8, 136)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            dropout(x, 0.3, seed=6, call=counter)
            dropout_add_layer_norm(x, res, p=0.3, seed=6, call=counter)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = dropout(x, 0.3, seed=6, call=counter)
            z, s = dropout_add_layer_norm(x, res, p=0.3, seed=6, call=counter)
            counter += 1
    torch.cuda.current_stream().wait_stream(stream)
    counter.fill_(5)
    for k in range(5, 8):
        graph.replay()
        assert torch.equal(y, dropout(x, 0.3, seed=6, call=k))
        zz, ss = dropout_add_layer_norm(x, res, p=0.3, seed=6, call=k)
        assert torch.equal(z, zz) and torch.equal(s, ss)
    counter.fill_((1 << 32) + 7)  # modulo 2^32
    assert torch.equal(dropout(x, 0.3, seed=6, call=counter), dropout(x, 0.3, seed=6, call=7))


def test_a_changed_call_is_found_in_the_backward_pass():
    for fn in (lambda x, c: dropout(x, 0.3, call=c), lambda x, c: dropout_add_layer_norm(x, x.detach(), p=0.3, call=c)[0],
               lambda x, c: low_rank_adapter(x, None, torch.ones(2, 16, device="cuda"), torch.ones(4, 2, device="cuda"), p=0.3, call=c)):
        x, c = rand(gen(), 2, 4, 16).requires_grad_(), torch.zeros(1, dtype=torch.int64, device="cuda")
        y = fn(x, c)
        c += 1
        with pytest.raises(RuntimeError):
            y.sum().backward()


# ---- layer norm ------------------------------------------------------------------------------------------------------------


def parameters(g, n, h, form):
    if form == "none":
        return None, None, torch.ones(1, 1, h).double(), torch.zeros(1, 1, h).double()
    w, b = 1 + 0.3 * rand(g, h), 0.3 * rand(g, h)
    if form == "apart":
        w, b = w.expand(n, h), b.expand(n, h)
    if form == "own":
        w, b = w + 0.1 * rand(g, n, h), b + 0.1 * rand(g, n, h)
    w, b = w.detach().requires_grad_(), b.detach().requires_grad_()
    wide = (lambda t: R.d(t).reshape(-1, 1, h).expand(n, 1, h))
    return w, b, wide(w), wide(b)


@pytest.mark.parametrize("form", ["apart", "shared", "own", "none"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", SHAPES + [(1, 0, 8), (0, 4, 8), (3, 600, 136), (2, 300, 1500)])
def test_layer_norm(shape, dtype, form):
    if form in ("own", "none") and shape not in SHAPES[:9]:
        pytest.skip("the same kernels")
    n, rows, h = shape
    g = gen(6)
    x = (rand(g, n, rows, h) * (1 + rand(g, h).abs()) + 0.5).to(dtype).requires_grad_()
    dy = rand(g, n, rows, h, dtype=dtype)
    w, b, w64, b64 = parameters(g, n, h, form)
    y = layer_norm(x, w, b, eps=1e-5)
    want, tol = R.norm(R.d(x), w64, b64, 1e-5)[:2]
    R.check(y, want, tol, "y")
    assert torch.equal(layer_norm(x.detach(), None if w is None else w.detach(), None if b is None else b.detach()), y)
    wanted = [t for t in (x, w, b) if t is not None]
    got = torch.autograd.grad(y, wanted, dy)
    (dx, tx), (dw, tw), (db, tb) = R.norm_gradients(R.d(dy), R.d(x), w64, 1e-5)
    R.check(got[0], dx, tx, "dx")
    if w is None:
        return
    if form == "shared":
        dw, tw, db, tb = dw.sum(0), tw.sum(0), db.sum(0), tb.sum(0)
    assert got[1].shape == w.shape and got[2].shape == b.shape
    R.check(got[1], dw, tw, "dweight")
    R.check(got[2], db, tb, "dbias")


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32)])
@pytest.mark.parametrize("shape", SHAPES + [(1, 0, 8), (3, 600, 136), (2, 40, 1500)])
def test_dropout_add_layer_norm(shape, types):
    n, rows, h = shape
    dtype, rtype = types
    g = gen(7)
    x, r = rand(g, n, rows, h, dtype=dtype).requires_grad_(), rand(g, n, rows, h, dtype=rtype, sigma=2.0).requires_grad_()
    dy, ds = rand(g, n, rows, h, dtype=dtype), rand(g, n, rows, h, dtype=rtype)
    w, b, w64, b64 = parameters(g, n, h, "apart")
    p, seed, call, worker = 0.2, 12345678901234567890, 77, 3
    y, s = dropout_add_layer_norm(x, r, w, b, p=p, eps=1e-6, seed=seed, call=call, worker=worker)
    f = R.factor(n, rows, h, p, seed, call, worker)
    s64 = R.d(r) + R.d(x) * f
    R.check(s, s64, 4 * R.E * (R.d(r).abs() + (R.d(x) * f).abs()), "s")
    assert s.dtype == rtype and y.dtype == dtype
    want, tol = R.norm(R.d(s), w64, b64, 1e-6)[:2]
    R.check(y, want, tol, "y")
    for ds_ in (ds, None):
        outs, seeds = ((y, s), (dy, ds_)) if ds_ is not None else ((y,), (dy,))
        got = torch.autograd.grad(outs, (x, r, w, b), seeds, retain_graph=True)
        (dv, tv), (dw, tw), (db, tb) = R.norm_gradients(R.d(dy), R.d(s), w64, 1e-6, None if ds_ is None else R.d(ds_))
        R.check(got[0], dv * f, tv * f + 2 * R.E * (dv * f).abs(), "dx")
        R.check(got[1], dv, tv, "dresidual")
        R.check(got[2], dw, tw, "dweight")
        R.check(got[3], db, tb, "dbias")
    only, = torch.autograd.grad(s, r, ds)
    R.check(only, R.d(ds), 4 * R.E * R.d(ds).abs(), "dresidual of s alone")


@pytest.mark.parametrize("h", [64, 128, 1000])
def test_norm_of_rows_far_from_zero_constant_rows_and_what_is_not_a_number(h):
    x = rand(gen(8), 1, 6, h) * 1e-2 + 1000.0
    x[0, 1] = 5.0
    x[0, 2, 17] = float("nan")
    x[0, 3, 18] = float("inf")
    y = layer_norm(x)
    want, tol = R.norm(R.d(x), torch.ones(1, 1, h).double(), torch.zeros(1, 1, h).double(), 1e-5)[:2]
    for j in (0, 1, 4, 5):
        R.check(y[:, j], want[:, j], tol[:, j], "row %d" % j)
    assert torch.isnan(y[0, 2]).all() and torch.isnan(y[0, 3]).all()


@pytest.mark.parametrize("h", [24, 33, 1400])
def test_norm_layouts(h):
    g = gen(9)
    n, rows = 3, 6
    wide = rand(g, n, rows, h + 16, dtype=BF16)
    for x, dy in ((wide[:, :, 8:8 + h], wide[:, :, 1:1 + h]), (rand(g, rows, n, h, dtype=BF16).transpose(0, 1), rand(g, n, rows, h, dtype=BF16)),
                  (rand(g, n, 1, h, dtype=BF16).expand(n, rows, h), rand(g, n, rows, 1, dtype=BF16).expand(n, rows, h)),
                  (rand(g, n, h, rows, dtype=BF16).transpose(1, 2), rand(g, 1, 1, h, dtype=BF16).expand(n, rows, h))):
        x = x.detach().requires_grad_()
        w, b, w64, b64 = parameters(g, n, h, "own")
        y = layer_norm(x, w, b)
        want, tol = R.norm(R.d(x), w64, b64, 1e-5)[:2]
        R.check(y, want, tol, "y")
        (dx, tx), (dw, tw), (db, tb) = R.norm_gradients(R.d(dy), R.d(x), w64, 1e-5)
        got = torch.autograd.grad(y, (x, w, b), dy)
        for q, v, t in zip(got, (dx, dw, db), (tx, tw, tb)):
            R.check(q, v, t, str(x.stride()))
    # a weight whose columns are not packed, [n, a, b, h], a single row per worker
    w = rand(g, h, 2)[:, 0]
    x = rand(g, n, 2, 3, h)
    want, tol = R.norm(R.flat(R.d(x)), R.d(w).expand(n, 1, h), torch.zeros(1, 1, h).double(), 1e-5)[:2]
    R.check(layer_norm(x, w), want, tol, "weight")
    want, tol = R.norm(R.d(x)[:, :1, 0], R.d(w).expand(n, 1, h), torch.zeros(1, 1, h).double(), 1e-5)[:2]
    R.check(layer_norm(x[:, 0, 0], w), want, tol, "2 axes")


def test_only_the_gradients_that_are_wanted():
    g = gen(10)
    n, rows, h = 2, 30, 264
    dy = rand(g, n, rows, h)
    w, b, w64, b64 = parameters(g, n, h, "apart")
    x = rand(g, n, rows, h)
    (dx, tx), (dw, tw), (db, tb) = R.norm_gradients(R.d(dy), R.d(x), w64, 1e-5)
    R.check(torch.autograd.grad(layer_norm(x, w, b.detach()), w, dy)[0], dw, tw, "dweight alone")
    R.check(torch.autograd.grad(layer_norm(x, w.detach(), b), b, dy)[0], db, tb, "dbias alone")
    v = x.requires_grad_()
    R.check(torch.autograd.grad(layer_norm(v, w.detach(), b.detach()), v, dy)[0], dx, tx, "dx alone")


def test_norm_gradients_against_differences():
    g = gen(11)
    n, rows, h = 2, 3, 40
    x, r, dy, ds = (rand(g, n, rows, h) for _ in range(4))
    w, b, _, _ = parameters(g, n, h, "own")

    def value(x, r, w, b):
        y, s = dropout_add_layer_norm(x, r, w, b, p=0.3, seed=4)
        return (y.double() * dy.double()).sum() + (s.double() * ds.double()).sum()

    leaves = [t.detach().requires_grad_() for t in (x, r, w, b)]
    grads = torch.autograd.grad(value(*leaves), leaves)
    for k, t in enumerate(leaves):
        along = rand(g, *t.shape)
        step = 2.0 ** -6
        hi, lo = ([q.detach() + (sign * step * along if i == k else 0) for i, q in enumerate(leaves)] for sign in (1, -1))
        slope = float((value(*hi) - value(*lo)) / (2 * step))
        want = float((grads[k].double() * along.double()).sum())
        # a central difference is off by step^2 / 6 of the third derivative along the direction, 2^-12 / 6 times a few tens here, and by
        # the values' fp32 noise over the step, sqrt(480) 2^-22 / 2^-6
        size = float((grads[k].double().abs() * along.double().abs()).sum())
        assert abs(slope - want) <= 2.0 ** -8 * size, (k, slope, want)


# ---- adapters --------------------------------------------------------------------------------------------------------------

ADAPTERS = [(1, 1, 1, 1, 1), (3, 5, 7, 9, 2), (2, 1, 64, 40, 8), (32, 1, 256, 264, 16), (2, 33, 100, 77, 3), (1, 70, 520, 1001, 12),
            (4, 16, 128, 128, 16), (2, 129, 264, 136, 17), (1, 200, 96, 1032, 64), (2, 40, 300, 200, 100), (1, 24, 2048, 64, 128),
            (3, 65, 192, 320, 32), (1, 1100, 64, 72, 4), (1, 5, 40, 33, 300), (2, 0, 8, 8, 4),
            (2, 300, 264, 136, 40), (1, 130, 1032, 520, 64), (3, 64, 72, 88, 33), (1, 1000, 256, 2048, 64), (2, 257, 200, 129, 48), (5, 512, 4096, 1024, 64)]


def adapter_case(g, n, rows, h, out, rank, dtype, form):
    many = n if form == "own" else 1
    a, b = rand(g, many, rank, h, sigma=h ** -0.5), rand(g, many, out, rank, sigma=rank ** -0.5)
    a64, b64 = R.d(a).expand(n, rank, h), R.d(b).expand(n, out, rank)
    if form == "apart":
        a, b = a.expand(n, rank, h), b.expand(n, out, rank)
    if form == "shared":
        a, b = a[0], b[0]
    x, base, dy = rand(g, n, rows, h, dtype=dtype), rand(g, n, rows, out, dtype=dtype), rand(g, n, rows, out, dtype=dtype)
    return [t.detach().requires_grad_() for t in (x, base, a, b)], dy, a64, b64


@pytest.mark.parametrize("form", ["apart", "own", "shared"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", ADAPTERS)
def test_low_rank_adapter(shape, dtype, form):
    n, rows, h, out, rank = shape
    for p in (0.0, 0.25):
        (x, base, a, b), dy, a64, b64 = adapter_case(gen(12), *shape, dtype, form)
        y = low_rank_adapter(x, base, a, b, scale=1.5, p=p, seed=21, call=2, worker=1)
        f = R.factor(n, rows, h, p, 21, 2, 1)
        _, want, tol, tol16 = R.adapter(R.d(x), R.d(base), a64, b64, 1.5, f)
        R.check(y, want, tol if dtype == F32 else tol16, "y")
        with torch.no_grad():
            assert torch.equal(low_rank_adapter(x, base, a, b, scale=1.5, p=p, seed=21, call=2, worker=1), y)
        dx, dbase, da, db = torch.autograd.grad(y, (x, base, a, b), dy)
        (wx, tx, tx16), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), a64, b64, 1.5, f)
        R.check(dx, wx, tx if dtype == F32 else tx16, "dx")
        assert torch.equal(dbase, dy) and da.shape == a.shape and db.shape == b.shape
        if form == "shared":
            wa, ta, wb, tb = wa.sum(0), ta.sum(0), wb.sum(0), tb.sum(0)
        R.check(da, wa, ta, "dA")
        R.check(db, wb, tb, "dB")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_adapter_without_a_base_and_with_few_gradients(dtype):
    (x, base, a, b), dy, a64, b64 = adapter_case(gen(13), 2, 40, 136, 72, 8, dtype, "apart")
    one = torch.zeros(2, 40, 136).double() + 1
    _, want, tol, tol16 = R.adapter(R.d(x), None, a64, b64, 0.5, one)
    y = low_rank_adapter(x, None, a, b, scale=0.5)
    R.check(y, want, tol if dtype == F32 else tol16, "y")
    (wx, tx, tx16), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), a64, b64, 0.5, one)
    R.check(torch.autograd.grad(low_rank_adapter(x, base, a.detach(), b.detach(), scale=0.5), x, dy)[0], wx, tx if dtype == F32 else tx16, "dx")
    R.check(torch.autograd.grad(low_rank_adapter(x.detach(), base.detach(), a, b.detach(), scale=0.5), a, dy)[0], wa, ta, "dA")
    R.check(torch.autograd.grad(low_rank_adapter(x.detach(), base.detach(), a.detach(), b, scale=0.5), b, dy)[0], wb, tb, "dB")
    got, = torch.autograd.grad(low_rank_adapter(x.detach(), base, a.detach(), b.detach(), scale=0.5), base, dy)
    assert torch.equal(got, dy)


@pytest.mark.parametrize("rows,rank", [(1, 8), (48, 8), (80, 8), (130, 40)])
def test_adapter_layouts(rows, rank):
    g = gen(14)
    n, h, out = 3, 64, 80
    (x, base, a, b), dy, a64, b64 = adapter_case(g, n, rows, h, out, rank, BF16, "own")
    one = torch.ones(n, rows, h).double()
    _, want, _, tol = R.adapter(R.d(x), R.d(base), a64, b64, 1.0, one)

    def padded(t, left, right):
        q = torch.zeros(*t.shape[:-1], t.shape[-1] + left + right, dtype=t.dtype, device="cuda")
        q[..., left:left + t.shape[-1]] = t.detach()
        return q[..., left:left + t.shape[-1]]

    for left, right in ((8, 8), (1, 0), (0, 3)):
        for which in range(4):
            args = [padded(t, left, right) if k == which else t.detach() for k, t in enumerate((x, base, a, b))]
            R.check(low_rank_adapter(*args), want, tol, "%d %d %d" % (which, left, right))
            args = [t.requires_grad_() for t in args]
            dx, da, db = torch.autograd.grad(low_rank_adapter(*args), [args[k] for k in (0, 2, 3)], padded(dy, left, right))
            (wx, _, tx), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), a64, b64, 1.0, one)
            R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")
    turned = [x.detach().transpose(0, 1).contiguous().transpose(0, 1), base.detach(), a.detach().transpose(1, 2).contiguous().transpose(1, 2),
              b.detach().transpose(1, 2).contiguous().transpose(1, 2)]
    R.check(low_rank_adapter(*turned), want, tol, "turned")
    # repeated workers and rows
    for v, z in ((x.detach()[:1].expand(n, rows, h), base.detach()), (x.detach()[:, :1].expand(n, rows, h), base.detach()[:, :1].expand(n, rows, out))):
        _, want, _, tol = R.adapter(R.d(v), R.d(z), a64, b64, 1.0, one)
        v, f, q = v.requires_grad_(), a.detach().requires_grad_(), b.detach().requires_grad_()
        y = low_rank_adapter(v, z, f, q)
        R.check(y, want, tol, "repeated")
        (wx, _, tx), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy[:, :1]).expand(n, rows, out), R.d(v), a64, b64, 1.0, one)
        dx, da, db = torch.autograd.grad(y, (v, f, q), dy[:, :1].expand(n, rows, out))
        R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")


def test_adapter_dropped_values_do_not_matter():
    (x, base, a, b), dy, _, _ = adapter_case(gen(15), 2, 40, 136, 72, 8, BF16, "apart")
    f = R.factor(2, 40, 136, 0.5, 3).cuda()
    with torch.no_grad():
        bad = torch.where(f == 0, torch.full_like(x, float("nan")), x)
    y = low_rank_adapter(x, base, a, b, p=0.5, seed=3)
    bad.requires_grad_()
    z = low_rank_adapter(bad, base, a, b, p=0.5, seed=3)
    assert torch.equal(y, z)
    for q, r in zip(torch.autograd.grad(y, (x, a, b), dy), torch.autograd.grad(z, (bad, a, b), dy)):
        assert torch.equal(q, r)


def test_adapter_rows_stay_to_themselves():
    """A row that holds an infinity or NaN leaves the other rows' results alone."""
    for dtype, rows in ((BF16, 40), (F32, 40), (F16, 1)):
        (x, base, a, b), _, a64, b64 = adapter_case(gen(16), 3, rows, 136, 72, 8, dtype, "apart")
        y = low_rank_adapter(x.detach(), base, a, b)
        v = x.detach().clone()
        v[1, -1, 5] = float("inf")
        v[2, 0, 100] = float("nan")
        z = low_rank_adapter(v, base, a, b)
        same = torch.ones(3, rows, dtype=torch.bool, device="cuda")
        same[1, -1] = same[2, 0] = False
        assert torch.equal(y[same], z[same])
        assert torch.isnan(z[2, 0]).all() and not torch.isfinite(z[1, -1]).any()


def test_adapter_values_of_any_size():
    """The fp32 operands are used in full: large, small and mixed magnitudes."""
    g = gen(17)
    n, rows, h, out, rank = 2, 40, 136, 72, 8
    for sx, sa, sb in ((1e18, 1e-18, 1.0), (1e-15, 1e15, 1e3), (1.0, 1e-12, 1e12)):
        (x, base, a, b), dy, a64, b64 = adapter_case(g, n, rows, h, out, rank, F32, "own")
        with torch.no_grad():
            x *= sx
            a *= sa
            b *= sb
        one = torch.ones(n, rows, h).double()
        y = low_rank_adapter(x, base, a, b)
        _, want, tol, _ = R.adapter(R.d(x), R.d(base), R.d(a), R.d(b), 1.0, one)
        R.check(y, want, tol, "y")
        dx, da, db = torch.autograd.grad(y, (x, a, b), dy)
        (wx, tx, _), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), R.d(a), R.d(b), 1.0, one)
        R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")


def test_no_wait_gave_up():
    import ctypes
    from paper_2205_05632_b200 import load_library
    low_rank_adapter(rand(gen(), 1, 128, 64, dtype=BF16), None, rand(gen(), 16, 64), rand(gen(), 64, 16))
    gave_up = ctypes.c_int32(-1)
    assert load_library().compams_adapter_status(ctypes.byref(gave_up)) == 0 and gave_up.value == 0


@pytest.mark.parametrize("rank", [16, 32, 64, 65, 144])
@pytest.mark.parametrize("rows", [63, 64, 65, 127, 128, 129, 255, 256, 257, 513])
def test_adapter_rows_around_the_tiles(rows, rank):
    n, h, out = 2, 136, 264
    (x, base, a, b), dy, a64, b64 = adapter_case(gen(21), n, rows, h, out, rank, BF16, "apart")
    y = low_rank_adapter(x, base, a, b, p=0.5, seed=2)
    f = R.factor(n, rows, h, 0.5, 2)
    _, want, _, tol = R.adapter(R.d(x), R.d(base), a64, b64, 1.0, f)
    R.check(y, want, tol, "y")
    dx, da, db = torch.autograd.grad(y, (x, a, b), dy)
    (wx, _, tx), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), a64, b64, 1.0, f)
    R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")


@pytest.mark.parametrize("h,out", [(8, 8), (56, 64), (64, 120), (72, 128), (120, 136), (128, 256), (136, 264), (1000, 65), (257, 1), (1, 129)])
def test_adapter_columns_around_the_tiles(h, out):
    for rank, rows in ((4, 70), (4, 134), (30, 70), (50, 70), (100, 70)):
        (x, base, a, b), dy, a64, b64 = adapter_case(gen(22), 2, rows, h, out, rank, BF16, "own")
        y = low_rank_adapter(x, base, a, b, p=0.25, seed=2)
        f = R.factor(2, rows, h, 0.25, 2)
        _, want, _, tol = R.adapter(R.d(x), R.d(base), a64, b64, 1.0, f)
        R.check(y, want, tol, "y")
        dx, da, db = torch.autograd.grad(y, (x, a, b), dy)
        (wx, _, tx), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), a64, b64, 1.0, f)
        R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")


@pytest.mark.parametrize("rank", [16, 32, 64, 130])
@pytest.mark.parametrize("h,out", [(1288, 1304), (1301, 1288)])
def test_adapter_several_tiles_to_a_block(h, out, rank):
    n, rows = 8, 400
    (x, base, a, b), dy, a64, b64 = adapter_case(gen(23), n, rows, h, out, rank, BF16, "own")
    f = R.factor(n, rows, h, 0.25, 9)
    y = low_rank_adapter(x, base, a, b, scale=0.5, p=0.25, seed=9)
    _, want, _, tol = R.adapter(R.d(x), R.d(base), a64, b64, 0.5, f)
    R.check(y, want, tol, "y")
    dx, da, db = torch.autograd.grad(y, (x, a, b), dy)
    (wx, _, tx), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy), R.d(x), a64, b64, 0.5, f)
    R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")


# ---- together --------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_results_do_not_change_from_run_to_run_and_streams_are_kept(dtype):
    g = gen(18)
    (x, base, a, b), dy, _, _ = adapter_case(g, 4, 100, 520, 264, 16, dtype, "apart")
    w, bias, _, _ = parameters(g, 4, 264, "apart")

    def once():
        z = low_rank_adapter(x, base, a, b, p=0.1, seed=1)
        y, s = dropout_add_layer_norm(z, base.detach(), w, bias, p=0.1, seed=1, call=1)
        return [y, s, *torch.autograd.grad((y, s), (x, a, b, w, bias), (dy, dy))]

    first = once()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [once() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for other in again:
        assert all(torch.equal(p, q) for p, q in zip(first, other))


@pytest.mark.parametrize("rows", [3, 50, 200])
def test_forward_and_backward_in_a_graph(rows):
    g = gen(19)
    (x, base, a, b), dy, _, _ = adapter_case(g, 2, rows, 136, 72, 8, BF16, "apart")
    w, bias, _, _ = parameters(g, 2, 72, "apart")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")

    def once(call):
        leaves = [t.detach().requires_grad_() for t in (x, a, b, w, bias)]
        z = low_rank_adapter(leaves[0], base.detach(), leaves[1], leaves[2], p=0.1, seed=1, call=call)
        y, s = dropout_add_layer_norm(z, base.detach(), leaves[3], leaves[4], p=0.1, seed=2, call=call)
        return [y.detach(), s.detach(), *torch.autograd.grad((y, s), leaves, (dy, dy))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            once(counter)
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        outs = []
        for graph in graphs:
            with torch.cuda.graph(graph, stream=side):
                outs.append(once(counter))
    torch.cuda.current_stream().wait_stream(side)
    for k in (3, 4):
        counter.fill_(k)
        for graph in graphs:
            graph.replay()
        want = once(k)
        for out in outs:
            assert all(torch.equal(p, q) for p, q in zip(want, out))


def test_fine_tuning_with_all_workers_in_one_batch():
    """Norms and adapters trained by COMP-AMS: the rows of G from one pass over all workers are those of the workers run one after
    the other, and the optimizer's steps on them are the same."""
    from paper_2205_05632_b200 import TOPK
    from paper_2205_05632_b200.optim import CompAMSOptimizer
    n, rows, h, rank = 4, 24, 96, 8

    def model():
        torch.manual_seed(5)
        params = [torch.ones(h), torch.zeros(h), torch.randn(rank, h) * h ** -0.5, torch.randn(h, rank) * 0.1, torch.ones(h), torch.zeros(h)]
        return [torch.nn.Parameter(p.cuda()) for p in params]

    g = gen(20)
    x, proj = rand(g, n, rows, h), rand(g, h, h, sigma=h ** -0.5)
    target = rand(g, n, rows, h)

    def loss(x, target, w, b, A, B, w2, b2, t, worker):
        u = layer_norm(x, w, b)
        z = low_rank_adapter(u, u @ proj, A, B, scale=2.0, p=0.1, seed=9, call=2 * t, worker=worker)
        y, s = dropout_add_layer_norm(z, x, w2, b2, p=0.1, seed=9, call=2 * t + 1, worker=worker)
        return ((y + s - target) ** 2).mean((1, 2)).sum()

    together, alone = model(), model()
    opts = [CompAMSOptimizer(m, n, TOPK, 0.05, lr=1e-2) for m in (together, alone)]
    leaves = opts[0].worker_parameters()
    assert leaves is opts[0].worker_parameters() and all(w.data_ptr() == p.data_ptr() for w, p in zip(leaves, together))
    for t in range(4):
        loss(x, target, *leaves, t, 0).backward()
        opts[0].collect_all()
        assert all(w.grad is None for w in leaves)
        for i in range(n):
            loss(x[i:i + 1], target[i:i + 1], *alone, t, i).backward()
            opts[1].collect(i)
        scale = opts[1].G.abs().amax()
        # the same sums in another order: fp32 sums over at most 96 rows and columns, several in a row, on values of the gradient's size
        assert float((opts[0].G - opts[1].G).abs().max()) <= 2.0 ** -14 * float(scale), t
        opts[1].G.copy_(opts[0].G)
        for o in opts:
            o.step()
        assert torch.equal(opts[0].theta, opts[1].theta)
    # a parameter without a gradient gives zeros
    leaves[0].grad = torch.ones(n, h, device="cuda")
    opts[0].collect_all()
    assert torch.equal(opts[0].G[:, :h], torch.ones(n, h, device="cuda")) and not opts[0].G[:, h:].any()
    for o in opts:
        o.close()
