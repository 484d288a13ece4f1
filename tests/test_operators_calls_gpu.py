"""Calls that the documentation allows and that are easily forgotten: few axes and many, the largest numbers of workers and ranks, the same
tensor twice, everything dropped, two streams at once, another shape behind a trace of streams."""
import pytest
import torch

import operators64 as R
from paper_2205_05632_b200 import CompAMSError
from paper_2205_05632_b200.layers import dropout, dropout_add_layer_norm, layer_norm, low_rank_adapter

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def rand(g, *shape, dtype=F32, sigma=1.0):
    return (sigma * torch.randn(*shape, generator=g, device="cuda")).to(dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def adapter(x, base, a, b, dy, p=0.0, seed=0, scale=1.0):
    """The operator with all its gradients against 64 bits; x [n, rows, h] for the reference whatever its axes."""
    n, (rank, out) = x.shape[0], (a.shape[-2], b.shape[-2])
    v = R.flat(R.d(x)) if x.dim() > 2 else R.d(x)[:, None]
    rows, h = v.shape[1:]
    f = R.factor(n, rows, h, p, seed)
    a64, b64 = R.d(a).expand(n, rank, h), R.d(b).expand(n, out, rank)
    leaves = [t.detach().requires_grad_() for t in (x, a, b)]
    y = low_rank_adapter(leaves[0], base, leaves[1], leaves[2], scale=scale, p=p, seed=seed)
    z = None if base is None else R.d(base).reshape(n, rows, out)
    _, want, tol, _ = R.adapter(v, z, a64, b64, scale, f)
    R.check(y, want, tol, "y")
    assert y.shape == (*x.shape[:-1], out)
    dx, da, db = torch.autograd.grad(y, leaves, dy)
    (wx, tx, _), (wa, ta), (wb, tb) = R.adapter_gradients(R.d(dy).reshape(n, rows, out), v, a64, b64, scale, f)
    if a.dim() == 2:
        wa, ta, wb, tb = wa.sum(0), ta.sum(0), wb.sum(0), tb.sum(0)
    R.check(dx, wx, tx, "dx"), R.check(da, wa, ta, "dA"), R.check(db, wb, tb, "dB")
    assert dx.shape == x.shape


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("axes", [(9,), (3, 24), (2, 5, 13), (3, 2, 40)])
def test_adapters_of_two_to_five_axes(axes, dtype):
    g = gen(1)
    x, base, dy = rand(g, 4, *axes, 72, dtype=dtype), rand(g, 4, *axes, 40, dtype=dtype), rand(g, 4, *axes, 40, dtype=dtype)
    a, b = rand(g, 4, 8, 72, sigma=0.1), rand(g, 4, 40, 8, sigma=0.3)
    adapter(x, base, a, b, dy, p=0.25, seed=3)
    adapter(x[:, 0], base[:, 0], a, b, dy[:, 0])  # an axis less: rows that are not packed
    adapter(x.transpose(0, 1).contiguous().transpose(0, 1), None, a[0], b[0], dy)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,rows,h,out,rank", [(65535, 1, 8, 8, 1), (20000, 5, 8, 16, 2), (1, 70, 8, 8, 1024), (2, 3, 40, 24, 1024), (1, 200, 136, 72, 1024),
                                               (2, 20, 300, 9, 500), (1, 3000, 1, 1, 3)])
def test_adapters_at_the_ends_of_the_range(n, rows, h, out, rank, dtype):
    g = gen(2)
    x, base, dy = rand(g, n, rows, h, dtype=dtype), rand(g, n, rows, out, dtype=dtype), rand(g, n, rows, out, dtype=dtype)
    adapter(x, base, rand(g, rank, h, sigma=h ** -0.5), rand(g, out, rank, sigma=rank ** -0.5), dy, p=0.5, seed=1)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_the_largest_number_of_workers(dtype):
    g = gen(3)
    n, h = 65535, 24
    x, dy = rand(g, n, 1, h, dtype=dtype), rand(g, n, 1, h, dtype=dtype)
    w, b = 1 + rand(g, h, sigma=0.2), rand(g, h)
    leaves = [t.detach().requires_grad_() for t in (x, w, b)]
    y, s = dropout_add_layer_norm(leaves[0], x, leaves[1], leaves[2], p=0.5, seed=4)
    f = R.factor(n, 1, h, 0.5, 4)
    R.check(s, R.d(x) + R.d(x) * f, 4 * R.E * (R.d(x).abs() * (1 + f)), "s")
    w64, b64 = R.d(w).expand(n, 1, h), R.d(b).expand(n, 1, h)
    want, tol = R.norm(R.d(s), w64, b64, 1e-5)[:2]
    R.check(y, want, tol, "y")
    got = torch.autograd.grad(y, leaves, dy)
    (dv, tv), (dw, tw), (db, tb) = R.norm_gradients(R.d(dy), R.d(s), w64, 1e-5)
    R.check(got[0], dv * f, tv * f + 2 * R.E * (dv * f).abs(), "dx")
    # (n rows of a column, one after another in the worst order)
    R.check(got[1], dw.sum(0), tw.sum(0), "dweight"), R.check(got[2], db.sum(0), tb.sum(0), "dbias")
    for call in (lambda t: dropout(t, 0.5), layer_norm, lambda t: low_rank_adapter(t, None, rand(g, 2, h), rand(g, 8, 2))):
        with pytest.raises(CompAMSError):
            call(torch.zeros(65536, h, dtype=dtype, device="cuda"))


def test_the_same_tensor_twice():
    g = gen(5)
    n, rows, h = 2, 70, 136
    x = rand(g, n, rows, h).requires_grad_()
    y, s = dropout_add_layer_norm(x, x, p=0.0)  # s = 2 x
    assert torch.equal(s, 2 * x)
    dy = rand(g, n, rows, h)
    one = torch.ones(1, 1, h).double()
    (dv, tv), _, _ = R.norm_gradients(R.d(dy), R.d(s), one, 1e-5)
    dx, = torch.autograd.grad(y, x, dy)
    R.check(dx, 2 * dv, 2 * tv + 4 * R.E * dv.abs(), "dx")
    a = rand(g, n, 8, h, sigma=0.1)
    z = low_rank_adapter(x, x, a, a.transpose(1, 2))  # base and x, A and B of one tensor
    _, want, tol, _ = R.adapter(R.d(x), R.d(x), R.d(a), R.d(a).transpose(1, 2), 1.0, torch.ones(n, rows, h).double())
    R.check(z, want, tol, "y")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [2, 40, 200])
def test_everything_dropped(rows, dtype):
    g = gen(6)
    x, base, dy = rand(g, 2, rows, 136, dtype=dtype).requires_grad_(), rand(g, 2, rows, 72, dtype=dtype), rand(g, 2, rows, 72, dtype=dtype)
    a, b = rand(g, 2, 8, 136).requires_grad_(), rand(g, 2, 72, 8).requires_grad_()
    y = low_rank_adapter(x, base, a, b, p=1.0)
    assert torch.equal(y, base)
    for t in torch.autograd.grad(y, (x, a, b), dy):
        assert not t.any()
    r = rand(g, 2, rows, 136, dtype=dtype)
    z, s = dropout_add_layer_norm(x, r, p=1.0)
    assert torch.equal(s, r) and torch.equal(z, layer_norm(r))
    assert not torch.autograd.grad(z, x, torch.ones_like(z))[0].any()


def test_two_streams_at_once():
    g = gen(7)
    shapes = [(4, 600, 1032, 520, 64), (8, 300, 520, 1032, 16), (2, 900, 264, 264, 130), (4, 30, 520, 264, 8)]
    cases = []
    for dtype in (BF16, BF16, F16):
        for n, rows, h, out, rank in shapes:
            cases.append([rand(g, n, rows, h, dtype=dtype).requires_grad_(), rand(g, n, rows, out, dtype=dtype), rand(g, n, rank, h).requires_grad_(),
                          rand(g, n, out, rank).requires_grad_(), rand(g, n, rows, out, dtype=dtype)])

    def once(x, base, a, b, dy):
        y = low_rank_adapter(x, base, a, b, p=0.1, seed=8)
        z, s = dropout_add_layer_norm(y, base, p=0.1, seed=9)
        return [z.detach(), s.detach(), *torch.autograd.grad((z, s), (x, a, b), (dy, dy))]

    alone = [once(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for turn in range(4):
        for k, c in enumerate(cases):
            with torch.cuda.stream(streams[(k + turn) % 3]):
                got.append((k, once(*c)))
    torch.cuda.synchronize()
    for k, outs in got:
        assert all(torch.equal(p, q) for p, q in zip(outs, alone[k]))


@pytest.mark.parametrize("rows", [95, 96, 100, 127, 129])
@pytest.mark.parametrize("h,out", [(8, 8), (56, 64), (64, 120), (72, 128), (120, 136), (128, 256), (136, 264), (1000, 65), (257, 1), (1, 129)])
def test_columns_around_the_tiles_at_ranks_of_17_to_32(h, out, rows):
    g = gen(9)
    x, base, dy = rand(g, 2, rows, h, dtype=BF16), rand(g, 2, rows, out, dtype=BF16), rand(g, 2, rows, out, dtype=BF16)
    adapter(x, base, rand(g, 2, 30, h, sigma=h ** -0.5), rand(g, 2, out, 30, sigma=0.2), dy, p=0.25, seed=2)
