"""linear_cross_entropy against 64 bits: types, forms of the weight, reductions, ragged sizes, strides, masks, far places, streams, graphs."""
import ctypes

import pytest
import torch

import blocks64 as B
from paper_2205_05632_b200 import load_library
from paper_2205_05632_b200.layers import linear_cross_entropy

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(BF16, BF16), (F16, F16), (F32, F32), (BF16, F32), (F16, F32)]


def inputs(seed, n, rows, h, vocab, kind, wkind, form, ignored=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, rows, h, generator=g, device="cuda").to(kind)
    many = (n,) if form == "own" else ()
    w = (2.0 * h ** -0.5 * torch.randn(*many, vocab, h, generator=g, device="cuda")).to(wkind)
    w = w.expand(n, vocab, h) if form == "apart" else w
    t = torch.randint(0, vocab, (n, rows), generator=g, device="cuda")
    t[torch.rand(n, rows, generator=g, device="cuda") < ignored] = -100
    return x, w, t, g


def verify(x, w, t, reduction, dloss, xs=None, ignored=-100, lengths=True):
    """Everything of a call against 64 bits; xs: x as [n, rows, h]; lengths: the gradients as a whole too."""
    leaf, wleaf = x.detach().requires_grad_(), w.detach().requires_grad_()
    loss = linear_cross_entropy(leaf, wleaf, t, reduction, ignored)
    dx, dw = torch.autograd.grad(loss, (leaf, wleaf), dloss)
    assert loss.dtype == F32 and dx.dtype == x.dtype and dw.dtype == w.dtype and dx.shape == x.shape and dw.shape == w.shape
    v = x.reshape(x.shape[0], -1, x.shape[-1]) if xs is None else xs
    want, tol, wx, tx, ww, tw = B.head(v, w, t, reduction, ignored, dloss)
    B.check(loss, want, tol, "loss")
    B.check(dx.reshape(v.shape), wx, tx, "dx")
    B.check(dw, ww, tw, "dweight")
    if lengths and torch.isfinite(ww).all():
        for got, exact, kind in ((dx.reshape(v.shape), wx, x.dtype), (dw, ww, w.dtype)):
            B.near(got, exact, max(2 * B.U[kind], 2e-6), "gradient")
    with torch.no_grad():
        assert torch.equal(linear_cross_entropy(x, w, t, reduction, ignored).view(torch.int32), loss.detach().view(torch.int32))
    return loss, dx, dw


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("form", ["shared", "apart", "own"])
@pytest.mark.parametrize("n,rows,h,vocab", [(1, 1, 64, 128), (2, 1, 40, 1), (3, 2, 72, 513), (2, 5, 8, 257), (2, 130, 264, 700), (3, 257, 100, 129),
                                            (1, 300, 1, 3), (2, 33, 1001, 300), (5, 1, 515, 1000), (2, 64, 512, 256)])
def test_against_64_bits(n, rows, h, vocab, form, kinds):
    x, w, t, g = inputs(rows + h, n, rows, h, vocab, *kinds, form)
    for reduction in ("mean", "none", "sum"):
        shape = (n, rows) if reduction == "none" else (n,)
        verify(x, w, t, reduction, torch.randn(*shape, generator=g, device="cuda"))


@pytest.mark.parametrize("kinds", TYPES, ids=str)
def test_many_tiles_pieces_and_parts(kinds):
    # several tiles of every kind to a pair of CTAs; a vocabulary in several pieces beside an fp32 weight
    x, w, t, g = inputs(1, 4, 300, 1100, 21000, *kinds, "apart")
    verify(x, w, t, "mean", torch.ones(4, device="cuda"))
    x, w, t, g = inputs(2, 2, 1, 4096, 30001, *kinds, "shared")  # a long sum for dx, few rows
    verify(x, w, t, "none", torch.ones(2, 1, device="cuda"))
    x, w, t, g = inputs(3, 40, 3, 256, 600, *kinds, "shared", 0.0)  # segments of three rows
    verify(x, w, t, "sum", torch.linspace(0.1, 50.0, 40, device="cuda"))


@pytest.mark.parametrize("kinds", TYPES, ids=str)
def test_pieces_of_one_batch_of_gradients(kinds):
    # d of 30000 rows fills its room with a few thousand columns: dx grows over pieces, the last one shorter
    x, w, t, g = inputs(4, 3, 10000, 64, 20000 if kinds[1] != F32 else 7000, *kinds, "shared")
    leaf, wleaf = x.detach().requires_grad_(), w.detach().requires_grad_()
    loss = linear_cross_entropy(leaf, wleaf, t)
    dx, dw = torch.autograd.grad(loss, (leaf, wleaf), torch.ones(3, device="cuda"))
    z = x.double().flatten(0, 1) @ w.double().T
    lse = torch.logsumexp(z, -1)
    counted = (t != -100).flatten()
    at = torch.where(counted, t.flatten(), 0)
    row = torch.where(counted, lse - z.gather(1, at[:, None])[:, 0], 0.0).view(3, -1)
    by = (t != -100).sum(1).double()
    B.near(loss, row.sum(1) / by, 1e-6, "loss")
    d = z.sub_(lse[:, None]).exp_()
    d[torch.arange(len(d), device="cuda"), at] -= 1.0
    d.mul_((counted / by.repeat_interleave(10000))[:, None])
    B.near(dx, (d @ w.double()).view(x.shape), max(2 * B.U[kinds[0]], 2e-6), "dx")
    B.near(dw, d.T @ x.double().flatten(0, 1), max(2 * B.U[kinds[1]], 2e-6), "dweight")


@pytest.mark.parametrize("kinds", TYPES, ids=str)
def test_strides_and_axes(kinds):
    n, rows, h, vocab = 3, 36, 64, 400
    x, w, t, g = inputs(5, n, rows, 2 * h + 8, vocab, *kinds, "own")
    one = torch.ones(n, device="cuda")
    verify(x[..., :h], w[..., :h], t, "mean", one)                      # rows further apart, on 16-byte boundaries
    verify(x[..., 3:h + 3], w[..., 5:h + 5], t, "mean", one)            # off them
    verify(x[..., :h], w[0, :, :h], t, "mean", one)
    verify(x[:, ::2, :h], w[:, ::3, :h], t[:, ::2].remainder(100), "mean", one)
    verify(x[:, :1, :h], w[0, :, :h], t[:, :1], "mean", one)            # one row a worker, workers far apart
    verify(x[:, 0, :h], w[:, :, :h], t[:, 0], "none", one)              # two axes
    verify(x[:, :2, :h], w[0, :, :h], t[:, :2], "none", torch.ones(n, 2, device="cuda"))
    verify(x[:1, :2, :h].transpose(0, 1), w[:2, :, :h], t[:1, :2].t(), "sum", one[:2])
    y = x[..., :h].reshape(n, 4, 9, h)
    verify(y, w[..., :h], t.view(n, 4, 9), "none", torch.rand(n, 4, 9, generator=g, device="cuda"))
    verify(y.transpose(1, 2), w[..., :h], t.view(n, 4, 9).transpose(1, 2), "none", torch.rand(n, 9, 4, generator=g, device="cuda").transpose(1, 2).transpose(1, 2))
    verify(x[:1, :, :h].expand(n, rows, h), w[:1, :, :h].expand(n, vocab, h), t, "mean", one)
    verify(x[:, :1, :h].expand(n, rows, h), w[0, :, :h], t, "none", torch.ones(1, 1, device="cuda").expand(n, rows))
    verify(x.transpose(1, 2)[:, :h].transpose(1, 2), w[0, :, :h].t().contiguous().t(), t, "mean", one)  # columns that are not packed


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("rows", [2, 40])
def test_masks(kinds, rows):
    x, w, t, g = inputs(6, 3, rows, 96, 300, *kinds, "shared", 0.0)
    t[1] = -100  # a worker without targets
    t[2, 1:] = -100
    for reduction, dloss in (("mean", torch.ones(3, device="cuda")), ("sum", torch.ones(3, device="cuda")), ("none", torch.ones(3, rows, device="cuda"))):
        loss, dx, dw = verify(x, w, t, reduction, dloss)
        assert not loss[1].any() and not dx[1].any() and not dx[2, 1:].any()
    t[:] = -100
    loss, dx, dw = verify(x, w, t, "mean", torch.ones(3, device="cuda"))
    assert not loss.any() and not dx.any() and not dw.any()
    t[:] = 7  # another number to ignore
    t[0] = 5
    loss, dx, dw = verify(x, w, t, "mean", torch.ones(3, device="cuda"), ignored=7)
    assert loss[0] > 0 and not loss[1:].any()


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("rows", [2, 300])
def test_targets_outside_the_vocabulary_are_nan(kinds, rows):
    x, w, t, g = inputs(7, 2, rows, 64, 200, *kinds, "own", 0.0)
    t[0, 0], t[0, 1] = 200, -1
    loss, dx, dw = verify(x, w, t, "none", torch.ones(2, rows, device="cuda"))
    assert torch.isnan(loss[0, :2]).all() and torch.isfinite(loss[0, 2:]).all() and torch.isfinite(loss[1]).all()
    assert torch.isnan(dx[0, :2]).all() and torch.isnan(dw[0]).all() and torch.isfinite(dw[1]).all()
    t[0, 0] = 1 << 40
    t[0, 1] = -(1 << 62)
    loss, dx, dw = verify(x, w, t, "mean", torch.ones(2, device="cuda"))
    assert torch.isnan(loss[0]) and torch.isfinite(loss[1])


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("rows", [1, 150])
def test_values_that_are_not_finite_stay_in_their_rows(kinds, rows):
    x, w, t, g = inputs(8, 2, rows, 64, 200, *kinds, "own", 0.0)
    clean = linear_cross_entropy(x, w, t, "none")
    x[0, 0, 3] = float("nan")
    loss = linear_cross_entropy(x, w, t, "none")
    assert torch.isnan(loss[0, 0]) and torch.equal(loss.flatten()[1:], clean.flatten()[1:])
    t[0, 0] = -100
    loss = linear_cross_entropy(x, w, t, "none")
    assert loss[0, 0] == 0 and torch.equal(loss.flatten()[1:], clean.flatten()[1:])


@pytest.mark.parametrize("kinds", [(BF16, BF16), (F32, F32)], ids=str)
@pytest.mark.parametrize("rows", [2, 100])
def test_large_logits(kinds, rows):
    # differences of thousands: exponentials that vanish, and a probability of 1
    x, w, t, g = inputs(9, 2, rows, 256, 500, *kinds, "shared", 0.0)
    # an fp32 logit of 6000 is off by 6000 2^-24 = 4e-4 and a probability by as much, above the 2e-6 that lengths are held to elsewhere;
    # the elementwise tolerance counts it
    verify(x * 1000, w, t, "none", torch.ones(2, rows, device="cuda"), lengths=False)
    verify(x, w * 0, t, "none", torch.ones(2, rows, device="cuda"))  # all the same


@pytest.mark.parametrize("scale", [1e-6, 1.0, 65536.0])
def test_gradients_of_half_precision_under_a_loss_scale(scale):
    x, w, t, g = inputs(10, 2, 200, 128, 1000, F16, F16, "shared")
    verify(x, w, t, "sum", torch.full((2,), scale, device="cuda") * 0.1)
    verify(x, w, t, "none", scale * 0.01 * torch.rand(2, 200, generator=g, device="cuda"))


@pytest.mark.parametrize("kinds", TYPES, ids=str)
def test_one_gradient_alone_is_the_same(kinds):
    x, w, t, g = inputs(11, 2, 70, 200, 600, *kinds, "apart")
    leaf, wleaf = x.detach().requires_grad_(), w.detach().requires_grad_()
    dx, dw = torch.autograd.grad(linear_cross_entropy(leaf, wleaf, t).sum(), (leaf, wleaf))
    only, = torch.autograd.grad(linear_cross_entropy(leaf, w, t).sum(), leaf)
    assert torch.equal(only, dx)
    only, = torch.autograd.grad(linear_cross_entropy(x, wleaf, t).sum(), wleaf)
    assert torch.equal(only, dw)
    again = torch.autograd.grad(linear_cross_entropy(leaf, wleaf, t).sum(), (leaf, wleaf))
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_no_rows_and_no_workers():
    w = torch.randn(50, 16, device="cuda", requires_grad=True)
    x = torch.zeros(3, 0, 16, device="cuda", requires_grad=True)
    t = torch.zeros(3, 0, dtype=torch.int64, device="cuda")
    for reduction, shape in (("mean", (3,)), ("sum", (3,)), ("none", (3, 0))):
        loss = linear_cross_entropy(x, w, t, reduction)
        assert loss.shape == shape and not loss.any()
        dx, dw = torch.autograd.grad(loss.sum(), (x, w))
        assert dx.shape == x.shape and not dw.any()
    assert linear_cross_entropy(x[:0], w, t[:0]).shape == (0,)


def test_gradients_against_differences():
    g = torch.Generator(device="cuda").manual_seed(12)
    x, w, t, _ = inputs(12, 2, 9, 24, 50, F32, F32, "own")
    leaf, wleaf = x.requires_grad_(), w.requires_grad_()
    dx, dw = torch.autograd.grad(linear_cross_entropy(leaf, wleaf, t).sum(), (leaf, wleaf))
    u, v = torch.randn(x.shape, generator=g, device="cuda"), torch.randn(w.shape, generator=g, device="cuda")
    e = 1e-2
    with torch.no_grad():
        up, down = (linear_cross_entropy(x + k * e * u, w + k * e * v, t).double().sum() for k in (1, -1))
    along = float((dx.double() * u).sum() + (dw.double() * v).sum())
    # the third derivative along (u, v) is a few units of |u w + x v|^3, about 30; fp32 losses of 4 are off by 1e-6
    assert abs(float(up - down) / (2 * e) - along) < 30 * e * e + 1e-3


@pytest.mark.parametrize("kinds", TYPES, ids=str)
def test_a_few_rows_of_growing_width(kinds):
    # more shared memory from call to call, up to what a few rows may have, and beyond, where other kernels take over
    for rows, h in ((1, 12800), (1, 16000), (1, 24576), (1, 24577), (2, 8000), (2, 12288), (4, 4000), (4, 6144), (4, 6145)):
        x, w, t, g = inputs(rows + h, 1, rows, h, 40, *kinds, "shared", 0.0)
        want, tol = B.head(x, w, t, "none")
        B.check(linear_cross_entropy(x, w, t, "none"), want, tol, "loss")


@pytest.mark.parametrize("rows", [1, 130])
def test_offsets_beyond_32_bits(rows):
    vocab, h = 140000, 16384  # 2.3 G elements
    g = torch.Generator(device="cuda").manual_seed(13)
    w = torch.empty(vocab, h, dtype=BF16, device="cuda")
    for k in range(0, vocab, 20000):
        w[k:k + 20000] = (2.0 / 128 * torch.randn(20000, h, generator=g, device="cuda")).to(BF16)
    x = torch.randn(1, rows, h, generator=g, device="cuda").to(BF16).requires_grad_()
    t = torch.randint(0, vocab, (1, rows), generator=g, device="cuda")
    t[0, 0] = vocab - 1
    loss = linear_cross_entropy(x, w.requires_grad_(), t, "none")
    dx, dw = torch.autograd.grad(loss.sum(), (x, w))
    with torch.no_grad():
        z = torch.cat([x[0].double() @ w[k:k + 10000].double().T for k in range(0, vocab, 10000)], 1)
        want = torch.logsumexp(z, 1) - z.gather(1, t.T)[:, 0]
        B.near(loss[0], want, 1e-6, "loss")
        d = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
        d[torch.arange(rows, device="cuda"), t[0]] -= 1.0
        B.near(dx[0], sum(d[:, k:k + 10000] @ w[k:k + 10000].double() for k in range(0, vocab, 10000)), 2 * B.U[BF16], "dx")
        for k in (0, 65536, vocab - 1000):
            B.near(dw[k:k + 1000], d[:, k:k + 1000].T @ x[0].double(), 2 * B.U[BF16], "dweight")


def test_captured_and_replayed():
    x, w, t, g = inputs(14, 2, 140, 72, 600, BF16, F32, "apart")
    few = x[:, :1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    leaf, wleaf = x.clone().requires_grad_(), w.detach().requires_grad_()
    with torch.cuda.stream(side):
        for _ in range(2):
            torch.autograd.grad(linear_cross_entropy(leaf, wleaf, t).sum(), (leaf, wleaf))
            linear_cross_entropy(few, w, t[:, :1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            loss = linear_cross_entropy(leaf, wleaf, t)
            dx, dw = torch.autograd.grad(loss.sum(), (leaf, wleaf))
            one = linear_cross_entropy(few, w, t[:, :1])
    torch.cuda.current_stream().wait_stream(side)
    for k in range(2):
        with torch.no_grad():
            leaf.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            few.copy_(leaf[:, 1:2])
            t.copy_(torch.randint(0, 600, t.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        a, b = leaf.detach().clone().requires_grad_(), w.detach().requires_grad_()
        want = linear_cross_entropy(a, b, t)
        wx, ww = torch.autograd.grad(want.sum(), (a, b))
        assert torch.equal(loss, want) and torch.equal(dx, wx) and torch.equal(dw, ww)
        assert torch.equal(one, linear_cross_entropy(few, w, t[:, :1]))


def test_two_streams_at_once():
    a, b = inputs(15, 2, 300, 512, 5000, BF16, BF16, "shared"), inputs(16, 3, 200, 264, 7000, F32, F32, "own")

    def both(x, w, t, _):
        leaf, wleaf = x.detach().requires_grad_(), w.detach().requires_grad_()
        loss = linear_cross_entropy(leaf, wleaf, t)
        return (loss.detach(), *torch.autograd.grad(loss.sum(), (leaf, wleaf)))

    want = both(*a), both(*b)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, (s, inp) in enumerate(zip(streams, (a, b))):
            with torch.cuda.stream(s):
                got[k].append(both(*inp))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(torch.equal(p, q) for p, q in zip(g, want[k]))


@pytest.mark.parametrize("n", [1000, 65535])
def test_many_workers(n):
    g = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(n, 2, 16, generator=g, device="cuda").to(BF16).requires_grad_()
    w = torch.randn(300, 16, generator=g, device="cuda").to(BF16).requires_grad_()
    t = torch.randint(0, 300, (n, 2), generator=g, device="cuda")
    loss = linear_cross_entropy(x, w, t)
    dx, dw = torch.autograd.grad(loss.sum(), (x, w))
    x64, w64 = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    z = (x64.flatten(0, 1) @ w64.T).view(n, 2, -1)
    want = (torch.logsumexp(z, -1) - z.gather(-1, t[..., None])[..., 0]).mean(1)
    wx, ww = torch.autograd.grad(want.sum(), (x64, w64))
    B.near(loss, want.detach(), 1e-6, "loss"), B.near(dx, wx, 2 * B.U[BF16], "dx"), B.near(dw, ww, 2 * B.U[BF16], "dweight")


def test_no_wait_gave_up():
    v = ctypes.c_int32(-1)
    assert load_library().compams_head_status(ctypes.byref(v)) == 0 and v.value == 0
