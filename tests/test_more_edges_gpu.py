"""Edges of the operators around a block and at the two ends of the backward pass: gradients that are the negative of what lies in memory, rows
with infinities, clipping at its borders, a few rows of every width, tensors without axes, streams that cancel, rows' gradients that are large
or far apart, tangents of gradients, saved tensors that hooks give back in another order; on the path of the extension and on Python's."""
import pytest
import torch

import blocks64 as B
import paper_2205_05632_b200.binding as binding
from paper_2205_05632_b200 import CompAMSError
from paper_2205_05632_b200.layers import gated_add_rms_norm, linear_cross_entropy, rms_norm
from paper_2205_05632_b200.optim import clip_gradients, collect_gradients

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(BF16, BF16), (F16, F16), (F32, F32), (BF16, F32), (F16, F32)]


class _Nothing:
    """No call is a usual one."""

    def __getattr__(self, name):
        return lambda *args: None


@pytest.fixture(params=["extension", "python"])
def path(request, monkeypatch):
    binding.load_operators()
    if request.param == "python":
        monkeypatch.setattr(binding, "_ops", _Nothing())
    return request.param


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("h", [64, 1001, 8200])
def test_gradients_that_are_negatives_of_what_lies_in_memory(h, kinds, path):
    g = gen(h)
    x, dy, res, ds = rand(g, 2, 5, h, dtype=kinds[0]), rand(g, 2, 5, h, dtype=kinds[0]), rand(g, 2, 5, h, dtype=kinds[1]), rand(g, 2, 5, h, dtype=kinds[1])
    p = [1.0 + 0.2 * rand(g, 2, h) for _ in range(3)]
    w, t = rand(g, 30, h, dtype=kinds[1]), torch.randint(0, 30, (2, 5), generator=g, device="cuda")
    negative = torch._neg_view
    assert negative(dy).is_neg() and negative(dy).is_contiguous()

    def norm(dy):
        a = [v.detach().requires_grad_() for v in (x, p[0])]
        return torch.autograd.grad(rms_norm(*a), a, dy)

    def gated(dy, ds):
        a = [v.detach().requires_grad_() for v in (x, res, *p)]
        return torch.autograd.grad(gated_add_rms_norm(*a), a, (dy, ds))

    def head(dloss, reduction):
        a = [v.detach().requires_grad_() for v in (x, w)]
        return torch.autograd.grad(linear_cross_entropy(*a, t, reduction), a, dloss)

    assert same(norm(negative(dy)), norm(-dy))
    assert same(gated(negative(dy), ds), gated(-dy, ds))
    assert same(gated(dy, negative(ds)), gated(dy, -ds))
    for reduction, shape in (("mean", (2,)), ("none", (2, 5))):
        dloss = rand(g, *shape)
        assert same(head(negative(dloss), reduction), head(-dloss, reduction))


@pytest.mark.parametrize("kind", [BF16, F16, F32])
@pytest.mark.parametrize("h", [500, 512, 1000, 2001, 4096, 9000])
def test_rows_with_an_infinity(h, kind, path):
    # 1 / sqrt(infinity) is 0: a norm's row is 0 but for 0 * infinity, and the stream is what the residual is, the 16-bit ones' borders included
    g = gen(h)
    x, res, dy = (rand(g, 3, 60, h, dtype=kind) for _ in range(3))
    w, gate = 1.0 + 0.2 * rand(g, 3, h), 0.5 + 0.2 * rand(g, 3, h)
    x[:, ::2, 7], x[:, 1::2, 9] = float("inf"), -float("inf")
    if kind != F16:
        x[:, 2, 7] = 1e30  # its square is beyond fp32, itself it is not
    at = torch.isinf(x)
    a = [v.detach().requires_grad_() for v in (x, res, w, gate)]
    y, s = gated_add_rms_norm(*a, None, residual_scale=0.9)
    want = torch.where(at, float("nan"), 0.9 * res.double())
    B.check(s, want, 4 * B.E * want.abs(), "s")  # alpha, the product and the sum with 0 are rounded
    rows = at.any(-1)
    assert torch.isnan(y[rows]).all() and torch.isfinite(y[~rows]).all()
    dx, = torch.autograd.grad(y, a[0], dy)
    assert torch.isnan(dx[rows]).all()
    y = rms_norm(a[0], a[2])
    assert torch.equal(torch.isnan(y), at) and not y.nan_to_num().any()
    dx, dw = torch.autograd.grad(y, (a[0], a[2]), dy)
    assert torch.isnan(dx[rows]).all() and torch.equal(torch.isnan(dw), at.any(1))


@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_clipping_at_its_borders(kind, path):
    t = torch.zeros(3, 100, dtype=kind, device="cuda")
    t[1], t[2, 5] = 2.0, 4.0  # norms 0, 20 and 4
    for max_norm, eps, factors in ((0.0, 0.0, (1.0, 0.0, 0.0)), (0.0, 1.0, (0.0, 0.0, 0.0)), (4.0, 0.0, (1.0, 0.2, 1.0)), (4.0, 4.0, (1.0, 4 / 24, 0.5)),
                                   (20.0, 0.0, (1.0, 1.0, 1.0)), (float("inf"), 1.0, (1.0, 1.0, 1.0))):
        G, norms = collect_gradients([t], max_norm=max_norm, eps=eps)
        assert norms.tolist() == [0.0, 20.0, 4.0]
        f = torch.tensor(factors, dtype=torch.float64, device="cuda")[:, None]
        B.check(G, t.double() * f, 2 * B.E * t.double().abs(), "G")  # the factor is rounded, and the product
        kept = t.clone()
        clip_gradients([kept], max_norm, eps)
        B.check(kept, t.double() * f, 2 * B.E * t.double().abs(), "in place")
        assert torch.equal(kept[f[:, 0] == 1.0], t[f[:, 0] == 1.0])


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("rows,h", [(1, 12264), (1, 12280), (1, 12288), (1, 12296), (2, 6120), (2, 6136), (2, 6144), (3, 3064), (3, 6144), (3, 6145), (3, 7168),
                                    (3, 8192), (3, 8193), (4, 3058), (4, 3064), (4, 6144)])
def test_a_few_rows_of_every_width(rows, h, kinds):
    # x takes up to 96 KB of shared memory, three rows as much as four; from 48 KB on, the kernel's own arrays counted, it has to be asked for
    g = gen(rows + h)
    x, t = rand(g, rows, h, dtype=kinds[0]), torch.randint(0, 40, (rows,), generator=g, device="cuda")
    w = (2.0 * h ** -0.5 * rand(g, 2, 40, h)).to(kinds[1])
    one_worker, one_row_each, weights_of_their_own = (x[None], w[0], t[None]), (x[:, None], w[0], t[:, None]), (
        torch.stack([x, x.flip(0)]), w, torch.stack([t, t]))
    for call in (one_worker, one_row_each, weights_of_their_own):
        want, tol = B.head(*call, "none")
        B.check(linear_cross_entropy(*call, "none"), want, tol, "loss")


@pytest.mark.parametrize("kinds", [(BF16, BF16), (F16, F16), (BF16, F32)], ids=str)
@pytest.mark.parametrize("h", [72, 1000, 1001, 4104, 9000])
def test_a_padded_batch(h, kinds, path):
    # rows of zeros: their sum is 0 and their gradient what the norm's slope at 0 makes of it; the others do not notice. Sums that cancel to 0
    g = gen(h)
    x, res = rand(g, 3, 20, h, dtype=kinds[0]), rand(g, 3, 20, h, dtype=kinds[1])
    w, gate, v = (1.0 + 0.2 * rand(g, 3, h) for _ in range(3))
    y0, s0 = gated_add_rms_norm(x, res, w, gate, v, residual_scale=0.7)
    x[:, 11:], res[:, 11:] = 0.0, 0.0
    y, s = gated_add_rms_norm(x, res, w, gate, v, residual_scale=0.7)
    assert not s[:, 11:].any() and not y[:, 11:].any()
    assert torch.equal(s[:, :11], s0[:, :11]) and torch.equal(y[:, :11], y0[:, :11])
    one = torch.ones_like(x)
    y, s = gated_add_rms_norm(one, -one.to(kinds[1]), eps=0.0)  # 1 / sqrt(1) - 1
    assert not s.any()


def test_tensors_without_axes_are_refused(path):
    x, one, t = torch.zeros(2, 3, 8, device="cuda"), torch.ones((), device="cuda"), torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    for call in (lambda: rms_norm(x, one), lambda: rms_norm(one), lambda: gated_add_rms_norm(x, x, one), lambda: gated_add_rms_norm(x, x, gate=one),
                 lambda: gated_add_rms_norm(x, x, next_weight=one), lambda: gated_add_rms_norm(x, one), lambda: linear_cross_entropy(x, one, t),
                 lambda: linear_cross_entropy(x, torch.ones(5, 8, device="cuda"), t[0, 0]), lambda: collect_gradients([one]),
                 lambda: collect_gradients([x], out=one), lambda: clip_gradients([one], 1.0)):
        with pytest.raises(CompAMSError):
            call()


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("h", [2048, 1001])
def test_a_stream_that_cancels_is_rounded_as_the_exact_sum(h, kind):
    # down to the smallest numbers of the type: a third of the sums is below 2^-14, where fp16 has no more bits
    g = gen(4)
    x, w = rand(g, 4, 300, h, dtype=kind), 1.0 + 0.3 * rand(g, 4, h)
    gate = rand(g, 4, h) * 10.0 ** (4 * torch.rand(4, h, generator=g, device="cuda") - 3)
    u = B.rms(x.double(), w.double()[:, None], 1e-6)[0] * gate.double()[:, None]
    res = (-u / 0.7 * (1.0 + 0.01 * torch.randn(u.shape, generator=g, device="cuda"))).to(kind)
    _, s = gated_add_rms_norm(x, res, w, gate, None, residual_scale=0.7)
    want = 0.7 * res.double() + u
    assert int((want.abs() < 2.0 ** -14).sum()) > want.numel() // 4
    off = s.double() != want.float().to(kind).double()
    assert int(off.sum()) <= 2 + 1e-6 * off.numel()


@pytest.mark.parametrize("kinds", [(BF16, BF16), (F32, F32), (BF16, F32)], ids=str)
@pytest.mark.parametrize("top", [1e-38, 1.5e38, 3e38])
def test_rows_gradients_at_the_ends_of_the_range(top, kinds):
    g = gen(1)
    x, w = (1e-2 * rand(g, 2, 9, 64)).to(kinds[0]).requires_grad_(), (1e-2 * rand(g, 200, 64)).to(kinds[1]).requires_grad_()
    t = torch.randint(0, 200, (2, 9), generator=g, device="cuda")
    dloss = torch.full((2, 9), top, device="cuda")
    dloss[0, 3], dloss[1, 4], dloss[1, 5] = 1e-3 * top, -top, 0.0
    got = torch.autograd.grad(linear_cross_entropy(x, w, t, "none"), (x, w), dloss)
    _, _, wx, tx, ww, tw = B.head(x.detach(), w.detach(), t, "none", -100, dloss)
    B.check(got[0], wx, tx, "dx")
    B.check(got[1], ww, tw, "dweight")


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("n,rows,h,vocab,form", [(1, 64, 128, 5000, "shared"), (2, 40, 72, 700, "own"), (3, 33, 1001, 300, "apart"), (2, 300, 512, 40000, "shared"),
                                                   (3, 10000, 64, 20000, "shared")])
@pytest.mark.parametrize("span", [6, 24])
def test_rows_gradients_far_apart(span, n, rows, h, vocab, form, kinds):
    # each row's dx is as good as by itself: the weights of some rows are a millionth of the others'
    g = gen(span + h)
    x = rand(g, n, rows, h, dtype=kinds[0]).requires_grad_()
    w = (2.0 * h ** -0.5 * rand(g, *((n,) if form == "own" else ()), vocab, h)).to(kinds[1])
    w = (w.expand(n, vocab, h) if form == "apart" else w).detach().requires_grad_()
    t = torch.randint(0, vocab, (n, rows), generator=g, device="cuda")
    t[:, 1] = -100
    dloss = 4096.0 * 2.0 ** (-span * torch.rand(n, rows, generator=g, device="cuda"))
    dloss[:, 2], dloss[:, 3], dloss[:, 0] = 0.0, -dloss[:, 3], 4096.0
    dloss[:, 4:7] = 4096.0 * 2.0 ** -span

    def both(x, w):
        return torch.autograd.grad(linear_cross_entropy(x, w, t, "none"), [v for v in (x, w) if v.requires_grad], dloss)

    dx, dw = both(x, w)
    _, _, wx, tx, ww, tw = B.head(x.detach(), w.detach(), t, "none", -100, dloss)
    B.check(dx, wx, tx, "dx")
    # dweight is a sum over the rows, where fp16's d is relative to the worker's largest: off by up to 2^-39 of 8192, the power of two above it
    lost = x.detach().abs().double().sum((0, 1) if form == "shared" else 1).unsqueeze(-2) * (2.0 ** -38 * 4096.0 if kinds == (F16, F16) else 0.0)
    B.check(dw, ww, tw + lost, "dweight")
    if span == 6 or kinds != (F16, F16):
        for i in range(n):
            B.near(dx[i], wx[i], max(2 * B.U[kinds[0]], 2e-6), "dx")
    if rows < 10000:  # a piece of the vocabulary; of several, each gradient alone may have fewer, and sums in another order
        assert torch.equal(both(x, w.detach())[0], dx) and torch.equal(both(x.detach(), w)[0], dw)


def test_tangents_of_gradients_are_refused(path):
    from torch.autograd import forward_ad
    g = gen(1)
    x, w, t = rand(g, 2, 5, 16).requires_grad_(), rand(g, 30, 16).requires_grad_(), torch.randint(0, 30, (2, 5), generator=g, device="cuda")
    for y in (rms_norm(x), *gated_add_rms_norm(x, x), linear_cross_entropy(x, w, t)):
        with forward_ad.dual_level():
            dy = torch.ones_like(y)
            want, = torch.autograd.grad(y, x, dy, retain_graph=True)  # without a tangent a level changes nothing
            with pytest.raises(RuntimeError, match="forward-mode"):
                torch.autograd.grad(y, x, forward_ad.make_dual(dy, dy), retain_graph=True)
        assert torch.equal(torch.autograd.grad(y, x, dy, retain_graph=True)[0], want)


@pytest.mark.parametrize("kinds", [(BF16, BF16), (F32, F32), (BF16, F32)], ids=str)
def test_saved_tensors_that_hooks_unpack(kinds, path):
    g = gen(2)
    x, res = (rand(g, 3, 7, 72, dtype=k).requires_grad_() for k in kinds)
    w, p = rand(g, 40, 72, dtype=kinds[1]).requires_grad_(), [(1.0 + 0.2 * rand(g, 3, 72)).requires_grad_() for _ in range(3)]
    t = torch.randint(0, 40, (3, 7), generator=g, device="cuda")

    def otherwise(v):  # the same values, the first axis innermost
        return v.movedim(0, -1).contiguous().movedim(-1, 0) if v.dim() > 1 else torch.stack([v, v], 1)[:, 0]

    def negative(v):
        return torch._neg_view(-v) if v.is_floating_point() else v

    calls = ((lambda: (rms_norm(x, p[0]),), (x, p[0])), (lambda: (rms_norm(x, p[0][0]),), (x, p[0])), (lambda: gated_add_rms_norm(x, res, *p), (x, res, *p)),
             (lambda: (linear_cross_entropy(x, w, t),), (x, w)), (lambda: (linear_cross_entropy(x, w.expand(3, 40, 72), t, "none"),), (x, w)))
    def gradients(out, leaves):
        return torch.autograd.grad([y.float().square().sum() for y in out], leaves)

    hooks = [torch.autograd.graph.saved_tensors_hooks(lambda v: v, otherwise), torch.autograd.graph.saved_tensors_hooks(lambda v: v, negative),
             torch.autograd.graph.save_on_cpu()]
    for call, leaves in calls:
        want = gradients(call(), leaves)
        for hook in hooks:
            with hook:
                out = call()
            # (a weight that all share may come back as one of each worker's own: its sums then run in another order)
            for a, b in zip(gradients(out, leaves), want):
                B.near(a, b.double(), 2 * B.U[a.dtype] + 2.0 ** -20, "gradient")


def test_leaves_and_their_views_are_not_scaled_in_place():
    x = torch.ones(2, 3, 4, device="cuda", requires_grad=True)
    for bad in (x, x.view(2, 12), x[:, 1], x[:1]):
        with pytest.raises(CompAMSError):
            clip_gradients([bad], 0.01)
    assert torch.equal(x, torch.ones_like(x))
    with torch.no_grad():
        clip_gradients([x.view(2, 12)], 0.01, eps=0.0)
    B.near(x, x.detach().double().fill_(0.01 / 12 ** 0.5), 4 * B.E, "x")
    clip_gradients([x.detach()], 0.001)
    G, norms = collect_gradients([x, x * 2.0])  # a copy, which knows nothing of where it is from
    assert not G.requires_grad and not norms.requires_grad


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("n,rows,form", [(1, 1, "shared"), (1, 2, "shared"), (3, 1, "shared"), (1, 4, "apart"), (2, 3, "own"), (1, 6, "shared"), (2, 200, "own")])
@pytest.mark.parametrize("h,vocab", [(1024, 700), (1002, 9001)])
def test_rows_whose_target_is_nearly_certain(h, vocab, n, rows, form, kinds):
    # Logits of a few units from products that sum to thousands in magnitude: of another order, they are another 1e-3. d of the target is p - 1, of a
    # millionth; it is as exact as the statistics are as long as both passes have the same logits, whatever these are off by.
    g = gen(h + rows)
    half = rand(g, n, rows, h // 2).abs() + 0.1
    x = torch.cat([half, half], -1).to(kinds[0])
    along = torch.cat([torch.ones(h // 2, device="cuda"), -torch.ones(h // 2, device="cuda")])
    t = torch.full((n, rows), 7, device="cuda")
    to = torch.full((vocab, 1), -20.0, device="cuda")
    to[7] = 3.0
    w = (7.5 * along + 0.05 * rand(g, *((n,) if form == "own" else ()), vocab, h) + to / (0.9 * h)).to(kinds[1])
    w = (w.expand(n, vocab, h) if form == "apart" else w).detach().requires_grad_()
    x.requires_grad_()
    loss = linear_cross_entropy(x, w, t, "none")
    got = torch.autograd.grad(loss.sum(), (x, w))
    together, dws, tws = w.dim() == 2, [], []
    for i in range(n):
        x64, w64 = x[i].detach().double(), (w if together else w[i]).detach().double()
        z, dz = x64 @ w64.T, (h / 512 + 64) * 2 * B.E * (x64.abs() @ w64.abs().T)
        lse = torch.logsumexp(z, -1, keepdim=True)
        p = torch.exp(z - lse)
        assert float((1.0 - p[:, 7]).max()) < 1e-3
        # lse and its logarithm are rounded, the sum of exponentials at most 16 times beside 1; logits that are off shift p against p, of 1 - p
        off = 2 * B.E * (lse.abs() + z.amax(-1, keepdim=True).abs()) + 2.0 ** -20
        rest = 2 * dz.amax(-1, keepdim=True) + 2.0 ** -19
        d, err = p.clone(), p * (rest + off)
        d[:, 7] = -p[:, torch.arange(vocab, device="cuda") != 7].sum(1)
        err[:, 7] = (off - d[:, 7:8] * rest)[:, 0]
        planes = {BF16: B.U[BF16], F16: B.U[F16] if kinds[1] == F16 else 2.0 ** -17, F32: B.E}[kinds[0]] + (2.0 ** -16 if kinds[0] != kinds[1] else 3 * B.E)
        if kinds == (F16, F16):
            err = err + 2.0 ** -38
        B.check(got[0][i], d @ w64, err @ w64.abs() + (planes + (vocab / 512 + 64) * 2 * B.E) * (d.abs() @ w64.abs()), "dx")
        dws.append(d.T @ x64)
        planes = (B.E if kinds[1] == F32 else B.U[kinds[1]]) + 3 * B.E
        tws.append(err.T @ x64.abs() + (planes + (rows / 512 + 64) * 2 * B.E) * (d.T.abs() @ x64.abs()))
    dw, tw = torch.stack(dws), torch.stack(tws)
    B.check(got[1], dw.sum(0) if together else dw, tw.sum(0) if together else tw, "dweight")


@pytest.mark.parametrize("kinds", TYPES, ids=str)
@pytest.mark.parametrize("rows", [1, 3, 40, 300])
def test_small_losses_of_large_logits(rows, kinds):
    # a target's logit of 320 in front of others of about 300: a loss of a ten-thousandth or less, of which a rounding of the logits' size, up to
    # 2^-16, would leave little
    g = gen(rows)
    x = torch.ones(2, rows, 64, dtype=kinds[0], device="cuda")
    w = (torch.randint(296, 305, (500, 1), generator=g, device="cuda").float() / 64).expand(500, 64).contiguous()
    w[3] = 5.0
    w = w.to(kinds[1])
    t = torch.full((2, rows), 3, device="cuda")
    z = x.double() @ w.double().T
    want = torch.logsumexp(z, -1) - z[..., 3]
    assert 1e-7 < float(want.min()) and float(want.max()) < 1e-3
    # z is a sum of 64 equal numbers of 10 bits at most: exact. Beside the target's 1 the sum of exponentials is rounded, by 2^-24 at most, at each
    # of the 127 other columns of a tile, as they are added one after another, and where tiles or warps are joined, 16 times at most; the
    # exponentials themselves are 2^-21 off and their arguments, of 24, 2^-20
    B.check(linear_cross_entropy(x, w, t, "none"), want, (127 + 16) * B.E + 2.0 ** -18 * want, "loss")
