"""A training step as the operators make it up: an adapter beside a projection, the norms around its block, the head, each worker's gradient
gathered and clipped, the optimizer's step; every worker's row of G against a model in 64 bits, and the operators' refusals on the device."""
import pytest
import torch

import blocks64 as B
from paper_2205_05632_b200 import BLOCKSIGN, TOPK, CompAMSError
from paper_2205_05632_b200.layers import gated_add_rms_norm, linear_cross_entropy, low_rank_adapter, rms_norm
from paper_2205_05632_b200.optim import CompAMSOptimizer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("compressor", [TOPK, BLOCKSIGN])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_steps(kind, compressor):
    n, rows, h, rank, vocab, limit = 4, 24, 96, 4, 320, 0.5
    g = torch.Generator(device="cuda").manual_seed(1)

    def rand(*shape, sigma=1.0, dtype=torch.float32):
        return (sigma * torch.randn(*shape, generator=g, device="cuda")).to(dtype)

    params = [torch.nn.Parameter(p) for p in (1 + rand(h, sigma=0.1), rand(rank, h, sigma=0.1), rand(h, rank, sigma=0.1), 1 + rand(h, sigma=0.1),
                                              0.5 + rand(h, sigma=0.1), 1 + rand(h, sigma=0.1), rand(vocab, h, sigma=0.1))]
    opt = CompAMSOptimizer(params, n, compressor, k_ratio=0.1, lr=1e-2)
    fixed = rand(h, h, sigma=h ** -0.5, dtype=kind)

    def forward(p, x, t):
        first, a, b, behind, gate, before, head = p
        y = rms_norm(x, first)
        z = low_rank_adapter(y, y @ fixed, a, b, scale=2.0)
        y, _ = gated_add_rms_norm(z, x, behind, gate, before, residual_scale=0.9)
        return linear_cross_entropy(y, head, t)

    def exact(p, x, t):
        """Losses, and each worker's gradient, in 64 bits."""
        out = []
        for i in range(n):
            first, a, b, behind, gate, before, head = q = [v.detach().double().requires_grad_() for v in p]

            def normed(v, w):
                return v / (v.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w

            v = x[i].double()
            y = normed(v, first)
            z = y @ fixed.double() + 2.0 * (y @ a.T) @ b.T
            y = normed(0.9 * v + gate * normed(z, behind), before)
            logits, at = y @ head.T, t[i] != -100
            loss = (torch.logsumexp(logits, -1) - logits.gather(-1, t[i].clamp(min=0)[:, None])[:, 0])[at].mean()
            out.append((loss.detach(), torch.cat([v.flatten() for v in torch.autograd.grad(loss, q)])))
        return torch.stack([o[0] for o in out]), torch.stack([o[1] for o in out])

    for step in range(3):
        x, t = rand(n, rows, h, dtype=kind), torch.randint(0, vocab, (n, rows), generator=g, device="cuda")
        t[0, :5] = -100
        leaves = opt.worker_parameters()
        loss = forward(leaves, x, t)
        loss.sum().backward()
        want, rows64 = exact(params, x, t)
        norms = opt.collect_all(max_norm=limit)
        size = rows64.norm(dim=1)
        # fp32: what the operators' own tests allow is far below; bfloat16: a few roundings of 2^-8 on the way there and back
        most = 1e-5 if kind == torch.float32 else 8 * 2.0 ** -8
        assert float(((loss.detach().double() - want).abs() / want).max()) <= most
        assert float(((norms.double() - size).abs() / size).max()) <= most
        assert float(size.max()) > limit  # something is clipped
        clipped = rows64 * (limit / (size + 1e-6)).clamp(max=1.0)[:, None]
        for i in range(n):
            B.near(opt.G[i], clipped[i], 2 * most, "G")
        before = opt.theta.clone()
        opt.step()
        assert not torch.equal(before, opt.theta) and torch.isfinite(opt.theta).all()
    assert opt.opt.check_status() == 0
    opt.close()


def test_refusals():
    x, w, t = torch.zeros(2, 3, 8, device="cuda"), torch.zeros(5, 8, device="cuda"), torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    half = torch.bfloat16
    for bad in (dict(weight=w.to(half)), dict(weight=w.double()), dict(weight=w[:, :7]), dict(weight=w[0]), dict(weight=w.cpu()), dict(weight=None),
                dict(weight=w.expand(3, 5, 8)), dict(weight=w[:0]), dict(target=t.int()), dict(target=t[:, :2]), dict(target=t.cpu()), dict(target=None),
                dict(reduction="max"), dict(reduction=None), dict(x=x.double()), dict(x=x[0, 0]), dict(ignore_index=1 << 63),
                dict(x=x.half(), weight=w.to(half))):
        with pytest.raises(CompAMSError):
            linear_cross_entropy(**{**dict(x=x, weight=w, target=t), **bad})
    p = torch.ones(8, device="cuda")
    for bad in (dict(weight=p[:7]), dict(weight=p.to(half)), dict(weight=p.cpu()), dict(weight=p.expand(3, 8)), dict(eps=-1.0), dict(eps=float("nan")),
                dict(x=x.double())):
        with pytest.raises(CompAMSError):
            rms_norm(**{**dict(x=x), **bad})
        with pytest.raises(CompAMSError):
            gated_add_rms_norm(**{**dict(x=x, residual=x), **bad})
    for bad in (dict(residual=x.to(half)), dict(residual=x[:1]), dict(residual=None), dict(gate=p.expand(2, 8), weight=p), dict(next_weight=p[:3])):
        with pytest.raises(CompAMSError):
            gated_add_rms_norm(**{**dict(x=x, residual=x), **bad})
    from torch.func import grad
    from torch.fx.experimental.proxy_tensor import make_fx
    for call in (lambda v: linear_cross_entropy(v, w, t).sum(), lambda v: rms_norm(v).sum(), lambda v: gated_add_rms_norm(v, v)[0].sum()):
        with pytest.raises(Exception):
            grad(call)(x)
        with pytest.raises(CompAMSError):
            make_fx(call)(x)


def test_a_second_derivative_is_refused():
    x, w = torch.randn(2, 3, 8, device="cuda", requires_grad=True), torch.randn(5, 8, device="cuda", requires_grad=True)
    t = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    for y in (linear_cross_entropy(x, w, t).sum(), rms_norm(x).sum(), gated_add_rms_norm(x, x)[0].sum()):
        dx, = torch.autograd.grad(y, x, create_graph=True)
        with pytest.raises(RuntimeError):
            dx.sum().backward()


def test_tangents_are_refused_and_tracing_records():
    from torch.autograd import forward_ad
    x, w = torch.randn(2, 3, 8, device="cuda"), torch.randn(5, 8, device="cuda")
    t = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    calls = (lambda v: linear_cross_entropy(v, w, t), rms_norm, lambda v: gated_add_rms_norm(v, v)[0])
    for call in calls:
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(x, torch.ones_like(x))
            with pytest.raises(Exception):
                call(dual)
            assert torch.equal(call(x), call(x.clone()))  # without a tangent a level changes nothing
        traced = torch.jit.trace(call, (x,), check_trace=False)
        other = torch.randn(2, 3, 8, device="cuda")
        assert torch.equal(traced(other), call(other))


def test_a_library_error_is_the_bindings_own():
    # a size that the library refuses and no check before it: 2^31 pieces of gradients cannot be had, a vocabulary of 2^31 rows can, of none
    w = torch.zeros(1, 8, device="cuda").expand(1 << 31, 8)
    with pytest.raises(CompAMSError):
        linear_cross_entropy(torch.zeros(2, 3, 8, device="cuda"), w, torch.zeros(2, 3, dtype=torch.int64, device="cuda"))
