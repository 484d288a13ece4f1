"""Calls of the newer operators that the documentation allows and that are easily forgotten: packed tensors that start off 16-byte boundaries,
inference mode, a backward pass taken twice, threads that call at once, results that are changed afterwards, the extension against its fallback."""
import threading

import pytest
import torch

import paper_2205_05632_b200.binding as binding
from paper_2205_05632_b200.layers import gated_add_rms_norm, linear_cross_entropy, rms_norm
from paper_2205_05632_b200.optim import collect_gradients

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


class _Nothing:
    """No call is a usual one."""

    def __getattr__(self, name):
        return lambda *args: None


@pytest.fixture
def fallback():
    """Calls a function on the path that the extension leaves to Python."""
    def run(f):
        kept = binding.load_operators()
        binding._ops = _Nothing()
        try:
            return f()
        finally:
            binding._ops = kept
    return run


def off(t, by):
    """The same values, packed, `by` elements behind a 16-byte boundary."""
    flat = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")[by:]
    return flat.view(t.shape).copy_(t)


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def calls(g, kind, wkind, n, rows, h, by):
    """Functions that run each operator forward and backward on inputs `by` elements off."""
    def rand(*shape, dtype=F32):
        return off(torch.randn(*shape, generator=g, device="cuda").to(dtype), by)

    x, res, dy, ds = rand(n, rows, h, dtype=kind), rand(n, rows, h, dtype=wkind), rand(n, rows, h, dtype=kind), rand(n, rows, h, dtype=wkind)
    p = [rand(n, h) for _ in range(3)]
    w, t = rand(70, h, dtype=wkind), off(torch.randint(0, 70, (n, rows), generator=g, device="cuda"), by)

    def norm():
        a = [v.detach().requires_grad_() for v in (x, p[0])]
        y = rms_norm(*a)
        return [y.detach(), *torch.autograd.grad(y, a, dy)]

    def gated():
        a = [v.detach().requires_grad_() for v in (x, res, *p)]
        y, s = gated_add_rms_norm(*a, residual_scale=0.5)
        return [y.detach(), s.detach(), *torch.autograd.grad((y, s), a, (dy, ds))]

    def head():
        a = [v.detach().requires_grad_() for v in (x, w)]
        loss = linear_cross_entropy(*a, t)
        return [loss.detach(), *torch.autograd.grad(loss.sum(), a)]

    def collect():
        return list(collect_gradients([x, res, *p], max_norm=3.0))

    return {"norm": norm, "gated": gated, "head": head, "collect": collect}


@pytest.mark.parametrize("kinds", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)], ids=str)
@pytest.mark.parametrize("rows,h", [(1, 64), (70, 64), (40, 1032), (5, 9000)])
def test_where_a_packed_tensor_starts_does_not_matter(rows, h, kinds, fallback):
    at = [calls(torch.Generator(device="cuda").manual_seed(h), *kinds, 2, rows, h, by) for by in (0, 1, 2)]
    for name in at[0]:
        base = at[0][name]()
        assert same(fallback(at[0][name]), base), name
        for other in at[1:]:
            got = other[name]()
            assert same(fallback(other[name]), got), name
            # A sum over a row's columns is taken in another order where they are not read 16 bytes at a time. The head's logits are then off
            # from each other by 2 (h / 512 + 64) 2^-24 of the sum of |x w| (blocks64), which is 2 h / pi here, and exponentials of them
            # relatively by as much, as far as they are below 1
            most = min(1.0, (h / 512 + 64) * 2.0 ** -23 * 0.64 * h) if name == "head" else 0.0
            for a, b in zip(got, base):
                scale = b.double().norm()
                assert float((a.double() - b.double()).norm()) <= (2 * torch.finfo(b.dtype).eps + most) * float(scale), name


def test_inference_mode_and_no_grad():
    f = calls(torch.Generator(device="cuda").manual_seed(1), BF16, F32, 2, 9, 72, 0)
    want = {k: v() for k, v in f.items()}
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w, t = torch.randn(2, 9, 72, generator=g, device="cuda"), torch.randn(30, 72, generator=g, device="cuda"), torch.zeros(2, 9, dtype=torch.int64, device="cuda")
    plain = rms_norm(x), *gated_add_rms_norm(x, x), linear_cross_entropy(x, w, t), *collect_gradients([x], max_norm=1.0)
    for mode in (torch.inference_mode, torch.no_grad):
        with mode():
            got = rms_norm(x), *gated_add_rms_norm(x, x), linear_cross_entropy(x, w, t), *collect_gradients([x], max_norm=1.0)
            out = torch.zeros(2, 9 * 72, device="cuda")
            collect_gradients([x], out=out, max_norm=1.0)
        assert same(got, plain) and torch.equal(out, plain[-2])
    with torch.no_grad():
        y = rms_norm(x.requires_grad_())
    assert not y.requires_grad
    assert all(same(v(), want[k]) for k, v in f.items())


def test_a_backward_pass_taken_twice_and_values_changed_in_between():
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = (torch.randn(2, 20, 64, generator=g, device="cuda").requires_grad_(), torch.randn(50, 64, generator=g, device="cuda").requires_grad_())
    t = torch.randint(0, 50, (2, 20), generator=g, device="cuda")
    for f in (lambda v: linear_cross_entropy(v, w, t).sum(), lambda v: rms_norm(v).square().sum(), lambda v: gated_add_rms_norm(v, v)[0].square().sum()):
        y = f(x)
        first, = torch.autograd.grad(y, x, retain_graph=True)
        again, = torch.autograd.grad(y, x, retain_graph=True)
        assert torch.equal(first, again)
        v = x * 1.0
        y = f(v)
        with torch.no_grad():
            v.add_(1.0)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    v = x * 1.0
    y, s = gated_add_rms_norm(v, v)
    with torch.no_grad():
        s.add_(1.0)  # the backward pass reads it
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_threads_at_once():
    sets = [calls(torch.Generator(device="cuda").manual_seed(k), (F32, BF16)[k % 2], F32, 2, 33, 136, 0) for k in range(4)]
    want = [{k: v() for k, v in s.items()} for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                for name, f in sets[k].items():
                    got = f()
                    torch.cuda.current_stream().synchronize()
                    if not same(got, want[k][name]):
                        wrong.append((k, name))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not wrong


def test_a_library_that_is_missing_is_said(monkeypatch):
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_ops", None)
    monkeypatch.setattr(binding, "library_path", lambda: "/nowhere/libcompams.so")
    with pytest.raises(binding.CompAMSError, match="not found"):
        rms_norm(torch.zeros(2, 3, 8, device="cuda"))
