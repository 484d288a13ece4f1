"""What the operators do under torch's transforms: none may lose the operator or a derivative without a word. On the CPU the launches are
replaced by a stub; with a GPU the same runs for real."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2205_05632_b200 import CompAMSError, layers

pytestmark = pytest.mark.filterwarnings("ignore::torch.jit.TracerWarning", "ignore::DeprecationWarning")
N, ROWS, H = 2, 3, 8
BOTH = pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])


@pytest.fixture
def stub(request, monkeypatch):
    if request.getfixturevalue("device") == "cpu":
        monkeypatch.setattr(layers, "_activation", lambda x: None)
        monkeypatch.setattr(layers, "_run", lambda *a: None)
        monkeypatch.setattr(layers, "_workspace", lambda name, like, *shape: like.new_empty(16, dtype=torch.uint8))


def operands(device, seed=0):
    g = torch.Generator().manual_seed(seed)
    shapes = dict(x=(N, ROWS, H), r=(N, ROWS, H), w=(N, H), b=(N, H), base=(N, ROWS, 5), A=(N, 4, H), B=(N, 5, 4))
    return {k: torch.randn(*s, generator=g).to(device) for k, s in shapes.items()}


# the operator, and what it takes
OPERATORS = {
    "dropout": (lambda x: layers.dropout(x, 0.3, seed=5), ["x"]),
    "layer_norm": (lambda x, w, b: layers.layer_norm(x, w, b), ["x", "w", "b"]),
    "layer_norm without weights": (lambda x: layers.layer_norm(x), ["x"]),
    "dropout_add_layer_norm": (lambda x, r, w, b: torch.stack(layers.dropout_add_layer_norm(x, r, w, b, p=0.3, seed=5)), ["x", "r", "w", "b"]),
    "low_rank_adapter": (lambda x, base, A, B: layers.low_rank_adapter(x, base, A, B, scale=0.5, p=0.3, seed=5), ["x", "base", "A", "B"]),
    "low_rank_adapter without a base": (lambda x, A, B: layers.low_rank_adapter(x, None, A, B), ["x", "A", "B"]),
}
EACH = pytest.mark.parametrize("name", list(OPERATORS))


@BOTH
@EACH
@pytest.mark.parametrize("grad", [False, True])
def test_forward_mode_is_refused(name, device, grad, stub):
    fn, takes = OPERATORS[name]
    v = operands(device)
    with forward_ad.dual_level():
        for which in takes:
            args = [forward_ad.make_dual(v[k], torch.ones_like(v[k])) if k == which else v[k] for k in takes]
            with torch.set_grad_enabled(grad), pytest.raises((NotImplementedError, CompAMSError)):
                fn(*args)
        fn(*[v[k] for k in takes])  # without a tangent it is the ordinary call


@BOTH
@EACH
def test_a_tangent_of_the_incoming_gradient_is_refused(name, device, stub):
    fn, takes = OPERATORS[name]
    v = operands(device)
    args = [v[k].requires_grad_() for k in takes]
    y = fn(*args)
    with forward_ad.dual_level():
        dy = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises((NotImplementedError, CompAMSError)):
            torch.autograd.grad(y, args[0], dy)


@BOTH
@EACH
@pytest.mark.parametrize("grad", [False, True])
def test_a_traced_call_holds_the_operator(name, device, grad, stub):
    fn, takes = OPERATORS[name]
    v, other = operands(device), operands(device, 1)
    traced = torch.jit.trace(fn, tuple(v[k].clone().requires_grad_(grad) for k in takes), check_trace=False)
    assert "^_" in str(traced.graph)  # a Python function's node
    if device == "cuda":
        with torch.set_grad_enabled(grad):
            args = [other[k].clone().requires_grad_(grad) for k in takes]
            got, want = traced(*args), fn(*args)
            assert torch.equal(got, want)
            if grad:
                dy = torch.ones_like(want)
                for p, q in zip(torch.autograd.grad(got, args, dy), torch.autograd.grad(want, args, dy)):
                    assert torch.equal(p, q)


@BOTH
@EACH
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("pre_dispatch", [False, True])
def test_make_fx_is_refused(name, device, grad, pre_dispatch, stub):
    from torch.fx.experimental.proxy_tensor import make_fx
    fn, takes = OPERATORS[name]
    v = operands(device)
    with pytest.raises(CompAMSError):
        make_fx(fn, pre_dispatch=pre_dispatch)(*[v[k].requires_grad_(grad) for k in takes])


@BOTH
@EACH
@pytest.mark.parametrize("transform", ["vmap", "grad", "jvp"])
def test_transforms_of_functions_are_refused(name, device, transform, stub):
    fn, takes = OPERATORS[name]
    v = operands(device)
    args = tuple(v[k] for k in takes)
    with pytest.raises(Exception):
        if transform == "vmap":
            torch.vmap(fn)(*[torch.stack((t, t)) for t in args])
        elif transform == "grad":
            torch.func.grad(lambda *a: fn(*a).sum())(*args)
        else:
            torch.func.jvp(fn, args, tuple(torch.ones_like(t) for t in args))
