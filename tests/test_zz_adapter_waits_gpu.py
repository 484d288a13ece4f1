"""The bounded waits of the adapters' kernels on tcgen05: none gave up in the tests before these (which is why this file comes late), and
what a call gives whose waits do. The limit is set to no tries at all, so every wait runs out, or to one, so some may."""
import ctypes

import pytest
import torch

import operators64 as R
from paper_2205_05632_b200 import load_library
from paper_2205_05632_b200.layers import low_rank_adapter

pytestmark = pytest.mark.gpu
MOST = 1 << 14


def gave_up():
    v = ctypes.c_int32(-1)
    assert load_library().compams_adapter_status(ctypes.byref(v)) == 0
    return v.value


def test_no_wait_gave_up_until_now():
    assert gave_up() == 0


@pytest.fixture
def tries():
    yield load_library().compams_adapter_wait_tries
    assert load_library().compams_adapter_wait_tries(MOST) == 0
    gave_up()


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("p", [0.0, 0.5])
@pytest.mark.parametrize("rank", [8, 24, 40, 130])
def test_waits_that_give_up_leave_nan(rank, p, shift, tries):
    n, rows, h, out = 2, 700, 1032, 520
    g = torch.Generator(device="cuda").manual_seed(rank)

    def rand(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    x = rand(n, rows, h + 8, dtype=torch.bfloat16)[..., shift:shift + h].detach().requires_grad_()  # shift 1: not by TMA
    base, dy = rand(n, rows, out, dtype=torch.bfloat16), rand(n, rows, out, dtype=torch.bfloat16)
    a, b = rand(n, rank, h).requires_grad_(), rand(n, out, rank).requires_grad_()
    kept = R.factor(n, rows, h, p, 3).cuda() != 0

    def both(backward_tries):
        y = low_rank_adapter(x, base, a, b, p=p, seed=3)
        assert tries(backward_tries) == 0
        return [y, *torch.autograd.grad(y, (x, a, b), dy)]

    right = both(MOST)
    assert gave_up() == 0 and all(torch.isfinite(t).all() for t in right)
    tries(0)
    y, dx, da, db = both(0)
    assert torch.isnan(y).all() and torch.isnan(da).all() and torch.isnan(db).all()
    assert torch.isnan(dx[kept]).all() and not dx[~kept].any()
    assert gave_up() == 1 and gave_up() == 0
    tries(MOST)
    y, dx, da, db = both(0)  # the backward pass alone
    assert torch.equal(y, right[0]) and gave_up() == 1
    assert torch.isnan(da).all() and torch.isnan(db).all() and torch.isnan(dx[kept]).all() and not dx[~kept].any()
    tries(1)
    for got, want in zip(both(1), right):  # some may give up
        assert (torch.isnan(got) | (got == want)).all()
    gave_up()
    tries(MOST)
    assert all(torch.equal(p, q) for p, q in zip(both(MOST), right)) and gave_up() == 0
