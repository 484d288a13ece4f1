"""The bounded waits of the head's kernels on tcgen05: none gave up in the tests before these (which is why this file comes late), and what
a call gives whose waits do. The limit is set to no tries at all, so every wait runs out."""
import ctypes

import pytest
import torch

from paper_2205_05632_b200 import load_library
from paper_2205_05632_b200.layers import linear_cross_entropy

pytestmark = pytest.mark.gpu
MOST = 1 << 14


def gave_up():
    v = ctypes.c_int32(-1)
    assert load_library().compams_head_status(ctypes.byref(v)) == 0
    return v.value


def test_no_wait_gave_up_until_now():
    assert gave_up() == 0


@pytest.fixture
def tries():
    yield load_library().compams_head_wait_tries
    assert load_library().compams_head_wait_tries(MOST) == 0
    gave_up()


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_waits_that_give_up_leave_nan(kind, tries):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(2, 300, 264, generator=g, device="cuda").to(kind).requires_grad_()
    w = (0.1 * torch.randn(1000, 264, generator=g, device="cuda")).to(kind).requires_grad_()
    t = torch.randint(0, 1000, (2, 300), generator=g, device="cuda")

    def both(backward_tries):
        loss = linear_cross_entropy(x, w, t)
        assert tries(backward_tries) == 0
        return [loss, *torch.autograd.grad(loss.sum(), (x, w))]

    right = both(MOST)
    assert gave_up() == 0 and all(torch.isfinite(v).all() for v in right)
    tries(0)
    got = both(0)
    assert all(torch.isnan(v).all() for v in got)
    assert gave_up() == 1 and gave_up() == 0
    tries(MOST)
    got = both(0)  # going forward all is well, going back nothing is
    assert torch.equal(got[0], right[0]) and torch.isnan(got[1]).all() and torch.isnan(got[2]).all()
    assert gave_up() == 1
    tries(MOST)
    assert all(torch.equal(a, b) for a, b in zip(both(MOST), right)) and gave_up() == 0
