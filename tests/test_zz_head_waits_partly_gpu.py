"""Waits of the head's kernels with so few tries that some may run out and others not: what a call gives is then NaN or, to the bit, what it
gives otherwise. (Behind the tests that look whether a wait has given up before.)"""
import ctypes

import pytest
import torch

from paper_2205_05632_b200 import load_library
from paper_2205_05632_b200.layers import linear_cross_entropy

pytestmark = pytest.mark.gpu
MOST = 1 << 14


@pytest.fixture
def tries():
    L = load_library()
    yield L.compams_head_wait_tries
    assert L.compams_head_wait_tries(MOST) == 0
    assert L.compams_head_status(ctypes.byref(ctypes.c_int32())) == 0  # the flag is cleared


@pytest.mark.parametrize("kinds", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)], ids=str)
def test_results_are_right_or_nan(kinds, tries):
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(3, 700, 520, generator=g, device="cuda").to(kinds[0]).requires_grad_()
    w = (0.1 * torch.randn(9000, 520, generator=g, device="cuda")).to(kinds[1]).requires_grad_()
    t = torch.randint(0, 9000, (3, 700), generator=g, device="cuda")

    def both(forward, backward):
        assert tries(forward) == 0
        loss = linear_cross_entropy(x, w, t, "none")
        assert tries(backward) == 0
        return [loss.detach(), *torch.autograd.grad(loss.sum(), (x, w))]

    right = both(MOST, MOST)
    assert all(torch.isfinite(v).all() for v in right)
    for some in (1, 2, 3, 5, 9, 17):
        for got in (both(some, some), both(MOST, some)):
            for a, b in zip(got, right):
                assert torch.equal(torch.where(torch.isnan(a), b, a), b)
    assert all(torch.equal(a, b) for a, b in zip(both(MOST, MOST), right))
