"""Calls at the operators' edges that need no GPU: what is refused, and what is done without a launch."""
import pytest

from paper_2205_05632_b200 import load_library
from test_operators import adapter_backward_args


@pytest.fixture(scope="module")
def lib():
    from paper_2205_05632_b200 import build
    build.build()
    return load_library()


@pytest.mark.parametrize("rows", [0, 1, 4, 5, 30, 200])
@pytest.mark.parametrize("type_", [0, 1, 2])
def test_an_adapters_backward_pass_without_a_wanted_gradient(lib, rows, type_):
    none = dict(dx=None, da=None, db=None, rows=rows, type=type_, gws=8 * rows, xws=8 * rows)
    assert lib.compams_adapter_backward(*adapter_backward_args(**none)) == 0
    if rows:
        assert lib.compams_adapter_backward(*adapter_backward_args(**dict(none, dy=None))) == -1  # arguments are looked at all the same
        assert lib.compams_adapter_backward(*adapter_backward_args(**dict(none, rank=0))) == -1


def test_tries_of_a_wait(lib):
    for bad in (-1, (1 << 14) + 1, 1 << 30):
        assert lib.compams_adapter_wait_tries(bad) == -1
    for good in (0, 1, 1 << 14):
        assert lib.compams_adapter_wait_tries(good) == 0
    assert lib.compams_adapter_status(None) == -1
