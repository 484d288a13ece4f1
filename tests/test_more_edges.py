"""Workspaces of the operators around a block and at the two ends of the backward pass, without a GPU."""
import ctypes

import pytest

from paper_2205_05632_b200 import load_library


@pytest.fixture(scope="module")
def lib():
    from paper_2205_05632_b200 import build
    build.build()
    return load_library()


@pytest.mark.parametrize("kinds", [(1, 1), (2, 2), (0, 0), (1, 0), (2, 0)], ids=str)
@pytest.mark.parametrize("n,rows,h,vocab", [(8, 1024, 4096, 100000), (8, 1024, 4096, 99999), (1, 1, 4096, 32000), (3, 7, 64, 100), (2, 30000, 64, 20000),
                                            (1, 300, 16384, 1000000), (16, 5, 2048, 50257), (4, 100, 512, 8000), (1, 4, 6144, 777)])
def test_a_head_workspace_for_copies_has_room_without_them(lib, n, rows, h, vocab, kinds):
    def need(shared, x_copied, weight_copied, wanted):
        b = ctypes.c_size_t(0)
        assert lib.compams_head_workspace_bytes(ctypes.byref(b), n, rows, h, vocab, *kinds, shared, x_copied, weight_copied, wanted) == 0
        return b.value

    for shared in (0, 1):
        for wanted in range(4):
            least = [need(shared, x, w, wanted) for x in (0, 1) for w in (0, 1)]
            assert need(shared, 1, 1, wanted) == max(least)
            assert need(shared, 0, 1, wanted) >= need(shared, 0, 0, wanted) and need(shared, 1, 0, wanted) >= need(shared, 0, 0, wanted)
