"""Refusals and sizes of the head, the root-mean-square norms and the clipped gradients, without a GPU."""
import ctypes

import pytest
import torch

from paper_2205_05632_b200 import CompAMSError, load_library
from paper_2205_05632_b200.layers import gated_add_rms_norm, linear_cross_entropy, rms_norm
from paper_2205_05632_b200.optim import clip_gradients, collect_gradients

A = 4096  # an aligned address that no refused call looks at
INVALID, TOO_LARGE = -1, -5


@pytest.fixture(scope="module")
def lib():
    from paper_2205_05632_b200 import build
    build.build()
    return load_library()


def test_host_tensors_are_refused():
    x, w, t = torch.zeros(2, 3, 8), torch.zeros(5, 8), torch.zeros(2, 3, dtype=torch.int64)
    for call in (lambda: linear_cross_entropy(x, w, t), lambda: rms_norm(x), lambda: gated_add_rms_norm(x, x), lambda: collect_gradients([x]),
                 lambda: clip_gradients([x], 1.0)):
        with pytest.raises(CompAMSError):
            call()


def forward_args(**kw):
    v = dict(loss=A, lse=A, x=A, type=1, weight=A, weight_type=1, target=A, n=2, rows=3, h=8, vocab=50, ws=24, rs=8, wws=0, wrs=8, ignored=-100,
             reduction=1, workspace=A, bytes=1 << 30, stream=None)
    v.update(kw)
    return list(v.values())


HEAD_BAD = [dict(x=None), dict(weight=None), dict(target=None), dict(lse=None), dict(type=3), dict(type=-1), dict(weight_type=2), dict(type=0),
            dict(n=0), dict(n=65536), dict(rows=-1), dict(rows=1 << 31), dict(h=0), dict(h=1 << 31), dict(vocab=0), dict(vocab=1 << 31),
            dict(ws=-1), dict(rs=-1), dict(wws=-1), dict(wrs=-1), dict(reduction=3), dict(reduction=-1), dict(workspace=None),
            dict(workspace=A + 16), dict(bytes=0), dict(x=A + 1), dict(weight=A + 1), dict(target=A + 4), dict(lse=A + 2)]


@pytest.mark.parametrize("bad", HEAD_BAD + [dict(loss=None), dict(loss=A + 2)], ids=str)
def test_head_forward_refuses(lib, bad):
    assert lib.compams_head_forward(*forward_args(**bad)) == INVALID


def backward_args(**kw):
    v = dict(dx=A, dweight=A, sum_workers=1, dloss=A, dws=1, drs=0, x=A, type=1, weight=A, weight_type=1, target=A, lse=A, n=2, rows=3, h=8, vocab=50,
             ws=24, rs=8, wws=0, wrs=8, ignored=-100, reduction=1, workspace=A, bytes=1 << 40, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", HEAD_BAD + [dict(dloss=None), dict(dloss=A + 2), dict(dws=-1), dict(drs=-1), dict(dx=A + 1), dict(dweight=A + 1),
                                            dict(wws=400)], ids=str)  # (the last: a weight of each worker's own has no sum over the workers)
def test_head_backward_refuses(lib, bad):
    assert lib.compams_head_backward(*backward_args(**bad)) == INVALID


def test_head_workspace(lib):
    def need(n, rows, h, vocab, type=1, weight_type=1, shared=1, x_copied=0, w_copied=0, wanted=0):
        b = ctypes.c_size_t(0)
        rc = lib.compams_head_workspace_bytes(ctypes.byref(b), n, rows, h, vocab, type, weight_type, shared, x_copied, w_copied, wanted)
        return b.value if rc == 0 else rc

    assert need(8, 1024, 4096, 100000) < 8 * 1024 * (100000 // 128 + 4) * 8          # statistics, not logits
    for vocab in (100000, 1000000):  # 512 MB of d, fp32 sums of dx, which do not grow with the vocabulary, and two numbers a row
        assert need(8, 1024, 4096, vocab, wanted=3) <= (512 << 20) + 8192 * 4096 * 4 + (1 << 20)
    assert need(1, 1, 4096, 32000) < 1 << 16                                          # a few rows: a number of CTAs' statistics
    for t, wt in ((1, 1), (2, 2), (0, 0), (1, 0), (2, 0)):
        for wanted in range(4):
            assert need(3, 0, 64, 100, t, wt, wanted=wanted) == 0
            most = need(3, 7, 64, 100, t, wt, x_copied=1, w_copied=1, wanted=wanted)
            assert 0 < need(3, 7, 64, 100, t, wt, wanted=wanted) <= most
    assert need(0, 1, 1, 1) == INVALID and need(1, 1, 0, 1) == INVALID and need(1, 1, 1, 1, 0, 1) == INVALID and need(1, 1, 1, 1, wanted=4) == INVALID
    assert lib.compams_head_workspace_bytes(None, 1, 1, 1, 1, 0, 0, 1, 0, 0, 0) == INVALID
    assert lib.compams_head_wait_tries(-1) == INVALID and lib.compams_head_wait_tries((1 << 14) + 1) == INVALID
    assert lib.compams_head_status(None) == INVALID


def norm_args(**kw):
    v = dict(y=A, s=A, stats=A, x=A, residual=A, type=1, residual_type=0, n=2, rows=3, h=8, ws=24, rs=8, rws=24, rrs=8, weight=A, weight_ws=8, gate=A,
             gate_ws=8, next=A, next_ws=8, scale=1.0, eps=1e-6, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(y=None), dict(x=None), dict(s=None), dict(residual=None), dict(type=3), dict(residual_type=2), dict(residual_type=1, type=0),
                                 dict(n=0), dict(n=65536), dict(rows=-1), dict(rows=1 << 31), dict(h=0), dict(h=1 << 31), dict(ws=-1), dict(rs=-1),
                                 dict(rws=-1), dict(rrs=-1), dict(weight_ws=-1), dict(gate_ws=-1), dict(next_ws=-1), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(x=A + 1), dict(residual=A + 2), dict(weight=A + 2), dict(gate=A + 1), dict(next=A + 3),
                                 dict(stats=A + 4), dict(y=A + 1), dict(residual=None, s=None), dict(residual=None, s=None, gate=None)], ids=str)
def test_norm_forward_refuses(lib, bad):
    assert lib.compams_rms_norm_forward(*norm_args(**bad)) == INVALID


def norm_backward_args(**kw):
    v = dict(dx=A, dresidual=A, dweight=A, dgate=A, dnext=A, sum_workers=0, dy=A, ds=A, x=A, s=A, stats=A, type=1, residual_type=0, n=2, rows=3, h=8,
             gws=24, grs=8, ews=24, ers=8, ws=24, rs=8, weight=A, weight_ws=8, gate=A, gate_ws=8, next=A, next_ws=8, scale=1.0, workspace=A,
             bytes=1 << 30, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(s=None), dict(stats=None), dict(type=3), dict(residual_type=2), dict(n=0), dict(rows=-1),
                                 dict(h=0), dict(gws=-1), dict(ers=-1), dict(ws=-1), dict(weight_ws=-1), dict(workspace=None), dict(workspace=A + 8),
                                 dict(bytes=0), dict(dweight=A + 2), dict(dgate=A + 1), dict(dnext=A + 2), dict(dx=A + 1), dict(dresidual=A + 2),
                                 dict(ds=A + 2), dict(stats=A + 4)], ids=str)
def test_norm_backward_refuses(lib, bad):
    assert lib.compams_rms_norm_backward(*norm_backward_args(**bad)) == INVALID


def test_norm_workspace(lib):
    b = ctypes.c_size_t(0)
    assert lib.compams_rms_norm_workspace_bytes(ctypes.byref(b), 2, 10, 100) == 0 and b.value >= 2 * 2 * 100 * 4
    assert lib.compams_rms_norm_workspace_bytes(None, 2, 10, 100) == INVALID
    assert lib.compams_rms_norm_workspace_bytes(ctypes.byref(b), 0, 10, 100) == INVALID


def collect_args(count=2, sizes=(3, 5), types=(0, 1), strides=None, tensors=None, offsets=None, **kw):
    offsets = offsets or [sum(sizes[:k]) for k in range(count + 1)]
    v = dict(rows=A, row_stride=offsets[-1], norms=A, tensors=(ctypes.c_void_p * count)(*(tensors or [A] * count)),
             strides=(ctypes.c_int64 * count)(*(strides or sizes)), types=(ctypes.c_int32 * count)(*types),
             offsets=(ctypes.c_int64 * (count + 1))(*offsets), count=count, n=2, max_norm=1.0, eps=1e-6, workspace=A, bytes=1 << 20, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(tensors=[A + 2, A]), dict(tensors=[A, A + 1]), dict(types=(0, 3)), dict(offsets=[0, 3, 3]), dict(offsets=[-1, 3, 8]),
                                 dict(strides=(-1, 5)), dict(n=0), dict(n=65536), dict(rows=A + 2), dict(norms=A + 2), dict(row_stride=7),
                                 dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(workspace=None), dict(workspace=A + 4),
                                 dict(bytes=8), dict(rows=None, strides=(2, 5)), dict(rows=None, norms=None, max_norm=float("inf"))], ids=str)
def test_collect_refuses(lib, bad):
    assert lib.compams_collect_workers(*collect_args(**bad)) == INVALID


def test_collect_refuses_what_is_missing(lib):
    for k in ("tensors", "strides", "types", "offsets"):
        args = dict(zip(("rows", "row_stride", "norms", "tensors", "strides", "types", "offsets", "count", "n", "max_norm", "eps", "workspace", "bytes", "stream"),
                        collect_args()))
        args[k] = None
        assert lib.compams_collect_workers(*args.values()) == INVALID
    assert lib.compams_collect_workers(*collect_args(n=65535, sizes=(1 << 30, 1 << 30))) == TOO_LARGE
    b = ctypes.c_size_t(0)
    assert lib.compams_collect_workers_workspace_bytes(ctypes.byref(b), 4, 1000) == 0 and b.value > 0
    assert lib.compams_collect_workers_workspace_bytes(ctypes.byref(b), 0, 1) == INVALID
    assert lib.compams_collect_workers_workspace_bytes(None, 1, 1) == INVALID


@pytest.mark.parametrize("parts, meet", [([(0, 8, 8, 4)], False), ([(0, 8, 8, 4), (0, 8, 8, 4)], True), ([(0, 8, 8, 4), (64, 8, 8, 4)], False),
                                         ([(64, 8, 8, 4), (0, 8, 8, 4)], False), ([(0, 8, 8, 4), (60, 8, 8, 4)], True),
                                         ([(0, 8, 5, 4), (20, 8, 3, 4)], False), ([(20, 8, 3, 4), (0, 8, 5, 4)], False),
                                         ([(0, 8, 6, 4), (20, 8, 3, 4)], True), ([(0, 8, 5, 4), (20, 16, 3, 2)], False),
                                         ([(0, 8, 5, 4), (20, 16, 7, 2)], True), ([(0, 8, 5, 4), (20, 9, 1, 4), (28, 8, 1, 4)], False),
                                         ([(0, 100, 50, 4), (200, 10, 3, 4)], False), ([], False)], ids=str)
def test_parts_that_overlap(parts, meet):
    """(address, elements from worker to worker, elements, bytes of one) of two workers' parts against every byte of them."""
    from paper_2205_05632_b200.optim import _overlap
    every = [b for a, stride, size, width in parts for i in range(2) for b in range(a + i * stride * width, a + (i * stride + size) * width)]
    assert (len(set(every)) < len(every)) == meet
    assert _overlap(2, *[[p[k] for p in parts] for k in range(4)]) == meet
