"""The operators' refusals, sizes and generator, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import operators64 as R
from paper_2205_05632_b200 import CompAMSError, load_library
from paper_2205_05632_b200.layers import dropout, dropout_add_layer_norm, layer_norm, low_rank_adapter


@pytest.fixture(scope="module")
def lib():
    from paper_2205_05632_b200 import build
    build.build()
    return load_library()


def test_the_generator_is_philox():
    """The published known answers of Philox4x32-10."""
    for counter, key, want in (((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
                                (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(w) for w in R.philox(counter, key)) == want


def test_the_mask_keeps_its_share():
    f = R.factor(2, 64, 1000, 0.25, seed=3, call=1)
    assert abs(float((f != 0).double().mean()) - 0.75) < 6 * (0.1875 / f.numel()) ** 0.5
    assert set(np.unique(f.numpy())) == {0.0, 65536.0 / 49152.0}


def test_host_tensors_are_refused():
    x = torch.zeros(2, 3, 8)
    for call in (lambda: dropout(x, 0.1), lambda: layer_norm(x), lambda: dropout_add_layer_norm(x, x),
                 lambda: low_rank_adapter(x, None, torch.zeros(2, 8), torch.zeros(4, 2))):
        with pytest.raises(CompAMSError):
            call()
    for bad in (None, 3, [1.0]):
        with pytest.raises(CompAMSError):
            layer_norm(bad)


A = 4096  # an aligned address that no refused call looks at


def dropout_args(**kw):
    v = dict(y=A, x=A, type=0, n=2, rows=3, h=8, ws=24, rs=8, p=0.1, seed=1, call=0, call_device=None, worker=0, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(y=None), dict(x=None), dict(type=3), dict(type=-1), dict(n=0), dict(n=65536), dict(rows=-1), dict(h=0),
                                 dict(h=1 << 31), dict(rows=1 << 31), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(x=A + 2),
                                 dict(y=A + 1), dict(call_device=A + 4), dict(type=1, x=A + 1), dict(ws=-24), dict(rs=-8)])
def test_dropout_refuses(lib, bad):
    assert lib.compams_dropout(*dropout_args(**bad)) == -1


def forward_args(**kw):
    v = dict(y=A, s=None, stats=A, x=A, residual=None, type=1, rtype=0, n=2, rows=3, h=8, ws=24, rs=8, rws=24, rrs=8, weight=A, wst=0, bias=A,
             bst=0, eps=1e-5, p=0.0, seed=1, call=0, call_device=None, worker=0, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(y=None), dict(x=None), dict(type=7), dict(n=0), dict(h=0), dict(rows=-2), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(p=0.5), dict(s=A), dict(residual=A), dict(residual=A, s=A, type=0, rtype=1), dict(residual=A, s=A, rtype=2),
                                 dict(residual=A + 2, s=A, rtype=0), dict(weight=A + 1), dict(bias=A + 2), dict(stats=A + 4), dict(x=A + 1), dict(rs=-8),
                                 dict(wst=-8), dict(bst=-8), dict(residual=A, s=A, rws=-24)])
def test_norm_forward_refuses(lib, bad):
    assert lib.compams_norm_forward(*forward_args(**bad)) == -1


def backward_args(**kw):
    v = dict(dx=A, dres=None, dw=A, db=A, sum=0, dy=A, ds=None, v=A, stats=A, type=1, vtype=1, n=2, rows=3, h=8, gws=24, grs=8, sws=0, srs=0,
             vws=24, vrs=8, weight=A, wst=0, added=0, p=0.0, seed=1, call=0, call_device=None, worker=0, work=A, bytes=1 << 30, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(dy=None), dict(v=None), dict(stats=None), dict(vtype=0), dict(ds=A), dict(dres=A), dict(p=0.1), dict(work=None),
                                 dict(bytes=16), dict(work=A + 8), dict(dw=A + 2), dict(added=1, vtype=2), dict(n=0), dict(h=0), dict(dx=A + 1), dict(gws=-1),
                                 dict(vrs=-8), dict(wst=-1)])
def test_norm_backward_refuses(lib, bad):
    assert lib.compams_norm_backward(*backward_args(**bad)) == -1


def adapter_args(**kw):
    v = dict(y=A, t=A, x=A, base=A, type=1, n=2, rows=30, inn=8, out=8, rank=4, xws=240, xrs=8, bws=240, brs=8, a=A, aws=0, ars=8, b=A, bbws=0, bbrs=4,
             scale=1.0, p=0.0, seed=1, call=0, call_device=None, worker=0, work=A, bytes=1 << 30, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(y=None), dict(work=None), dict(bytes=16), dict(work=A + 8), dict(t=None), dict(x=None), dict(a=None), dict(b=None), dict(type=4), dict(n=0), dict(rows=-1), dict(inn=0),
                                 dict(out=0), dict(rank=0), dict(rank=1025), dict(p=2.0), dict(a=A + 2), dict(b=A + 1), dict(t=A + 2), dict(x=A + 1),
                                 dict(base=A + 1), dict(y=A + 1), dict(xrs=-8), dict(bws=-1), dict(aws=-1), dict(ars=-8), dict(bbws=-1), dict(bbrs=-4)])
def test_adapter_forward_refuses(lib, bad):
    assert lib.compams_adapter_forward(*adapter_args(**bad)) == -1


def adapter_backward_args(**kw):
    v = dict(dx=A, da=A, db=A, sum=0, dy=A, x=A, t=A, type=1, n=2, rows=30, inn=8, out=8, rank=4, gws=240, grs=8, xws=240, xrs=8, a=A, aws=0, ars=8, b=A,
             bws=0, brs=4, scale=1.0, p=0.0, seed=1, call=0, call_device=None, worker=0, work=A, bytes=1 << 30, stream=None)
    v.update(kw)
    return list(v.values())


@pytest.mark.parametrize("bad", [dict(dy=None), dict(x=None), dict(t=None), dict(a=None), dict(b=None), dict(work=None), dict(bytes=64), dict(work=A + 4),
                                 dict(rank=0), dict(da=A + 2), dict(db=A + 1), dict(dx=A + 1), dict(dy=A + 1), dict(grs=-8), dict(xws=-1),
                                 dict(ars=-1), dict(bws=-1)])
def test_adapter_backward_refuses(lib, bad):
    assert lib.compams_adapter_backward(*adapter_backward_args(**bad)) == -1


def test_nothing_to_do_is_done(lib):
    assert lib.compams_dropout(*dropout_args(rows=0)) == 0
    assert lib.compams_norm_forward(*forward_args(rows=0)) == 0
    assert lib.compams_adapter_forward(*adapter_args(rows=0)) == 0


def test_workspaces(lib):
    need = ctypes.c_size_t(0)
    assert lib.compams_norm_workspace_bytes(ctypes.byref(need), 4, 100, 512) == 0 and need.value >= 4 * 2 * 512 * 4
    assert lib.compams_norm_workspace_bytes(None, 4, 100, 512) == -1
    assert lib.compams_norm_workspace_bytes(ctypes.byref(need), 0, 100, 512) == -1
    assert lib.compams_adapter_workspace_bytes(ctypes.byref(need), 4, 100, 512, 256, 16, 1, 1, 0) == 0 and need.value >= 4 * 100 * 16 * 4
    assert lib.compams_adapter_workspace_bytes(ctypes.byref(need), 4, 1, 512, 256, 16, 0, 0, 0) == 0 and need.value == 0
    assert lib.compams_adapter_workspace_bytes(ctypes.byref(need), 4, 100, 512, 256, 0, 1, 1, 0) == -1
