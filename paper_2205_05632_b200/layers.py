"""Operators for the layers of a torch model whose n workers' micro-batches run as one batch.

Activations are [n, ..., h], the worker on the leading axis, in float32, bfloat16 or float16. Weights are float32, as the optimizer
keeps them, and come in two forms: one for all workers ([h]), whose gradient is the sum over everything, or one per worker ([n, h]),
whose gradient stays apart by worker, row by row. CompAMSOptimizer.worker_parameters() gives the latter as leaves that are views of
the optimizer's parameter vector, and collect_all() makes their gradients the rows of G:

    w, b, A, B = opt.worker_parameters()                # [n, ...] each, all n rows are the one parameter
    for t in range(steps):
        y, s = dropout_add_layer_norm(x, residual, w, b, p=0.1, seed=seed, call=2 * t)
        z = low_rank_adapter(y, project(y), A, B, scale=2.0, p=0.1, seed=seed, call=2 * t + 1)
        ...
        loss = linear_cross_entropy(z, head, targets)   # [n], each worker's mean
        loss.sum().backward()
        opt.collect_all(max_norm=1.0)                   # every worker's gradient clipped by itself
        opt.step()

Dropout draws from a counter-based generator, Philox4x32-10: the bit of element (worker + i, row j, column c) of use number `call`
depends on these and the seed alone, so a mask is never stored, worker i's mask is the same whether it runs in a batch of workers or
alone (x[None] with worker=i), and a run that is taken up again draws on as before. `call` is a number below 2^32 that counts a
program's uses of the generator, or a one-element int64 CUDA tensor that holds it, which a captured graph reads at every replay; it has
to keep its value until the backward pass is done (add to it behind that).

The operators run on the current stream of x's device. They are differentiable once, backwards; their outputs are packed. Forward-mode
derivatives, torch.func's transforms and recording by make_fx are refused; torch.jit.trace records the operator as a Python function.
n is at most 65535. rms_norm, gated_add_rms_norm and linear_cross_entropy take their usual calls, packed tensors that nobody traces, through
an extension (binding.load_operators) and the others through this file: the same kernels and results, at a third of the host's time.

Forward and backward can be captured into a CUDA graph together. As with every torch backward pass, the leaves' gradient nodes belong to
the stream on which they were first used: warm up on the capturing stream, and let no autograd graph of the same leaves from another
stream live while capturing.

Not finite: a row of a norm with a NaN in it is NaN, and so are its gradients. An infinity makes a row of layer_norm NaN, too. In rms_norm its
reciprocal root is 0, as is that of a row whose squares are more than float32 holds (elements of 2^64): the row is 0, but NaN at the infinity; its
dx is NaN. gated_add_rms_norm keeps s = residual_scale * residual + 0 of such a row, NaN at the infinity, and where there is a NaN in s all of
the first result and the row's gradients are. A dropped element is 0 whatever it was. In
an adapter what an infinity or a NaN reaches is infinite or NaN, as a sum over it is, but which of the two may differ from a plain product.
NaN is also what a kernel of an adapter or of the head leaves whose bounded waits run out (compams_adapter_status, compams_head_status say so;
nothing should bring it about). In the head a row's NaN or infinity stays in its own loss and dx, and reaches all of its worker's dweight.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional, Tuple, Union

import torch
from torch.autograd import forward_ad

from .binding import CompAMSError, _check, load_library, load_operators

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
Call = Union[int, torch.Tensor]


def _rows(t: torch.Tensor) -> Tuple[torch.Tensor, int, int, int]:
    """(t or a copy that the kernels can walk, rows per worker, worker stride, row stride) of [n, ..., h]."""
    h = t.shape[-1]
    if t.is_neg():  # the negative of what lies in memory, the imaginary part of a conjugate for instance
        t = t.resolve_neg()
    if t.is_contiguous():
        rows = t.numel() // (t.shape[0] * h) if t.numel() else t[0].numel() // max(h, 1) if t.shape[0] else 0
        return t, rows, rows * h, h
    if t.stride(-1) != 1 and h > 1:
        return _rows(t.contiguous())
    if t.dim() == 2:
        return t, 1, t.stride(0), 0
    flat = t if t.dim() == 3 else t.reshape(t.shape[0], -1, h)  # (a copy only where the middle axes are no single stride)
    return flat, flat.shape[1], flat.stride(0), flat.stride(1)


def _like(t: torch.Tensor, x: torch.Tensor, what: str, dtypes=None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.device != x.device or t.dtype not in (dtypes or (x.dtype,)) or t.shape != x.shape:
        raise CompAMSError("%s must be a tensor like x: %s of type %s on %s" % (
            what, list(x.shape), " or ".join(str(d) for d in (dtypes or (x.dtype,))), x.device))
    return t


def _activation(x: torch.Tensor) -> None:
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in _TYPES:
        raise CompAMSError("x must be a float32, bfloat16 or float16 CUDA tensor")
    if x.dim() < 2 or x.shape[-1] < 1:
        raise CompAMSError("x must be [n, ..., h] with the worker on the leading axis and h >= 1: got %s" % list(x.shape))


def _factor(w: torch.Tensor, x: torch.Tensor, inner: Tuple[int, ...], what: str) -> torch.Tensor:
    """A float32 parameter of shape `inner`, for all workers or ([n, *inner]) for each; its last axis packed."""
    if not isinstance(w, torch.Tensor) or w.dtype is not torch.float32 or w.device != x.device or (
            w.shape != inner and w.shape != (x.shape[0], *inner)):
        raise CompAMSError("%s must be a float32 tensor %s or %s on %s" % (what, list(inner), [x.shape[0], *inner], x.device))
    if w.is_neg():
        w = w.resolve_neg()
    return w if w.stride(-1) == 1 or w.shape[-1] == 1 else w.contiguous()


def _affine(w: Optional[torch.Tensor]) -> Tuple[Optional[int], int]:
    return (None, 0) if w is None else (w.data_ptr(), w.stride(0) if w.dim() == 2 else 0)


class _Drop:
    """A checked p, seed, call and worker as the library takes them; call as a tensor is kept apart for the backward pass."""
    __slots__ = ("p", "seed", "call", "tensor", "worker")

    def __init__(self, x: torch.Tensor, p: float, seed: int, call: Call, worker: int):
        self.p, self.seed, self.worker, self.tensor = float(p), int(seed), int(worker), None
        if not 0.0 <= self.p <= 1.0:
            raise CompAMSError("p must be in [0, 1]: got %r" % (p,))
        if isinstance(call, torch.Tensor):
            if call.dtype != torch.int64 or call.numel() != 1 or call.device != x.device:
                raise CompAMSError("call must be a number or a one-element int64 tensor on %s" % x.device)
            self.call, self.tensor = 0, call.detach()
        else:
            self.call = int(call)
        if not 0 <= self.seed < 1 << 64 or not 0 <= self.call < 1 << 32:
            raise CompAMSError("seed must be in [0, 2^64) and call in [0, 2^32)")
        if not 0 <= self.worker <= (1 << 32) - max(1, x.shape[0]):
            raise CompAMSError("worker must be in [0, 2^32 - n]")

    def args(self):
        return self.p, self.seed, self.call, None if self.tensor is None else self.tensor.data_ptr(), self.worker


class _Nothing:
    """No dropout."""
    tensor = None

    @staticmethod
    def args():
        return 0.0, 0, 0, None, 0


_NOTHING = _Nothing()


def _run(name: str, device: torch.device, *args) -> None:
    fn = getattr(load_library(), name)
    index = device.index
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args, _stream(index))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream(index))
    if rc:
        _check(rc, name)


def _stream(index: int) -> int:
    """The current stream of a device, as the library takes it. (torch.cuda.current_stream(index).cuda_stream is the same number and
    takes 2 us, a tenth of a single token's layer norm.)"""
    return torch._C._cuda_getCurrentRawStream(index)


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(name: str, device: torch.device, *shape) -> int:
    need = ctypes.c_size_t(0)
    with torch.cuda.device(device):
        rc = getattr(load_library(), name)(ctypes.byref(need), *shape)
    if rc:
        _check(rc, name)
    return need.value


def _workspace(name: str, like: torch.Tensor, *shape) -> torch.Tensor:
    return like.new_empty(_workspace_bytes(name, like.device, *shape), dtype=torch.uint8)


def _once(backward):
    """A backward pass that is not differentiable itself. (torch's once_differentiable costs 8 us, and says no more than this where no
    graph of the backward pass is asked for.)"""
    guarded = torch.autograd.function.once_differentiable(backward)

    def run(ctx, *grads):
        if _has_tangent(grads):
            raise CompAMSError("forward-mode derivatives of a backward pass are not offered")
        return guarded(ctx, *grads) if torch.is_grad_enabled() else backward(ctx, *grads)

    return run


def _empty(like: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """Packed, of the same shape."""
    if dtype is None or dtype == like.dtype:
        return torch.empty_like(like) if like.is_contiguous() else like.new_empty(like.shape)
    return like.new_empty(like.shape, dtype=dtype)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _has_tangent(tensors) -> bool:
    return forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


_pre_dispatch_modes = torch._ops.mode_stack_state_for_pre_dispatch().count


def _through_autograd(*tensors) -> bool:
    """Whether a call goes through its autograd function: where a gradient is wanted, but also where torch.jit.trace would otherwise record
    the allocation of the result and nothing else (it records the function), and where a tensor carries a forward-mode tangent, which
    would be lost (the function refuses it). make_fx sees neither, so it is refused here."""
    if torch._C._len_torch_dispatch_stack() or _pre_dispatch_modes():
        from torch.fx.experimental.proxy_tensor import get_proxy_mode
        if get_proxy_mode() is not None:
            raise CompAMSError("make_fx cannot record this operator: it would keep the allocation of the result alone")
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        return True
    return torch._C._is_tracing() or _has_tangent(tensors)


# ---- dropout ---------------------------------------------------------------------------------------------------------------


def _dropout(x: torch.Tensor, drop: _Drop) -> torch.Tensor:
    y = _empty(x)
    if x.numel():
        v, rows, ws, rs = _rows(x)
        _run("compams_dropout", x.device, y.data_ptr(), v.data_ptr(), _TYPES[x.dtype], x.shape[0], rows, x.shape[-1], ws, rs,
             *drop.args())
    return y


class _DropoutFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, drop):
        ctx.drop = drop
        ctx.save_for_backward(*([drop.tensor] if drop.tensor is not None else []))
        return _dropout(x, drop)

    @staticmethod
    @_once
    def backward(ctx, dy):
        ctx.saved_tensors  # raises where the device-held call has been changed since
        return _dropout(dy, ctx.drop), None


def dropout(x: torch.Tensor, p: float, seed: int = 0, call: Call = 0, worker: int = 0) -> torch.Tensor:
    """Zeroes elements of x [n, ..., h] with probability p (rounded to a multiple of 2^-16) and divides the others by the share that
    is kept. Dropped elements are 0 whatever they were, NaN included; p = 0 copies."""
    _activation(x)
    drop = _Drop(x, p, seed, call, worker)
    return _DropoutFunction.apply(x, drop) if _through_autograd(x) else _dropout(x, drop)


# ---- layer norm ------------------------------------------------------------------------------------------------------------


def _norm_forward(x, residual, weight, bias, eps, drop, keep_stats):
    y = _empty(x)
    s = None if residual is None else _empty(x, residual.dtype)
    stats = x.new_empty((x.numel() // x.shape[-1], 2), dtype=torch.float32) if keep_stats else None
    if x.numel():
        v, rows, ws, rs = _rows(x)
        r, rws, rrs = None, 0, 0
        if residual is not None:
            r, _, rws, rrs = _rows(residual)
        _run("compams_norm_forward", x.device, y.data_ptr(), _ptr(s), _ptr(stats), v.data_ptr(), _ptr(r), _TYPES[x.dtype],
             0 if r is None else _TYPES[r.dtype], x.shape[0], rows, x.shape[-1], ws, rs, rws, rrs, *_affine(weight), *_affine(bias),
             eps, *drop.args())
    return y, s, stats


def _norm_backward(ctx, dy, ds, v, stats, weight, added):
    """(dx, dresidual, dweight, dbias) as ctx.needs_input_grad wants them."""
    needs_x, needs_r, needs_w, needs_b = ctx.wanted
    device, n, h = v.device, v.shape[0], v.shape[-1]
    apart = ctx.apart  # the workers' gradients stay apart
    dx = _empty(v, ctx.dtype) if needs_x else None
    dres = _empty(v) if needs_r else None
    make = v.new_empty if v.numel() else v.new_zeros
    dw = make((n, h) if apart else (h,), dtype=torch.float32) if needs_w else None
    db = make((n, h) if apart else (h,), dtype=torch.float32) if needs_b else None
    if v.numel():
        dy = v.new_zeros(v.shape, dtype=ctx.dtype) if dy is None else dy
        g, rows, gws, grs = _rows(dy)
        w, _, vws, vrs = _rows(v)
        e, ews, ers = None, 0, 0
        if ds is not None:
            e, _, ews, ers = _rows(ds)
        work = _workspace("compams_norm_workspace_bytes", v, n, rows, h) if needs_w or needs_b else None
        _run("compams_norm_backward", device, _ptr(dx), _ptr(dres), _ptr(dw), _ptr(db), 0 if apart else 1, g.data_ptr(), _ptr(e),
             w.data_ptr(), stats.data_ptr(), _TYPES[ctx.dtype], _TYPES[v.dtype], n, rows, h, gws, grs, ews, ers, vws, vrs,
             *_affine(weight), 1 if added else 0, *ctx.drop.args(), _ptr(work), 0 if work is None else work.numel())
    return dx, dres, dw, db


class _LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, _, stats = _norm_forward(x, None, weight, bias, eps, _NOTHING, True)
        ctx.save_for_backward(x, stats, *([weight] if weight is not None else []))
        ctx.drop, ctx.dtype, ctx.apart = _NOTHING, x.dtype, any(t is not None and t.dim() == 2 for t in (weight, bias))
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, stats, *weight = ctx.saved_tensors
        ctx.wanted = (ctx.needs_input_grad[0], False, *ctx.needs_input_grad[1:3])
        dx, _, dw, db = _norm_backward(ctx, dy, None, x, stats, weight[0] if weight else None, False)
        return dx, dw, db, None


class _AddNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps, drop):
        y, s, stats = _norm_forward(x, residual, weight, bias, eps, drop, True)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(s, stats, *([weight] if weight is not None else []), *([drop.tensor] if drop.tensor is not None else []))
        ctx.weighted = weight is not None
        ctx.drop, ctx.dtype, ctx.apart = drop, x.dtype, any(t is not None and t.dim() == 2 for t in (weight, bias))
        return y, s

    @staticmethod
    @_once
    def backward(ctx, dy, ds):
        s, stats, *more = ctx.saved_tensors
        ctx.wanted = ctx.needs_input_grad[:4]
        if dy is None and ds is None:
            return None, None, None, None, None, None
        return (*_norm_backward(ctx, dy, ds, s, stats, more[0] if ctx.weighted else None, True), None, None)


def _norm_parameters(x, weight, bias, eps):
    h = x.shape[-1]
    weight = None if weight is None else _factor(weight, x, (h,), "weight")
    bias = None if bias is None else _factor(bias, x, (h,), "bias")
    if weight is not None and bias is not None and weight.dim() != bias.dim():
        raise CompAMSError("weight and bias are both for all workers or both per worker")
    if not float(eps) >= 0.0:
        raise CompAMSError("eps must not be negative")
    return weight, bias, float(eps)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5) -> torch.Tensor:
    """(x - mean) / sqrt(var + eps) * weight + bias over the last axis of x [n, ..., h], in x's type; weight and bias are float32
    [h] or [n, h]."""
    _activation(x)
    weight, bias, eps = _norm_parameters(x, weight, bias, eps)
    if _through_autograd(x, weight, bias):
        return _LayerNormFunction.apply(x, weight, bias, eps)
    return _norm_forward(x, None, weight, bias, eps, _NOTHING, False)[0]


def dropout_add_layer_norm(x: torch.Tensor, residual: torch.Tensor, weight: Optional[torch.Tensor] = None,
                           bias: Optional[torch.Tensor] = None, p: float = 0.0, eps: float = 1e-5, seed: int = 0, call: Call = 0,
                           worker: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
    """(layer_norm(s), s) with s = residual + dropout(x). s has the residual's type, which is x's or float32, and is normalised as
    it is stored; the first result has x's type."""
    _activation(x)
    _like(residual, x, "residual", (x.dtype, torch.float32))
    weight, bias, eps = _norm_parameters(x, weight, bias, eps)
    drop = _Drop(x, p, seed, call, worker)
    if _through_autograd(x, residual, weight, bias):
        return _AddNormFunction.apply(x, residual, weight, bias, eps, drop)
    return _norm_forward(x, residual, weight, bias, eps, drop, False)[:2]


# ---- root-mean-square norms around a block ---------------------------------------------------------------------------------


def _unpacked(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A saved tensor that was packed: a hook of torch.autograd.graph.saved_tensors_hooks may give it back with other strides."""
    return None if t is None else t.resolve_neg().contiguous()


def _unpacked_columns(w: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A saved parameter whose last axis was packed."""
    return _unpacked(w) if w is not None and (w.is_neg() or w.stride(-1) != 1) else w


def _rms_forward(x, residual, weight, gate, after, scale, eps, keep_stats):
    y = _empty(x)
    s = None if residual is None else _empty(x, residual.dtype)
    stats = x.new_empty((x.numel() // x.shape[-1], 2), dtype=torch.float32) if keep_stats else None
    if x.numel():
        v, rows, ws, rs = _rows(x)
        r, rws, rrs = None, 0, 0
        if residual is not None:
            r, _, rws, rrs = _rows(residual)
        _run("compams_rms_norm_forward", x.device, y.data_ptr(), _ptr(s), _ptr(stats), v.data_ptr(), _ptr(r), _TYPES[x.dtype],
             0 if r is None else _TYPES[r.dtype], x.shape[0], rows, x.shape[-1], ws, rs, rws, rrs, *_affine(weight), *_affine(gate),
             *_affine(after), scale, eps)
    return y, s, stats


def _rms_backward(ctx, dy, ds, x, s, stats, weight, gate, after):
    """(dx, dresidual, dweight, dgate, dnext) as ctx.wanted wants them."""
    needs_x, needs_r, *needs = ctx.wanted
    n, h = x.shape[0], x.shape[-1]
    dx = _empty(x) if needs_x else None
    dres = _empty(s) if needs_r else None
    make = x.new_empty if x.numel() else x.new_zeros
    params = [make((n, h) if ctx.apart else (h,), dtype=torch.float32) if need else None for need in needs]
    if x.numel():
        dy = x.new_zeros(x.shape) if dy is None else dy
        g, rows, gws, grs = _rows(dy)
        v, _, ws, rs = _rows(x)
        e, ews, ers = None, 0, 0
        if ds is not None:
            e, _, ews, ers = _rows(ds)
        work = _workspace("compams_rms_norm_workspace_bytes", v, n, rows, h) if any(needs) else None
        _run("compams_rms_norm_backward", x.device, _ptr(dx), _ptr(dres), *map(_ptr, params), 0 if ctx.apart else 1, g.data_ptr(), _ptr(e),
             v.data_ptr(), _ptr(s), stats.data_ptr(), _TYPES[x.dtype], 0 if s is None else _TYPES[s.dtype], n, rows, h, gws, grs, ews, ers,
             ws, rs, *_affine(weight), *_affine(gate), *_affine(after), ctx.scale, _ptr(work), 0 if work is None else work.numel())
    return dx, dres, *params


class _RmsNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, eps):
        y, _, stats = _rms_forward(x, None, weight, None, None, 1.0, eps, True)
        ctx.save_for_backward(x, stats, *([weight] if weight is not None else []))
        ctx.apart, ctx.scale = weight is not None and weight.dim() == 2, 1.0
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, stats, *weight = ctx.saved_tensors
        ctx.wanted = (ctx.needs_input_grad[0], False, ctx.needs_input_grad[1], False, False)
        weight = _unpacked_columns(weight[0]) if weight else None
        dx, _, dw, _, _ = _rms_backward(ctx, dy, None, x, None, _unpacked(stats), weight, None, None)
        return dx, dw, None


class _GatedNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, gate, after, scale, eps):
        y, s, stats = _rms_forward(x, residual, weight, gate, after, scale, eps, True)
        ctx.set_materialize_grads(False)
        given = [t for t in (weight, gate, after) if t is not None]
        ctx.given = [t is not None for t in (weight, gate, after)]
        ctx.save_for_backward(x, s, stats, *given)
        ctx.apart, ctx.scale = any(t.dim() == 2 for t in given), scale
        return y, s

    @staticmethod
    @_once
    def backward(ctx, dy, ds):
        x, s, stats, *given = ctx.saved_tensors
        if dy is None and ds is None:
            return (None,) * 7
        ctx.wanted = ctx.needs_input_grad[:5]
        given = map(_unpacked_columns, given)
        return (*_rms_backward(ctx, dy, ds, x, _unpacked(s), _unpacked(stats), *[next(given) if there else None for there in ctx.given]), None, None)


def _rms_parameters(x, weight, gate, after):
    inner = x.shape[-1:]
    weight = None if weight is None else _factor(weight, x, inner, "weight")
    gate = None if gate is None else _factor(gate, x, inner, "gate")
    after = None if after is None else _factor(after, x, inner, "next_weight")
    dims = [p.dim() for p in (weight, gate, after) if p is not None]
    if dims and min(dims) != max(dims):
        raise CompAMSError("weight, gate and next_weight are all for all workers or all per worker")
    return weight, gate, after


def _epsilon(eps: float) -> float:
    eps = float(eps)
    if not eps >= 0.0:
        raise CompAMSError("eps must not be negative")
    return eps


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6) -> torch.Tensor:
    """x / sqrt(mean(x^2) + eps) * weight over the last axis of x [n, ..., h], in x's type; weight is float32 [h] or [n, h]."""
    y = None if forward_ad._current_level >= 0 else load_operators().rms_norm(x, weight, eps)
    if y is not None:  # a usual call; the others go through this file
        return y
    _activation(x)
    weight = None if weight is None else _factor(weight, x, x.shape[-1:], "weight")
    eps = _epsilon(eps)
    if _through_autograd(x, weight):
        return _RmsNormFunction.apply(x, weight, eps)
    return _rms_forward(x, None, weight, None, None, 1.0, eps, False)[0]


def gated_add_rms_norm(x: torch.Tensor, residual: torch.Tensor, weight: Optional[torch.Tensor] = None,
                       gate: Optional[torch.Tensor] = None, next_weight: Optional[torch.Tensor] = None, residual_scale: float = 1.0,
                       eps: float = 1e-6) -> Tuple[torch.Tensor, torch.Tensor]:
    """(rms_norm(s, next_weight), s) with s = residual_scale * residual + gate * rms_norm(x, weight): the norm behind a block, its gate, the
    residual stream and the norm before the next block. s has the residual's type, which is x's or float32, and is normalised as it is
    stored; the first result has x's type. weight, gate and next_weight are float32 [h], or all [n, h]; None: 1."""
    got = None if forward_ad._current_level >= 0 else load_operators().gated_add_rms_norm(x, residual, weight, gate, next_weight, residual_scale, eps)
    if got is not None:
        return got
    _activation(x)
    _like(residual, x, "residual", (x.dtype, torch.float32))
    args = (x, residual, *_rms_parameters(x, weight, gate, next_weight), float(residual_scale), _epsilon(eps))
    if _through_autograd(*args[:5]):
        return _GatedNormFunction.apply(*args)
    return _rms_forward(*args, False)[:2]


# ---- low-rank adapters -----------------------------------------------------------------------------------------------------


def _stacked(w: torch.Tensor) -> Tuple[int, int, int]:
    return (w.data_ptr(), w.stride(0), w.stride(1)) if w.dim() == 3 else (w.data_ptr(), 0, w.stride(0))


def _shared(a: torch.Tensor, b: torch.Tensor) -> int:
    """Whether all workers have one adapter, as the library counts it."""
    return int(a.dim() == 2 or a.shape[0] == 1 or (a.stride(0) == 0 and b.stride(0) == 0))


def _adapter_forward(x, base, a, b, scale, drop):
    n, rank, out = x.shape[0], a.shape[-2], b.shape[-2]
    y = x.new_empty((*x.shape[:-1], out)) if base is None else _empty(base)
    t = x.new_empty((x.numel() // x.shape[-1], rank), dtype=torch.float32)
    if x.numel():
        v, rows, ws, rs = _rows(x)
        z, zws, zrs = None, 0, 0
        if base is not None:
            z, _, zws, zrs = _rows(base)
        work = _workspace("compams_adapter_workspace_bytes", x, n, rows, x.shape[-1], out, rank, _shared(a, b), 0, 0)
        _run("compams_adapter_forward", x.device, y.data_ptr(), t.data_ptr(), v.data_ptr(), _ptr(z), _TYPES[x.dtype], n, rows,
             x.shape[-1], out, rank, ws, rs, zws, zrs, *_stacked(a), *_stacked(b), scale, *drop.args(), _ptr(work), work.numel())
    return y, t


class _AdapterFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, base, a, b, scale, drop):
        y, t = _adapter_forward(x, base, a, b, scale, drop)
        ctx.save_for_backward(x, t, a, b, *([drop.tensor] if drop.tensor is not None else []))
        ctx.scale, ctx.drop = scale, drop
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, t, a, b = ctx.saved_tensors[:4]
        needs_x, needs_base, needs_a, needs_b = ctx.needs_input_grad[:4]
        n, h, rank, out = x.shape[0], x.shape[-1], a.shape[-2], b.shape[-2]
        make = a.new_empty if x.numel() else a.new_zeros
        dx = _empty(x) if needs_x else None
        da = make(a.shape) if needs_a else None
        db = make(b.shape) if needs_b else None
        if x.numel() and (needs_x or needs_a or needs_b):
            g, rows, gws, grs = _rows(dy)
            v, _, ws, rs = _rows(x)
            work = _workspace("compams_adapter_workspace_bytes", x, n, rows, h, out, rank, _shared(a, b), 1,
                              0 if a.dim() == 3 else 1)
            _run("compams_adapter_backward", x.device, _ptr(dx), _ptr(da), _ptr(db), 0 if a.dim() == 3 else 1, g.data_ptr(),
                 v.data_ptr(), t.data_ptr(), _TYPES[x.dtype], n, rows, h, out, rank, gws, grs, ws, rs, *_stacked(a), *_stacked(b),
                 ctx.scale, *ctx.drop.args(), work.data_ptr(), work.numel())
        return dx, dy if needs_base else None, da, db, None, None


def low_rank_adapter(x: torch.Tensor, base: Optional[torch.Tensor], A: torch.Tensor, B: torch.Tensor, scale: float = 1.0,
                     p: float = 0.0, seed: int = 0, call: Call = 0, worker: int = 0) -> torch.Tensor:
    """base + scale (dropout(x) A^T) B^T: x is [n, ..., in], base, the projection that the adapter stands beside, [n, ..., out] in x's
    type or None for 0. A and B are float32, [rank, in] and [out, rank] for all workers or [n, rank, in] and [n, out, rank] for
    each worker (or request) of the leading axis; rank is at most 1024."""
    _activation(x)
    if not isinstance(A, torch.Tensor) or not isinstance(B, torch.Tensor) or A.dim() not in (2, 3) or B.dim() != A.dim():
        raise CompAMSError("A and B must be [rank, in] and [out, rank], or both with the workers in front")
    rank, out = A.shape[-2], B.shape[-2]
    if not 1 <= rank <= 1024 or out < 1:
        raise CompAMSError("rank must be in [1, 1024] and out at least 1: got %d, %d" % (rank, out))
    A, B = _factor(A, x, (rank, x.shape[-1]), "A"), _factor(B, x, (out, rank), "B")
    if base is not None and (not isinstance(base, torch.Tensor) or base.device != x.device or base.dtype != x.dtype
                             or tuple(base.shape) != (*x.shape[:-1], out)):
        raise CompAMSError("base must be %s of type %s on %s" % ([*x.shape[:-1], out], x.dtype, x.device))
    drop, scale = _Drop(x, p, seed, call, worker), float(scale)
    if _through_autograd(x, base, A, B):
        return _AdapterFunction.apply(x, base, A, B, scale, drop)
    return _adapter_forward(x, base, A, B, scale, drop)[0]


# ---- the head: cross entropy over a vocabulary -----------------------------------------------------------------------------

_REDUCTIONS = {"none": 0, "mean": 1, "sum": 2}


def _as_it_lies(p: int, h: int, rows: int, row_stride: int, batches: int, batch_stride: int) -> bool:
    """Whether TMA can read 16-bit rows where they are."""
    return (p % 16 == 0 and (rows == 1 or (row_stride % 8 == 0 and row_stride >= h))
            and (batches == 1 or (batch_stride % 8 == 0 and batch_stride >= 1)))


class _Head:
    """x, weight and target of a call as the library takes them."""
    __slots__ = ("x", "weight", "rows", "shape", "strides", "copied", "shared", "reduction", "ignored")

    def __init__(self, x, weight, reduction, ignored):
        n, h, vocab = x.shape[0], x.shape[-1], weight.shape[-2]
        self.x, self.rows, ws, rs = _rows(x)
        self.weight, self.reduction, self.ignored = weight, reduction, ignored
        wws = weight.stride(0) if weight.dim() == 3 and n > 1 else 0
        self.shared = wws == 0
        self.strides = (ws, rs, wws, weight.stride(-2))
        self.shape = (n, self.rows, h, vocab)
        x_copied = w_copied = True
        if x.dtype == torch.bfloat16 or (x.dtype == weight.dtype == torch.float16):
            if self.shared:
                stride = ws if self.rows == 1 else rs
                x_copied = not ((self.rows == 1 or n == 1 or ws == self.rows * rs)
                                and _as_it_lies(self.x.data_ptr(), h, n * self.rows, stride, 1, 0))
            else:
                x_copied = not _as_it_lies(self.x.data_ptr(), h, self.rows, rs, n, ws)
        if x.dtype == weight.dtype != torch.float32:
            w_copied = not _as_it_lies(weight.data_ptr(), h, vocab, weight.stride(-2), 1 if self.shared else n, wws)
        self.copied = (int(x_copied), int(w_copied))

    def workspace(self, wanted: int) -> torch.Tensor:
        return _workspace("compams_head_workspace_bytes", self.x, *self.shape, _TYPES[self.x.dtype], _TYPES[self.weight.dtype],
                          int(self.shared), *self.copied, wanted)


def _head_forward(x, weight, target, reduction, ignored):
    lse = x.new_empty(target.numel() + x.shape[0], dtype=torch.float32)  # and what each worker's rows count for
    make = x.new_empty if x.numel() else x.new_zeros
    loss = make(target.shape if reduction == 0 else x.shape[:1], dtype=torch.float32)
    if x.numel():
        z = _Head(x, weight, reduction, ignored)
        work = z.workspace(0)
        _run("compams_head_forward", x.device, loss.data_ptr(), lse.data_ptr(), z.x.data_ptr(), _TYPES[x.dtype], weight.data_ptr(),
             _TYPES[weight.dtype], target.data_ptr(), *z.shape, *z.strides, ignored, reduction, work.data_ptr(), work.numel())
    return loss, lse


class _HeadFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target, reduction, ignored):
        loss, lse = _head_forward(x, weight, target, reduction, ignored)
        ctx.save_for_backward(x, weight, target, lse)
        ctx.reduction, ctx.ignored = reduction, ignored
        return loss

    @staticmethod
    @_once
    def backward(ctx, dloss):
        x, weight, target, lse = ctx.saved_tensors
        weight, target, lse = _unpacked_columns(weight), _unpacked(target), _unpacked(lse)
        needs_x, needs_w = ctx.needs_input_grad[:2]
        dx = _empty(x) if needs_x else None
        dw = (weight.new_empty if x.numel() else weight.new_zeros)(weight.shape) if needs_w else None
        if x.numel() and (needs_x or needs_w):
            z = _Head(x, weight, ctx.reduction, ctx.ignored)
            g = dloss.resolve_neg()
            g = g if ctx.reduction else g.reshape(x.shape[0], -1)
            work = z.workspace((1 if needs_x else 0) + (2 if needs_w else 0))
            _run("compams_head_backward", x.device, _ptr(dx), _ptr(dw), 1 if weight.dim() == 2 else 0, g.data_ptr(), g.stride(0),
                 0 if ctx.reduction else g.stride(1), z.x.data_ptr(), _TYPES[x.dtype], weight.data_ptr(), _TYPES[weight.dtype],
                 target.data_ptr(), lse.data_ptr(), *z.shape, *z.strides, ctx.ignored, ctx.reduction, work.data_ptr(), work.numel())
        return dx, dw, None, None, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, reduction: str = "mean",
                         ignore_index: int = -100) -> torch.Tensor:
    """Softmax cross entropy of the logits x W^T with target, without the logits in memory as a whole: x is [n, ..., h], weight, which
    has x's type or float32, [vocab, h] for all workers or [n, vocab, h], target int64 [n, ...]. float32 results: "mean", [n], is over
    each worker's targets that are not ignore_index (0 where all are), "sum", [n], and "none", [n, ...], where an ignored target has 0.
    A target outside the vocabulary makes the loss NaN, and with it the gradients that it reaches.

    A float32 weight is taken as it is, in three products of bfloat16 for one (six where x is float32); a 16-bit weight in one."""
    number = _REDUCTIONS.get(reduction) if type(reduction) is str else None
    loss = None if forward_ad._current_level >= 0 else load_operators().linear_cross_entropy(x, weight, target, number, ignore_index)
    if loss is not None:
        return loss
    _activation(x)
    if number is None:
        raise CompAMSError("reduction must be one of %s: got %r" % (sorted(_REDUCTIONS), reduction))
    n, h = x.shape[0], x.shape[-1]
    if (not isinstance(weight, torch.Tensor) or weight.device != x.device or weight.dtype not in (x.dtype, torch.float32)
            or weight.dim() not in (2, 3) or weight.shape[-1] != h or weight.shape[-2] < 1 or (weight.dim() == 3 and weight.shape[0] != n)):
        raise CompAMSError("weight must be [vocab, %d] or [%d, vocab, %d] of type %s or float32 on %s" % (h, n, h, x.dtype, x.device))
    if not isinstance(target, torch.Tensor) or target.device != x.device or target.dtype != torch.int64 or target.shape != x.shape[:-1]:
        raise CompAMSError("target must be an int64 tensor %s on %s" % (list(x.shape[:-1]), x.device))
    if not -(1 << 63) <= int(ignore_index) < 1 << 63:
        raise CompAMSError("ignore_index must be a 64-bit number")
    if weight.is_neg():
        weight = weight.resolve_neg()
    if weight.stride(-1) != 1 and h > 1:
        weight = weight.contiguous()
    args = (x, weight, target.contiguous(), number, int(ignore_index))
    return _HeadFunction.apply(*args) if _through_autograd(x, weight) else _head_forward(*args)[0]
