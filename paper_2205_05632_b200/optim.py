"""COMP-AMS as the optimizer of a torch model: n workers = n micro-batches whose gradients are kept
apart, compressed separately with error feedback and averaged by the server (Algorithm 2).

The model's parameters are re-pointed at slices of one flat fp32 tensor theta, the vector Algorithm 2
updates; every parameter tensor is one block of the compressor ("the blocks are usually the layers",
Section 3.1) unless whole_vector is set. Per step:

    for i in range(n_workers):
        loss_i = ...            # forward / backward of worker i's micro-batch
        loss_i.backward()
        opt.collect(i)          # row i of G <- the gradients, which are then cleared
    opt.step()                  # one COMP-AMS iteration; the model's parameters move with theta

torch is used for the model and its autograd; the optimizer step itself runs in the CUDA library.
"""
from __future__ import annotations

import array
import ctypes
import functools
import itertools
from typing import Iterable, List, Optional, Sequence, Tuple, Union

import numpy as np
import torch

from .binding import RANDK, TOPK, CompAMS, CompAMSError, _check, load_library, load_operators

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_INFINITY = float("inf")


@functools.lru_cache(maxsize=256)
def _workspace_bytes(n: int, count: int) -> int:
    need = ctypes.c_size_t(0)
    _check(load_library().compams_collect_workers_workspace_bytes(ctypes.byref(need), n, count), "compams_collect_workers_workspace_bytes")
    return need.value


def _limit(max_norm: Optional[float], eps: float) -> Tuple[float, float]:
    limit, eps = _INFINITY if max_norm is None else float(max_norm), float(eps)
    if not limit >= 0.0 or not eps >= 0.0:
        raise CompAMSError("max_norm and eps must not be negative: got %r, %r" % (max_norm, eps))
    return limit, eps


def _collect_workers(rows: Optional[torch.Tensor], device: torch.device, n: int, addresses, strides, sizes, types, norms: bool, max_norm: float,
                     eps: float) -> Optional[torch.Tensor]:
    """compams_collect_workers on lists of the tensors' addresses (0: no gradient), elements from worker to worker, elements of a worker
    (none of them 0) and types."""
    got = torch.empty(n, dtype=torch.float32, device=device) if norms else None
    if not sizes:
        return None if got is None else got.zero_()
    count, index = len(sizes), device.index
    work = torch.empty(_workspace_bytes(n, count), dtype=torch.uint8, device=device) if norms or max_norm < _INFINITY else None
    lists = (array.array("Q", addresses), array.array("q", strides), array.array("i", types),
             array.array("q", itertools.accumulate(sizes, initial=0)))
    args = (None if rows is None else rows.data_ptr(), 0 if rows is None else rows.stride(0), None if got is None else got.data_ptr(),
            *[a.buffer_info()[0] for a in lists], count, n, max_norm, eps, None if work is None else work.data_ptr(),
            0 if work is None else work.numel(), torch._C._cuda_getCurrentRawStream(index))
    if torch._C._cuda_getDevice() == index:
        rc = load_library().compams_collect_workers(*args)
    else:
        with torch.cuda.device(device):
            rc = load_library().compams_collect_workers(*args)
    if rc:
        _check(rc, "compams_collect_workers")
    return got


def _changed(tensors) -> None:
    """Tells autograd, which would not know, that they are written."""
    tensors = [t for t in tensors if not t.is_inference()]
    if tensors:
        torch.autograd.graph.increment_version(tensors)


def _overlap(n: int, addresses, strides, sizes, widths) -> bool:
    """Whether two of the workers' parts (n of each tensor, its stride and size in elements of its width) have bytes in common."""
    if len(sizes) < 2:
        return False  # a tensor's own parts are apart: its stride has been looked at
    widths, starts = np.array(widths, dtype=np.int64), np.array(addresses, dtype=np.int64)
    steps, lengths = np.array(strides, dtype=np.int64) * widths, np.array(sizes, dtype=np.int64) * widths

    def meet(lo, length):
        order = np.argsort(lo)
        return bool((lo[order][1:] < (lo + length)[order][:-1]).any())

    if not meet(starts, (n - 1) * steps + lengths):
        return False
    return meet((starts[:, None] + steps[:, None] * np.arange(n)).ravel(), np.repeat(lengths, n))  # parts of one G, beside one another


_T = torch.Tensor


def _gradients(grads, what: str) -> Tuple[Sequence[torch.Tensor], int, torch.device, List[int]]:
    """The tensors, the number of workers, the device and the tensors' types. (Calls are mapped over the list: a model has hundreds.)"""
    grads = [grads] if isinstance(grads, torch.Tensor) else list(grads)
    if not grads or not all([isinstance(g, torch.Tensor) for g in grads]):
        raise CompAMSError("%s takes tensors, one at least" % what)
    device, n = grads[0].device, grads[0].shape[0] if grads[0].dim() else 0
    if device.type != "cuda" or not 1 <= n <= 65535:
        raise CompAMSError("gradients must be CUDA tensors with the workers, at most 65535, on the leading axis")
    types = [_TYPES.get(g.dtype, -1) for g in grads]
    if min(types) < 0 or set(map(_T.get_device, grads)) != {device.index} or not all(map(_T.dim, grads)) or not all([g.size(0) == n for g in grads]):
        raise CompAMSError("gradients must be float32, bfloat16 or float16 tensors [%d, ...] on %s: got %s" % (
            n, device, ", ".join("%s of type %s on %s" % (list(g.shape), g.dtype, g.device) for g in grads)))
    return grads, n, device, types


def _with_elements(sizes: List[int], *lists):
    """The lists without what belongs to tensors of no elements."""
    return [sizes, *lists] if all(sizes) else [[v for v, size in zip(of, sizes) if size] for of in (sizes, *lists)]


def collect_gradients(grads: Union[torch.Tensor, Sequence[torch.Tensor]], out: Optional[torch.Tensor] = None,
                      max_norm: Optional[float] = None, eps: float = 1e-6) -> Tuple[torch.Tensor, torch.Tensor]:
    """(G, norms): the workers' gradients, one tensor [n, *shape] per parameter in float32, bfloat16 or float16, gathered as the rows of a
    float32 tensor [n, d], `out` where given, and each worker's global norm over all of them, [n], as it was. Rows whose norm + eps is
    above max_norm are multiplied by max_norm / (norm + eps). The tensors may not lie between out's first and last element.
    Not recorded: as under torch.no_grad()."""
    got = load_operators().collect_gradients(grads, out, _INFINITY if max_norm is None else max_norm, eps)
    if got is not None:  # a usual call: a list of packed tensors
        return got
    grads, n, device, types = _gradients(grads, "collect_gradients")
    max_norm, eps = _limit(max_norm, eps)
    if not all(map(_T.is_contiguous, grads)) or any(map(_T.is_neg, grads)):
        grads = [g if g.is_contiguous() and not g.is_neg() else g.resolve_neg().contiguous() for g in grads]
    sizes = [k // n for k in map(_T.numel, grads)]
    d = sum(sizes)
    if out is None:
        out = torch.empty(n, d, dtype=torch.float32, device=device)
    elif (not isinstance(out, torch.Tensor) or out.dtype != torch.float32 or out.device != device or out.shape != (n, d)
          or (d > 1 and out.stride(1) != 1) or (n > 1 and out.stride(0) < d) or out.is_neg() or out.requires_grad):
        raise CompAMSError("out must be a float32 tensor [%d, %d] with packed rows on %s" % (n, d, device))
    else:
        lo = out.data_ptr()
        hi = lo + 4 * ((n - 1) * out.stride(0) + d)
        if any([g.data_ptr() < hi and lo < g.data_ptr() + g.numel() * g.element_size() for g in grads]):
            raise CompAMSError("the gradients must be apart from out")
        _changed([out])
    sizes, addresses, types = _with_elements(sizes, list(map(_T.data_ptr, grads)), types)
    return out, _collect_workers(out, device, n, addresses, sizes, sizes, types, True, max_norm, eps)


def clip_gradients(grads: Union[torch.Tensor, Sequence[torch.Tensor]], max_norm: float, eps: float = 1e-6) -> torch.Tensor:
    """Each worker's global norm, [n], over tensors [n, *shape] (G itself, or one tensor per parameter; every worker's part packed), which are
    scaled in place, worker by worker, by max_norm / (norm + eps) where norm + eps is above max_norm; the other workers' are not touched. No two
    tensors may have elements in common. Not recorded: as under torch.no_grad()."""
    grads, n, device, types = _gradients(grads, "clip_gradients")
    max_norm, eps = _limit(max_norm, eps)
    for g in grads:
        if g.is_neg() or not g[0].is_contiguous() or (n > 1 and g.stride(0) < g[0].numel()):
            raise CompAMSError("gradients that are clipped in place must be packed for every worker, and the workers' parts apart")
        if g.requires_grad and torch.is_grad_enabled() and (g.is_leaf or (g._base is not None and g._base.is_leaf)):
            raise CompAMSError("a leaf that requires a gradient, or a view of one, cannot be scaled in place")
    sizes, addresses, strides, types, widths = _with_elements([g.numel() // n for g in grads], [g.data_ptr() for g in grads],
                                                              [g.stride(0) for g in grads], types, [g.element_size() for g in grads])
    if _overlap(n, addresses, strides, sizes, widths):
        raise CompAMSError("gradients that are clipped in place must be apart from one another")
    _changed(grads)
    return _collect_workers(None, device, n, addresses, strides, sizes, types, True, max_norm, eps)


class CompAMSOptimizer:
    def __init__(self, params: Iterable[torch.nn.Parameter], n_workers: int, compressor: int = TOPK,
                 k_ratio: float = 0.01, whole_vector: bool = False, lr: float = 1e-3, beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, seed: int = 0):
        self.params: List[torch.nn.Parameter] = [p for p in params if p.requires_grad]
        if not self.params:
            raise CompAMSError("no trainable parameters")
        dev = self.params[0].device
        if dev.type != "cuda" or any(p.device != dev or p.dtype != torch.float32 for p in self.params):
            raise CompAMSError("all parameters must be float32 tensors on one CUDA device")
        sizes = [p.numel() for p in self.params]
        self.offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
        self.d = int(self.offsets[-1])
        self.n = int(n_workers)
        # theta: the flat parameter vector; the model's tensors become views of it
        self.theta = torch.empty(self.d, dtype=torch.float32, device=dev)
        for p, lo, hi in zip(self.params, self.offsets[:-1], self.offsets[1:]):
            self.theta[lo:hi].copy_(p.data.reshape(-1))
            p.data = self.theta[lo:hi].view(p.shape)
        self.G = torch.zeros(self.n, self.d, dtype=torch.float32, device=dev)
        # collect(): the tensors that have elements, their places in a row, and room for their gradients' addresses
        self._pieces = [(p, 4 * size) for p, size in zip(self.params, sizes) if size]
        self._sizes = sizes
        places = [int(o) for o, size in zip(self.offsets, sizes) if size] + [self.d]
        self._places = (ctypes.c_int64 * len(places))(*places)
        self._addresses = (ctypes.c_void_p * len(self._pieces))()
        self._leaves = None  # worker_parameters(): made when they are first asked for
        blocks = np.array([0, self.d], dtype=np.int64) if whole_vector else self.offsets
        with torch.cuda.device(dev):
            self.opt = CompAMS(self.n, self.d, blocks, compressor, k_ratio, lr, beta1, beta2, eps)
            if compressor == RANDK:
                self.opt.set_seed(seed)  # Random-k: the seed of the index sets

    def collect(self, worker: int) -> None:
        """Row `worker` of G <- the gradients accumulated since the last collect(); they are cleared."""
        if not 0 <= worker < self.n:
            raise CompAMSError("worker %d outside [0, %d)" % (worker, self.n))
        # one kernel for all tensors, which reads them by their addresses
        dev = self.G.device
        index = dev.index
        grads, addresses = [], []  # (the former keeps the packed copies until the kernel is enqueued)
        for p, nbytes in self._pieces:
            g = p.grad
            if g is not None:
                # not as the kernel reads it, after a model.half() or .cpu() for instance, channels-last, an expanded view; the
                # negative of what lies in memory (the imaginary part of a conjugate), which only one element can be and be packed
                if g.nbytes != nbytes or g.get_device() != index or not g.is_contiguous() or (nbytes == 4 and g.is_neg()):
                    if 4 * g.numel() != nbytes:
                        raise CompAMSError("a gradient of %d elements for a parameter of %d" % (g.numel(), nbytes // 4))
                    g = g.to(dev, torch.float32).resolve_neg().contiguous()
                grads.append(g)
            addresses.append(None if g is None else g.data_ptr())
        self._addresses[:] = addresses
        with torch.cuda.device(dev):
            stream = torch.cuda.current_stream(dev).cuda_stream
            _check(load_library().compams_collect(self.G.data_ptr() + 4 * self.d * worker, self._addresses, self._places,
                                                  len(addresses), stream), "compams_collect")
        for p in self.params:
            p.grad = None

    def worker_parameters(self) -> List[torch.Tensor]:
        """For models that run the n workers' micro-batches as one batch (the operators of .layers, or torch's batched products): per
        parameter a leaf [n, *shape] whose n rows are all the parameter itself, so that they move with theta, and whose .grad keeps the
        workers' gradients apart. The same leaves at every call; collect_all() takes their gradients."""
        if self._leaves is None:
            self._leaves = [self.theta[lo:hi].view(p.shape).expand(self.n, *p.shape).requires_grad_()
                            for p, lo, hi in zip(self.params, self.offsets[:-1], self.offsets[1:])]
        return self._leaves

    def collect_all(self, max_norm: Optional[float] = None, eps: float = 1e-6) -> Optional[torch.Tensor]:
        """All rows of G <- the gradients that worker_parameters() accumulated since the last call; they are cleared. With max_norm every
        worker's row whose norm over all parameters, with eps added, is above it is multiplied by max_norm / (norm + eps), and the norms, [n],
        are the result."""
        limit, eps = _limit(max_norm, eps)
        leaves = self.worker_parameters()
        dev = self.G.device
        grads = []
        for leaf in leaves:
            g = leaf.grad
            if g is not None and (g.dtype != torch.float32 or g.device != dev or not g.is_contiguous() or g.is_neg()):
                g = g.to(dev, torch.float32).resolve_neg().contiguous()
            grads.append(g)
        sizes, addresses = _with_elements(self._sizes, [0 if g is None else g.data_ptr() for g in grads])
        norms = _collect_workers(self.G, dev, self.n, addresses, sizes, sizes, [0] * len(sizes), max_norm is not None, limit, eps)
        for leaf in leaves:
            leaf.grad = None
        return norms

    def clip(self, max_norm: float, eps: float = 1e-6) -> torch.Tensor:
        """Between collect() of the workers and step(): rows of G whose norm + eps is above max_norm are multiplied by max_norm / (norm +
        eps). The norms, [n], as they were."""
        return clip_gradients(self.G, max_norm, eps)

    def step(self) -> None:
        self.opt.step(self.G, self.theta)

    def set_lr(self, lr: float) -> None:
        self.opt.set_lr(lr)

    def close(self) -> None:
        self.opt.close()
