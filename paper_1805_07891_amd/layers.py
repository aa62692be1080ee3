"""The worker's operators on torch tensors.

Plumbing only, as ``job``: torch allocates the outputs and workspaces, and
these functions check the tensors and pass their pointers to the HIP library
(``include/phub.h`` has the formulas).  Each call is ordered on torch's
current stream of the tensors' device.  Weight gradients are fp32 and written
(or added) where the caller says, such as ``TorchJob.gradient(worker, key)``,
the part of a worker's arena that it pushes.
A job has a stream of its own: the current stream waits for it before a call
reads its weights or writes an arena, and it for the current stream before the
push.  Autograd records nothing of these calls, whatever their inputs require:
the gradients are what the backward calls return and write.

Matrices are 2-D with adjacent columns; their rows may lie further apart than
they are long, but not overlap.
``workspace`` (a contiguous uint8 tensor, ``vocab_workspace``) is allocated
where it is not given.  Calls that share one must be ordered on one stream.
"""

from __future__ import annotations

import functools
from typing import Optional

from . import phub as _phub
from .job import load_library

import torch

_TYPES = {torch.float32: _phub.PHUB_F32, torch.bfloat16: _phub.PHUB_BF16,
          torch.float16: _phub.PHUB_F16}
_FP32 = torch.float32
# (the tensors are on a GPU already where these are called)
_empty, _current_device = torch.empty, torch._C._cuda_getDevice
_stream_of = torch._C._cuda_getCurrentRawStream
_default = None


def _library(lib):
    global _default
    if lib is not None:
        return lib
    if _default is None:
        _default = load_library()
    return _default


def _matrix(name, t, shape=None, dtype=None, device=None):
    """(pointer, distance of rows) of a matrix, checked."""
    size = t.shape
    if len(size) != 2 or (t.stride(1) != 1 and size[1] > 1):
        raise ValueError(f"{name} must be 2-D with adjacent columns")
    if shape is not None and size != shape:
        raise ValueError(f"{name} has shape {tuple(size)}, expected {tuple(shape)}")
    if (dtype is not None and t.dtype is not dtype) or not t.is_cuda or (
            device is not None and t.device != device):
        _wrong(name, t, dtype, device)
    # the stride of a matrix of one row says nothing
    return t.data_ptr(), (t.stride(0) if size[0] > 1 else size[1])


def _rows(x):
    """(type, device, pointer, distance of rows) of a matrix of hidden states."""
    kind = _TYPES.get(x.dtype)
    if kind is None:
        raise ValueError(f"{x.dtype} is not one of float32, bfloat16, float16")
    ptr, stride = _matrix("x", x)
    return kind, x.device, ptr, stride


def _vector(name, t, n, dtype, device):
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_cuda or t.device != device:
        _wrong(name, t, dtype, device)
    size = t.shape
    if len(size) != 1 or size[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be {n} adjacent values")
    return t.data_ptr()


def _wrong(name, t, dtype, device):
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} is {t.dtype}, expected {dtype}")
    raise ValueError(f"{name} is on {t.device}, expected {device or 'a GPU'}")


def _call(device, function, *args):
    """function(*args, torch's current stream of the device), on the device."""
    index = device.index
    before = _current_device()
    if before == index:
        return function(*args, _stream_of(index))
    torch.cuda.set_device(index)
    try:
        return function(*args, _stream_of(index))
    finally:
        torch.cuda.set_device(before)


@functools.lru_cache(maxsize=256)
def _norm_bytes(lib, rows, cols):
    return max(1, lib.phub_layer_norm_grad_bytes(rows, cols))


@functools.lru_cache(maxsize=256)
def _vocab_bytes(lib, *sizes):
    return lib.phub_vocab_bytes(*sizes)


def _workspace(workspace, device):
    """(pointer, bytes) of a workspace, checked."""
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    if workspace.device != device:
        _wrong("workspace", workspace, None, device)
    return workspace.data_ptr(), workspace.numel()


# -- layer norm ----------------------------------------------------------------
def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, lib=None):
    """(y, mean, rstd): every row of ``x`` normalised, times ``weight`` plus
    ``bias`` (fp32; None: ones, zeros), and what the backward pass needs."""
    lib = _library(lib)
    kind, dev, px, sx = _rows(x)
    rows, cols = x.shape
    pw = _vector("weight", weight, cols, _FP32, dev)
    pb = _vector("bias", bias, cols, _FP32, dev)
    y = _empty((rows, cols), dtype=x.dtype, device=dev)
    mean, rstd = _empty(rows, dtype=_FP32, device=dev), _empty(rows, dtype=_FP32, device=dev)
    _call(dev, lib.phub_layer_norm, kind, rows, cols, px, sx, pw, pb, eps, y.data_ptr(), cols,
          mean.data_ptr(), rstd.data_ptr())
    return y, mean, rstd


def layer_norm_grad(dy, x, weight, mean, rstd, dweight=None, dbias=None, accumulate: bool = False,
                    want_dx: bool = True, workspace=None, lib=None):
    """dx (or None).  ``dweight`` and ``dbias`` (fp32, each may be None)
    receive the sums over the rows, or have them added with ``accumulate``."""
    lib = _library(lib)
    kind, dev, px, sx = _rows(x)
    rows, cols = x.shape
    pdy, sdy = _matrix("dy", dy, x.shape, x.dtype, dev)
    pw = _vector("weight", weight, cols, _FP32, dev)
    pm, pr = _vector("mean", mean, rows, _FP32, dev), _vector("rstd", rstd, rows, _FP32, dev)
    pdw = _vector("dweight", dweight, cols, _FP32, dev)
    pdb = _vector("dbias", dbias, cols, _FP32, dev)
    dx = _empty((rows, cols), dtype=x.dtype, device=dev) if want_dx else None
    ptr, n = None, 0
    if pdw is not None or pdb is not None:
        if workspace is None:
            workspace = _empty(_norm_bytes(lib, rows, cols), dtype=torch.uint8, device=dev)
        ptr, n = _workspace(workspace, dev)
    _call(dev, lib.phub_layer_norm_grad, kind, rows, cols, pdy, sdy, px, sx, pw, pm, pr,
          None if dx is None else dx.data_ptr(), cols, pdw, pdb, 1 if accumulate else 0, ptr, n)
    return dx


# -- losses over a vocabulary --------------------------------------------------
def vocab_workspace(x, w, top: int = 0, grad: bool = True, most: Optional[int] = None, lib=None):
    """A workspace for the losses below (``top``: the teacher's entries a row,
    0 for targets; ``grad``: for the backward pass): as large as a call has
    use for, or of ``most`` bytes if that is less and enough.  The backward
    pass's is enough for the forward pass of the same sizes."""
    least, best = _library(lib).phub_vocab_bytes(*_sizes(x, w), top, 1 if grad else 0)
    n = best if most is None else max(least, min(best, int(most)))
    return _empty(n, dtype=torch.uint8, device=x.device)


def _sizes(x, w):
    kind, dev, px, sx = _rows(x)
    pw, sw = _matrix("w", w, None, x.dtype, dev)
    if w.shape[1] != x.shape[1]:
        raise ValueError(f"x has {x.shape[1]} columns, w {w.shape[1]}")
    return kind, x.shape[0], x.shape[1], w.shape[0], px, sx, pw, sw


def _teacher(x, index, logits, temperature):
    pi, _ = _matrix("index", index, None, torch.int64, x.device)
    if index.shape[0] != x.shape[0]:
        raise ValueError(f"index has {index.shape[0]} rows, x {x.shape[0]}")
    pl, _ = _matrix("logits", logits, index.shape, _FP32, x.device)
    if not index.is_contiguous() or not logits.is_contiguous():
        raise ValueError("index and logits must be contiguous")
    return index.shape[1], pi, pl, float(temperature)


def _space(lib, sizes, top, grad, workspace, device):
    """(pointer, bytes, tensor to keep) of the given workspace or a new one."""
    if workspace is None:
        kind, rows, cols, vocab, px, sx, pw, sw = sizes
        # (of the pointers only the alignment counts)
        n = _vocab_bytes(lib, kind, rows, cols, vocab, px % 16, sx, pw % 16, sw, top, grad)[1]
        workspace = _empty(n, dtype=torch.uint8, device=device)
    return (*_workspace(workspace, device), workspace)


def _forward(lib, call, x, w, targets, top, workspace):
    sizes, dev, rows = _sizes(x, w), x.device, x.shape[0]
    loss, lse = _empty(rows, dtype=_FP32, device=dev), _empty(rows, dtype=_FP32, device=dev)
    ptr, n, _keep = _space(lib, sizes, top, 0, workspace, dev)
    _call(dev, call, *sizes, *targets, loss.data_ptr(), lse.data_ptr(), ptr, n)
    return loss, lse


def _backward(lib, call, x, w, targets, top, lse, dloss, dw, accumulate, want_dx, workspace):
    sizes, dev, (rows, cols) = _sizes(x, w), x.device, x.shape
    plse = _vector("lse", lse, rows, _FP32, dev)
    pdl = _vector("dloss", dloss, rows, _FP32, dev)
    pdw, sdw = (None, 0) if dw is None else _matrix("dw", dw, w.shape, _FP32, dev)
    dx = _empty((rows, cols), dtype=x.dtype, device=dev) if want_dx else None
    ptr, n, _keep = _space(lib, sizes, top, 1, workspace, dev)
    _call(dev, call, *sizes, *targets, plse, pdl, None if dx is None else dx.data_ptr(), cols, pdw,
          sdw, 1 if accumulate else 0, ptr, n)
    return dx


def vocab_loss(x, w, target, workspace=None, lib=None):
    """(loss, lse) of every row: softmax cross entropy of ``target`` (int64)
    over the products of ``x`` with the rows of ``w`` (same type).  Rows whose
    target is not a row of ``w`` have loss 0."""
    lib = _library(lib)
    target = _vector("target", target, x.shape[0], torch.int64, x.device)
    return _forward(lib, lib.phub_vocab_loss, x, w, (target,), 0, workspace)


def vocab_loss_grad(x, w, target, lse, dloss=None, dw=None, accumulate: bool = False,
                    want_dx: bool = True, workspace=None, lib=None):
    """dx (or None) for ``dloss``, the gradient of every row's loss (None:
    ones); ``dw`` (fp32, may be None) receives w's gradient, or has it added
    with ``accumulate``."""
    lib = _library(lib)
    target = _vector("target", target, x.shape[0], torch.int64, x.device)
    return _backward(lib, lib.phub_vocab_loss_grad, x, w, (target,), 0, lse, dloss, dw, accumulate,
                     want_dx, workspace)


def distill_loss(x, w, index, logits, temperature: float = 1.0, workspace=None, lib=None):
    """(loss, lse) of every row: its divergence from a teacher whose entries
    ``index`` (int64) have ``logits`` (fp32), rows x entries, at
    ``temperature``.  Entries whose index is not a row of ``w`` or whose logit
    is -inf are absent; rows without entries have loss 0."""
    lib = _library(lib)
    targets = _teacher(x, index, logits, temperature)
    return _forward(lib, lib.phub_distill_loss, x, w, targets, targets[0], workspace)


def distill_loss_grad(x, w, index, logits, temperature, lse, dloss=None, dw=None,
                      accumulate: bool = False, want_dx: bool = True, workspace=None, lib=None):
    """As ``vocab_loss_grad``, for ``distill_loss``."""
    lib = _library(lib)
    targets = _teacher(x, index, logits, temperature)
    return _backward(lib, lib.phub_distill_loss_grad, x, w, targets, targets[0], lse, dloss, dw,
                     accumulate, want_dx, workspace)
