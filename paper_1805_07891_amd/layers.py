"""The worker's operators on torch tensors.

Plumbing only, as ``job``: torch allocates the outputs and workspaces, and
these functions check the tensors and pass their pointers to the HIP library
(``include/phub.h`` has the formulas).  Each call is ordered on torch's
current stream of the tensors' device.  Weight gradients are fp32 and written
(or added) where the caller says, such as ``TorchJob.gradient(worker, key)``,
the part of a worker's arena that it pushes.

Matrices are 2-D with adjacent columns; rows may be any distance apart.
``workspace`` (a contiguous uint8 tensor, ``vocab_workspace``) is allocated
where it is not given.  Calls that share one must be ordered on one stream.
"""

from __future__ import annotations

from typing import Optional

from . import phub as _phub
from .job import load_library

_types = None


def _type(x) -> int:
    global _types
    if _types is None:
        import torch
        _types = {torch.float32: _phub.PHUB_F32, torch.bfloat16: _phub.PHUB_BF16,
                  torch.float16: _phub.PHUB_F16}
    try:
        return _types[x.dtype]
    except KeyError:
        raise ValueError(f"{x.dtype} is not one of float32, bfloat16, float16") from None


def _matrix(name, t, shape=None, dtype=None, device=None):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D with adjacent columns")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    _same(name, t, dtype, device)
    # the stride of a matrix of one row says nothing
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _vector(name, t, n, dtype, device):
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be {n} adjacent values")
    _same(name, t, dtype, device)
    return t.data_ptr()


def _same(name, t, dtype, device):
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, expected {dtype}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} is on {t.device}, expected {device or 'a GPU'}")


class _On:
    """Makes a device current for a call and gives torch's current stream."""

    def __init__(self, device):
        import torch
        self.cuda, self.index = torch.cuda, device.index

    def __enter__(self):
        self.before = self.cuda.current_device()
        if self.before != self.index:
            self.cuda.set_device(self.index)
        return self.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *exc):
        if self.before != self.index:
            self.cuda.set_device(self.before)


def _bytes(workspace, n, device):
    """(pointer, bytes, tensor to keep) of a workspace of n bytes."""
    import torch
    if workspace is None:
        workspace = torch.empty(max(n, 1), dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    _same("workspace", workspace, None, device)
    return workspace.data_ptr(), workspace.numel(), workspace


# -- layer norm ----------------------------------------------------------------
def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, lib=None):
    """(y, mean, rstd): every row of ``x`` normalised, times ``weight`` plus
    ``bias`` (fp32; None: ones, zeros), and what the backward pass needs."""
    import torch
    lib = lib or load_library()
    dev, (rows, cols) = x.device, x.shape
    px, sx = _matrix("x", x)
    y = torch.empty(rows, cols, dtype=x.dtype, device=dev)
    stats = torch.empty(2, rows, dtype=torch.float32, device=dev)
    with _On(dev) as stream:
        lib.phub_layer_norm(_type(x), rows, cols, px, sx,
                            _vector("weight", weight, cols, torch.float32, dev),
                            _vector("bias", bias, cols, torch.float32, dev), eps, y.data_ptr(),
                            cols, stats.data_ptr(), stats.data_ptr() + 4 * rows, stream)
    return y, stats[0], stats[1]


def layer_norm_grad(dy, x, weight, mean, rstd, dweight=None, dbias=None, accumulate: bool = False,
                    want_dx: bool = True, workspace=None, lib=None):
    """dx (or None).  ``dweight`` and ``dbias`` (fp32, each may be None)
    receive the sums over the rows, or have them added with ``accumulate``."""
    import torch
    lib = lib or load_library()
    dev, (rows, cols) = x.device, x.shape
    px, sx = _matrix("x", x)
    pdy, sdy = _matrix("dy", dy, x.shape, x.dtype, dev)
    dx = torch.empty(rows, cols, dtype=x.dtype, device=dev) if want_dx else None
    space = (None, 0, None)
    if dweight is not None or dbias is not None:
        need = 0 if workspace is not None else lib.phub_layer_norm_grad_bytes(rows, cols)
        space = _bytes(workspace, need, dev)
    with _On(dev) as stream:
        lib.phub_layer_norm_grad(_type(x), rows, cols, pdy, sdy, px, sx,
                                 _vector("weight", weight, cols, torch.float32, dev),
                                 _vector("mean", mean, rows, torch.float32, dev),
                                 _vector("rstd", rstd, rows, torch.float32, dev),
                                 None if dx is None else dx.data_ptr(), cols,
                                 _vector("dweight", dweight, cols, torch.float32, dev),
                                 _vector("dbias", dbias, cols, torch.float32, dev),
                                 int(bool(accumulate)), space[0], space[1], stream)
    return dx


# -- losses over a vocabulary --------------------------------------------------
def vocab_workspace(x, w, top: int = 0, grad: bool = True, most: Optional[int] = None, lib=None):
    """A workspace for the losses below (``top``: the teacher's entries a row,
    0 for targets; ``grad``: for the backward pass): as large as a call has
    use for, or of ``most`` bytes if that is less and enough."""
    import torch
    lib = lib or load_library()
    least, best = lib.phub_vocab_bytes(*_sizes(x, w), top, int(bool(grad)))
    n = best if most is None else max(least, min(best, int(most)))
    return torch.empty(n, dtype=torch.uint8, device=x.device)


def _sizes(x, w):
    px, sx = _matrix("x", x)
    pw, sw = _matrix("w", w, None, x.dtype, x.device)
    if w.shape[1] != x.shape[1]:
        raise ValueError(f"x has {x.shape[1]} columns, w {w.shape[1]}")
    return _type(x), x.shape[0], x.shape[1], w.shape[0], px, sx, pw, sw


def _teacher(x, index, logits, temperature):
    import torch
    pi, _ = _matrix("index", index, (x.shape[0], index.shape[-1]), torch.int64, x.device)
    pl, _ = _matrix("logits", logits, index.shape, torch.float32, x.device)
    if not index.is_contiguous() or not logits.is_contiguous():
        raise ValueError("index and logits must be contiguous")
    return index.shape[1], pi, pl, float(temperature)


def _forward(call, x, w, targets, top, workspace, lib):
    import torch
    sizes, dev, rows = _sizes(x, w), x.device, x.shape[0]
    out = torch.empty(2, rows, dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = vocab_workspace(x, w, top, False, lib=lib)
    ptr, n, _keep = _bytes(workspace, 0, dev)
    with _On(dev) as stream:
        call(*sizes, *targets, out.data_ptr(), out.data_ptr() + 4 * rows, ptr, n, stream)
    return out[0], out[1]


def _backward(call, x, w, targets, top, lse, dloss, dw, accumulate, want_dx, workspace, lib):
    import torch
    sizes, dev, (rows, cols) = _sizes(x, w), x.device, x.shape
    plse = _vector("lse", lse, rows, torch.float32, dev)
    pdl = _vector("dloss", dloss, rows, torch.float32, dev)
    pdw, sdw = (None, 0) if dw is None else _matrix("dw", dw, w.shape, torch.float32, dev)
    dx = torch.empty(rows, cols, dtype=x.dtype, device=dev) if want_dx else None
    if workspace is None:
        workspace = vocab_workspace(x, w, top, True, lib=lib)
    ptr, n, _keep = _bytes(workspace, 0, dev)
    with _On(dev) as stream:
        call(*sizes, *targets, plse, pdl, None if dx is None else dx.data_ptr(), cols, pdw, sdw,
             int(bool(accumulate)), ptr, n, stream)
    return dx


def vocab_loss(x, w, target, workspace=None, lib=None):
    """(loss, lse) of every row: softmax cross entropy of ``target`` (int64)
    over the products of ``x`` with the rows of ``w`` (same type).  Rows whose
    target is not a row of ``w`` have loss 0."""
    import torch
    lib = lib or load_library()
    target = _vector("target", target, x.shape[0], torch.int64, x.device)
    return _forward(lib.phub_vocab_loss, x, w, (target,), 0, workspace, lib)


def vocab_loss_grad(x, w, target, lse, dloss=None, dw=None, accumulate: bool = False,
                    want_dx: bool = True, workspace=None, lib=None):
    """dx (or None) for ``dloss``, the gradient of every row's loss (None:
    ones); ``dw`` (fp32, may be None) receives w's gradient, or has it added
    with ``accumulate``."""
    import torch
    lib = lib or load_library()
    target = _vector("target", target, x.shape[0], torch.int64, x.device)
    return _backward(lib.phub_vocab_loss_grad, x, w, (target,), 0, lse, dloss, dw, accumulate,
                     want_dx, workspace, lib)


def distill_loss(x, w, index, logits, temperature: float = 1.0, workspace=None, lib=None):
    """(loss, lse) of every row: its divergence from a teacher whose entries
    ``index`` (int64) have ``logits`` (fp32), rows x entries, at
    ``temperature``.  Entries whose index is not a row of ``w`` or whose logit
    is -inf are absent; rows without entries have loss 0."""
    lib = lib or load_library()
    targets = _teacher(x, index, logits, temperature)
    return _forward(lib.phub_distill_loss, x, w, targets, targets[0], workspace, lib)


def distill_loss_grad(x, w, index, logits, temperature, lse, dloss=None, dw=None,
                      accumulate: bool = False, want_dx: bool = True, workspace=None, lib=None):
    """As ``vocab_loss_grad``, for ``distill_loss``."""
    lib = lib or load_library()
    targets = _teacher(x, index, logits, temperature)
    return _backward(lib.phub_distill_loss_grad, x, w, targets, targets[0], lse, dloss, dw,
                     accumulate, want_dx, workspace, lib)
