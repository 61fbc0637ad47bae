"""Python binding of the gradients' global norm and their clipping.

Argument marshalling only, as in losses.py: the computation runs in libvsd.so on
the current HIP stream of the tensors' device.
"""
import ctypes
import functools
from typing import NamedTuple

import torch

from . import _lib
from .losses import _check, _device, _workspace
from .vsd import _ptr, _stream

__all__ = ["GradClip", "grad_norm", "clip_gradients", "norm_workspace_bytes"]


class GradClip(NamedTuple):
    norm: torch.Tensor   # [1] f32: the gradients' norm before
    scale: torch.Tensor  # [1] f32: what they were multiplied by (NaN: the norm is not finite, nothing was)
    grads: list          # the clipped gradients (the given ones, or out)


@functools.lru_cache(maxsize=256)
def norm_workspace_bytes(n):
    """Workspace bytes of grad_norm and clip_gradients for n tensors."""
    b = ctypes.c_size_t(0)
    _lib.check(_lib.load().vsd_norm_workspace_bytes(n, ctypes.byref(b)))
    return b.value


_KINDS = {torch.float32: _lib.VSD_F32, torch.bfloat16: _lib.VSD_BF16}


def _fields(name, t, on):
    """VsdTensor's fields of a tensor that lies in one piece, or of [R, C] rows with a stride."""
    kind = _KINDS.get(getattr(t, "dtype", None))
    if kind is None:
        raise ValueError(f"{name} must be bfloat16 or float32 tensors, got {getattr(t, 'dtype', t)}")
    if t.get_device() != on:
        raise ValueError(f"{name} must be tensors on one device")
    if t.is_contiguous():
        n = t.numel()
        return (t.data_ptr(), 1, n, n, kind)
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.shape[1]:
        return (t.data_ptr(), t.shape[0], t.shape[1], t.stride(0), kind)
    raise ValueError(f"{name}: a tensor must be contiguous, or [R, C] with unit column stride and rows that do not "
                     f"overlap; got {tuple(t.shape)} with strides {t.stride()}")


def _table(fields):
    """Host array of VsdTensor (its five fields as 64-bit words: 1.5 us less a tensor
    than as structures)."""
    return (ctypes.c_int64 * (5 * len(fields)))(*[v for f in fields for v in f])


def _given(grads):
    grads = list(grads)
    if not grads or not isinstance(grads[0], torch.Tensor) or not grads[0].is_cuda:
        raise ValueError("grads must be one or more device tensors")
    dev = grads[0].device
    return grads, dev, [_fields("grads", t, dev.index) for t in grads]


def grad_norm(grads, workspace=None):
    """[1] float32: the square root of the sum of all elements' squares of the
    gradients (bfloat16 or float32 tensors, contiguous or [R, C] with a row stride)."""
    lib = _lib.load()
    grads, dev, fields = _given(grads)
    with _device(dev):
        norm = torch.empty(1, dtype=torch.float32, device=dev)
        need = norm_workspace_bytes(len(grads))
        ws = _workspace(need, workspace, dev)
        _lib.check(lib.vsd_grad_norm(_table(fields), len(grads), norm.data_ptr(), _ptr(ws), need, _stream(dev)))
    return norm


def clip_gradients(grads, max_norm, norm=None, out=None, workspace=None):
    """Scales the gradients by max_norm / norm where their global norm is larger than
    max_norm, in place or into `out` (as many tensors of the same shapes, bfloat16
    or float32: an optimizer's buffers).

    norm [1] float32: the norm to use in place of these tensors' own (that of more
    tensors, or of all ranks' shards).  A norm that is not finite scales nothing
    and returns the scale NaN.  Returns GradClip; nothing waits for the device."""
    lib = _lib.load()
    grads, dev, fields = _given(grads)
    res, to = grads, None
    if out is not None:
        res = list(out)
        if len(res) != len(grads) or any(o.shape != g.shape for o, g in zip(res, grads)):
            raise ValueError("out must hold a tensor of each gradient's shape")
        to = [_fields("out", t, dev.index) for t in res]
        for i, (f, o) in enumerate(zip(fields, to)):
            if f[1] != o[1] or f[2] != o[2]:  # one lies in one piece, the other does not: both by rows
                rows, cols = grads[i].shape
                fields[i] = (f[0], rows, cols, grads[i].stride(0), f[4])
                to[i] = (o[0], rows, cols, res[i].stride(0), o[4])
        to = _table(to)
    _check("norm", norm, torch.float32, (1,), dev)
    with _device(dev):
        stat = torch.empty(2, dtype=torch.float32, device=dev)
        need = norm_workspace_bytes(len(grads)) if norm is None else 0
        ws = _workspace(need, workspace, dev)
        at = stat.data_ptr()
        _lib.check(lib.vsd_clip_gradients(_table(fields), to, len(grads), max_norm, _ptr(norm), at, at + 4, _ptr(ws), need,
                                          _stream(dev)))
    return GradClip(stat[:1], stat[1:], res)
