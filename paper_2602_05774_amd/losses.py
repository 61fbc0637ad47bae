"""Python binding of the base losses and of the teacher's top logits.

Argument marshalling only, as in vsd.py: tensors are checked for device, dtype,
shape and strides, outputs are allocated with torch, and the computation runs in
libvsd.so on the current HIP stream of the tensors' device.  All of a call's
tensors lie on one device.

Rows are [R, v] logits with unit column stride (a column range of a wider
buffer is fine: base address and row stride are multiples of 16 bytes), or an
LmHead(hidden [R, H], weight [v, H]), whose logits are not kept (those of
few rows or of a small vocabulary lie in the workspace, 256 MB at most).
"""
import contextlib
import ctypes
import functools
from typing import NamedTuple, Optional, Union

import torch

from . import _lib
from ._lib import VSD_BF16, VSD_F32, VSD_MAX_TOP
from .vsd import LmHead, LmHeadGrad, _dtype_code, _ptr, _stream

__all__ = ["LossResult", "TopLogits", "cross_entropy", "distill_loss", "top_logits", "loss_workspace_bytes",
           "top_workspace_bytes"]


class LossResult(NamedTuple):
    loss_row: torch.Tensor    # [R] f32: each row's loss, unweighted (0 for rows out of play)
    lse: torch.Tensor         # [R] f32: log-sum-exp of the row's logits / temp_draft
    loss_total: torch.Tensor  # [1] f32: loss_scale * sum of row_weight * loss_row
    grad: Optional[Union[torch.Tensor, LmHeadGrad]]  # of loss_total: [R, v] in the logits' dtype, or LmHeadGrad
    device_error: torch.Tensor


class TopLogits(NamedTuple):
    idx: torch.Tensor         # [R, k] int32: indices (draft indices with a map), -1 past the row's entries
    logits: torch.Tensor      # [R, k] f32: their logits, the larger first, -inf past the row's entries
    lse: torch.Tensor         # [R] f32: log-sum-exp of the whole row / temp_target
    device_error: torch.Tensor


def _source(name, src):
    """(device, VsdRows, VsdSrc) of logits or an LM head."""
    if isinstance(src, LmHead):
        h, w = src.hidden, src.weight
        for nm, t in (("hidden", h), ("weight", w)):
            if not t.is_cuda or t.dtype != torch.bfloat16 or not t.is_contiguous() or t.dim() != 2:
                raise ValueError(f"{name}.{nm} must be a contiguous 2-D bfloat16 device tensor")
        if h.shape[1] != w.shape[1] or w.device != h.device:
            raise ValueError(f"{name}: hidden [R, H] and weight [v, H] must share H and the device, got "
                             f"{tuple(h.shape)} and {tuple(w.shape)}")
        if h.shape[1] == 0:
            raise ValueError(f"{name}: the hidden size is 0")
        return (h.device, _lib.VsdRows(h.shape[0], 0, w.shape[0], VSD_BF16, h.shape[1]),
                _lib.VsdSrc(None, h.data_ptr(), w.data_ptr()))
    if not src.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if src.dim() != 2 or (src.stride(1) != 1 and src.shape[1] != 1):
        raise ValueError(f"{name} must be [R, v] with unit column stride, got {tuple(src.shape)} "
                         f"with strides {src.stride()}")
    return (src.device, _lib.VsdRows(src.shape[0], _row_stride(src), src.shape[1], _dtype_code(src), 0),
            _lib.VsdSrc(src.data_ptr(), None, None))


def _row_stride(t):
    """Row stride in elements; a single row's stride is never used and may be anything."""
    per16 = 16 // t.element_size()
    return t.stride(0) if t.shape[0] > 1 else (t.shape[1] + per16 - 1) // per16 * per16


def _check(name, t, dtype, shape, dev):
    if t is None:
        return
    if t.dtype != dtype or not t.is_contiguous() or tuple(t.shape) != shape or t.device != dev:
        raise ValueError(f"{name} must be a contiguous {str(dtype).split('.')[-1]} tensor {list(shape)} on {dev}, got "
                         f"{str(t.dtype).split('.')[-1]} {list(t.shape)} on {t.device}")


def loss_workspace_bytes(R, v, hidden_dim=0, k=0, grad=True):
    """Workspace bytes of cross_entropy (k = 0) or distill_loss (k members) for R
    rows of v logits through an LM head (materialised logits need none)."""
    return _query_loss(R, v, hidden_dim, k, bool(grad))


@functools.lru_cache(maxsize=256)
def _query_loss(R, v, hidden_dim, k, grad):
    rows, n = _lib.VsdRows(R, v, v, VSD_BF16, hidden_dim), ctypes.c_size_t(0)
    _lib.check(_lib.load().vsd_loss_workspace_bytes(ctypes.byref(rows), k, int(grad), ctypes.byref(n)))
    return n.value


@functools.lru_cache(maxsize=256)
def top_workspace_bytes(v):
    """Workspace bytes of top_logits over rows of v logits with a map (none without)."""
    rows, n = _lib.VsdRows(1, v, v, VSD_BF16, 0), ctypes.c_size_t(0)
    _lib.check(_lib.load().vsd_top_workspace_bytes(ctypes.byref(rows), 1, ctypes.byref(n)))
    return n.value


def _workspace(need, given, dev):
    """The given workspace if it is large enough, else a new one."""
    if need == 0:
        return None
    if given is not None:
        if given.dtype != torch.uint8 or not given.is_contiguous() or given.device != dev:
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
        if given.numel() >= need:
            return given
    return torch.empty(need, dtype=torch.uint8, device=dev)


# Zeroed words [error, counter] of one call each, made 256 at a time per device
# and stream (a fill a call took 4 of its 21 us on the host); a word is handed out
# once.  A captured call gets a fill of its own, which its graph repeats.
_words = {}


def _call_words(dev, stream):
    """A zeroed [1] int32 tensor with a zeroed word behind it."""
    if torch.cuda.is_current_stream_capturing():
        return torch.zeros(2, dtype=torch.int32, device=dev)[:1]
    try:
        return _words[dev.index, stream].pop()
    except (KeyError, IndexError):
        with torch.inference_mode(False):
            made = list(torch.zeros(256, 2, dtype=torch.int32, device=dev).narrow(1, 0, 1).unbind(0))
        mine = made.pop()
        _words[dev.index, stream] = made
        return mine


def _gradient(X, rows, dev, grad, weight_grad):
    """(result, VsdLossGrad) of the gradient asked for: True (allocated) or buffers to fill."""
    if isinstance(X, LmHead):
        R, H, v = rows.R, rows.hidden_dim, rows.v
        if grad is True:
            kind = torch.float32 if weight_grad is True else weight_grad or None
            grad = LmHeadGrad(torch.empty(R, H, dtype=torch.bfloat16, device=dev), None,
                              None if kind is None else torch.empty(v, H, dtype=kind, device=dev))
        if not isinstance(grad, LmHeadGrad):
            raise ValueError("the gradient of an LmHead source is an LmHeadGrad")
        if grad.grad_logits is not None:
            raise ValueError("the logits' gradient of an LmHead source is not kept: grad_logits must be None")
        _check("grad_hidden", grad.grad_hidden, torch.bfloat16, (R, H), dev)
        gw = grad.grad_weight
        if gw is not None:
            if gw.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError(f"grad_weight must be float32 or bfloat16, got {gw.dtype}")
            _check("grad_weight", gw, gw.dtype, (v, H), dev)
        if grad.grad_hidden is None:
            raise ValueError("grad_hidden is required")
        if weight_grad and gw is None:
            raise ValueError("weight_grad needs grad=True, or a grad_weight to fill")
        return grad, _lib.VsdLossGrad(None, 0, grad.grad_hidden.data_ptr(), _ptr(gw),
                                      VSD_BF16 if gw is not None and gw.dtype == torch.bfloat16 else VSD_F32)
    if weight_grad:
        raise ValueError("weight_grad needs an LmHead source")
    if grad is True:
        per16 = 16 // X.element_size()
        ld = (rows.v + per16 - 1) // per16 * per16
        grad = torch.empty(rows.R, ld, dtype=X.dtype, device=dev)
        if ld != rows.v:
            grad = grad[:, :rows.v]
        return grad, _lib.VsdLossGrad(grad.data_ptr(), ld, None, None, VSD_F32)
    if (not isinstance(grad, torch.Tensor) or grad.shape != X.shape or grad.dtype != X.dtype or grad.device != dev
            or (grad.stride(1) != 1 and grad.shape[1] != 1)):
        raise ValueError("grad must match the logits in shape, dtype and device, with unit column stride")
    return grad, _lib.VsdLossGrad(grad.data_ptr(), _row_stride(grad), None, None, VSD_F32)


_here = contextlib.nullcontext()


def _device(dev):
    """Makes the tensors' device the current one, as kernel launches need."""
    return _here if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


def _loss(X, k, dev, rows, src, call, grad, weight_grad, row_weight, workspace, device_error):
    """Checks and allocations that both losses share, with the tensors' device the
    current one; call(rows, src, weight, out, grad, workspace, bytes, stream)."""
    R = rows.R
    if R < 1 or rows.v < 1:
        raise ValueError(f"rows must be [R >= 1, v >= 1], got [{R}, {rows.v}]")
    _check("row_weight", row_weight, torch.float32, (R,), dev)
    if grad is None or grad is False:
        if weight_grad:
            raise ValueError("weight_grad needs grad")
        result, g = None, None
    else:
        result, g = _gradient(X, rows, dev, grad, weight_grad)
    out = torch.empty(2 * R + 1, dtype=torch.float32, device=dev)
    loss_row, lse, total = torch.split_with_sizes(out, (R, R, 1))
    stream = _stream(dev)
    words = _call_words(dev, stream)
    if device_error is None:
        err = words
    else:
        _check("device_error", device_error, torch.int32, (1,), dev)
        err = device_error
    need = _query_loss(R, rows.v, rows.hidden_dim, k, g is not None) if rows.hidden_dim else 0
    ws = _workspace(need, workspace, dev)
    at = out.data_ptr()
    lo = _lib.VsdLossOut(at, at + 4 * R, at + 8 * R, err.data_ptr(), words.data_ptr() + 4)
    _lib.check(call(ctypes.byref(rows), ctypes.byref(src), _ptr(row_weight), ctypes.byref(lo),
                    None if g is None else ctypes.byref(g), _ptr(ws), need, stream))
    return LossResult(loss_row, lse, total, result, err)


def cross_entropy(X, labels, row_weight=None, temp_draft=1.0, loss_scale=1.0, grad=None, weight_grad=False,
                  workspace=None, device_error=None):
    """Softmax cross entropy of rows X (logits [R, v] or an LmHead) against labels
    ([R] int32 in [0, v); -1: the row is out of play), with its gradient.

    row_weight [R] float32 weights the rows in loss_total and in the gradient (for
    a mean, 1 / count; a row of weight 0 is out of play).  grad: None (the loss
    only), True, or the buffer to fill: for logits a tensor like X (X itself
    included), for an LmHead LmHeadGrad(grad_hidden, None, grad_weight or None).
    weight_grad (with grad=True): False, True (float32) or the dtype of the
    weight's gradient.  Returns LossResult."""
    lib = _lib.load()
    dev, rows, src = _source("X", X)
    _check("labels", labels, torch.int32, (rows.R,), dev)
    if labels is None:
        raise ValueError("labels are required")

    def call(r, s, weight, out, g, ws, need, stream):
        return lib.vsd_cross_entropy(r, s, labels.data_ptr(), weight, temp_draft, loss_scale, out, g, ws, need, stream)

    with _device(dev):
        return _loss(X, 0, dev, rows, src, call, grad, weight_grad, row_weight, workspace, device_error)


def distill_loss(X, teacher_idx, teacher_logits, teacher_lse=None, row_weight=None, temp_draft=1.0, temp_target=1.0,
                 loss_scale=1.0, grad=None, weight_grad=False, workspace=None, device_error=None):
    """Distillation of rows X (logits [R, v] or an LmHead) from a teacher's k top
    logits: KL(p || q) over the row's members, q over all v columns.

    teacher_idx [R, k] int32 in [0, v), -1: none; teacher_logits [R, k] float32 or
    bfloat16; teacher_lse [R] float32: the teacher's log-sum-exp at temp_target
    (p over its whole vocabulary; None: p renormalised over the members).
    The other arguments are cross_entropy's.  Returns LossResult."""
    lib = _lib.load()
    dev, rows, src = _source("X", X)
    if teacher_idx is None or teacher_logits is None:
        raise ValueError("teacher_idx and teacher_logits are required")
    k = teacher_idx.shape[1] if teacher_idx.dim() == 2 else 0
    if not 1 <= k <= VSD_MAX_TOP:
        raise ValueError(f"teacher_idx must be [R, k] with 1 <= k <= {VSD_MAX_TOP}, got {tuple(teacher_idx.shape)}")
    _check("teacher_idx", teacher_idx, torch.int32, (rows.R, k), dev)
    if teacher_logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"teacher_logits must be float32 or bfloat16, got {teacher_logits.dtype}")
    _check("teacher_logits", teacher_logits, teacher_logits.dtype, (rows.R, k), dev)
    _check("teacher_lse", teacher_lse, torch.float32, (rows.R,), dev)

    def call(r, s, weight, out, g, ws, need, stream):
        return lib.vsd_distill_loss(r, s, k, teacher_idx.data_ptr(), teacher_logits.data_ptr(),
                                    _dtype_code(teacher_logits), _ptr(teacher_lse), weight, temp_draft, temp_target,
                                    loss_scale, out, g, ws, need, stream)

    with _device(dev):
        return _loss(X, k, dev, rows, src, call, grad, weight_grad, row_weight, workspace, device_error)


def top_logits(Y, k, d2t=None, temp_target=1.0, workspace=None, device_error=None):
    """The k largest logits of each row of Y [R, v] (the teacher's), their indices
    and the rows' log-sum-exp at temp_target: what distill_loss takes.

    d2t [v_draft] int32: only the columns d2t[u] take part, each with its draft
    index u (lse stays that of the whole row).  Equal logits: the smaller index
    first; -inf and NaN logits are no entries (NaN and +inf make lse NaN).  Returns
    TopLogits."""
    lib = _lib.load()
    if isinstance(Y, LmHead):
        raise ValueError("top_logits takes materialised logits")
    dev, rows, src = _source("Y", Y)
    R, k = rows.R, int(k)
    if R < 1 or rows.v < 1:
        raise ValueError(f"Y must be [R >= 1, v >= 1], got [{R}, {rows.v}]")
    if not 1 <= k <= VSD_MAX_TOP:
        raise ValueError(f"k={k} outside [1, {VSD_MAX_TOP}]")
    if d2t is not None:
        _check("d2t", d2t, torch.int32, (d2t.numel(),), dev)
    with _device(dev):
        idx = torch.empty(R, k, dtype=torch.int32, device=dev)
        val = torch.empty(R, k, dtype=torch.float32, device=dev)
        lse = torch.empty(R, dtype=torch.float32, device=dev)
        stream = _stream(dev)
        err = _call_words(dev, stream) if device_error is None else device_error
        _check("device_error", err, torch.int32, (1,), dev)
        need = top_workspace_bytes(rows.v) if d2t is not None else 0
        ws = _workspace(need, workspace, dev)
        _lib.check(lib.vsd_top_logits(ctypes.byref(rows), ctypes.byref(src), k, _ptr(d2t),
                                      0 if d2t is None else d2t.numel(), temp_target, idx.data_ptr(), val.data_ptr(),
                                      lse.data_ptr(), _ptr(ws), need, err.data_ptr(), stream))
    return TopLogits(idx, val, lse, err)
