"""Python binding of the draws under the deployed rule.

Argument marshalling only, as in losses.py: the computation runs in libvsd.so on
the current HIP stream of the tensors' device.
"""
import ctypes
import functools
import operator
from typing import NamedTuple

import torch

from . import _lib
from ._lib import VSD_BF16, VSD_F32
from .losses import _call_words, _check, _device, _source, _workspace
from .vsd import LmHead, _ptr, _stream

__all__ = ["RowSamples", "sample_rows", "draw_workspace_bytes"]


class RowSamples(NamedTuple):
    tok: torch.Tensor       # [R] int32: the token, -1 for a row without a logit above -inf, with a NaN or a bad setting
    log_prob: torch.Tensor  # [R] f32: its log-probability among the kept entries (0 with token -1, NaN for a NaN)
    kept: torch.Tensor      # [R] int32: the entries that the rule kept
    device_error: torch.Tensor


@functools.lru_cache(maxsize=256)
def draw_workspace_bytes(R, v, dtype=torch.bfloat16):
    """Workspace bytes of sample_rows for R rows of v logits."""
    rows = _lib.VsdRows(R, (v + 7) // 8 * 8, v, VSD_F32 if dtype == torch.float32 else VSD_BF16, 0)
    n = ctypes.c_size_t(0)
    _lib.check(_lib.load().vsd_draw_workspace_bytes(ctypes.byref(rows), ctypes.byref(n)))
    return n.value


def _setting(name, value, dtype, R, dev):
    """(the setting of all rows, the tensor of one per row)."""
    if not isinstance(value, torch.Tensor):
        return value, None
    _check(name, value, dtype, (R,), dev)
    return 0, value.data_ptr()


def sample_rows(Y, u, temp_target=1.0, top_k=0, top_p=1.0, min_p=0.0, workspace=None, device_error=None):
    """Draws one token per row of logits Y [R, v] with the given numbers u [R]
    (float32 in [0, 1)): temperature, then top-k, then top-p among what top-k keeps,
    then min-p relative to the row's largest probability; of the kept entries, in
    index order, the one in which their cumulative probability passes u.

    temp_target (0: the largest logit), top_k (0: off), top_p (1: off) and min_p
    (0: off) are a number for all rows or a [R] tensor (float32; top_k: int32).  A
    top_k of all of a row's entries or more keeps what 0 does, more slowly.
    Equal logits: the smaller index first.  Returns RowSamples."""
    lib = _lib.load()
    if isinstance(Y, LmHead):
        raise ValueError("sample_rows takes materialised logits")
    dev, rows, src = _source("Y", Y)
    R = rows.R
    if R < 1 or rows.v < 1:
        raise ValueError(f"Y must be [R >= 1, v >= 1], got [{R}, {rows.v}]")
    if u is None:
        raise ValueError("u is required")
    _check("u", u, torch.float32, (R,), dev)
    t, row_t = _setting("temp_target", temp_target, torch.float32, R, dev)
    k, row_k = _setting("top_k", top_k, torch.int32, R, dev)
    p, row_p = _setting("top_p", top_p, torch.float32, R, dev)
    m, row_m = _setting("min_p", min_p, torch.float32, R, dev)
    k = operator.index(k)
    if k < 0:
        raise ValueError(f"top_k={k} must be >= 0")
    # (more than a row has is all of them: larger numbers than 32 bits hold are too)
    draw = _lib.VsdDraw(t, min(k, 0x7FFFFFFF), p, m, row_t, row_k, row_p, row_m)
    with _device(dev):
        out = torch.empty(3 * R, dtype=torch.int32, device=dev)
        tok, lp, kept = torch.split_with_sizes(out, (R, R, R))
        stream = _stream(dev)
        err = _call_words(dev, stream) if device_error is None else device_error
        _check("device_error", err, torch.int32, (1,), dev)
        need = draw_workspace_bytes(R, rows.v, Y.dtype)
        ws = _workspace(need, workspace, dev)
        _lib.check(lib.vsd_sample_rows(ctypes.byref(rows), ctypes.byref(src), ctypes.byref(draw), u.data_ptr(),
                                       tok.data_ptr(), lp.data_ptr(), kept.data_ptr(), _ptr(ws), need,
                                       err.data_ptr(), stream))
    return RowSamples(tok, lp.view(torch.float32), kept, err)
