"""Python binding of the 8-bit block matrices: their quantiser and their products.

Argument marshalling only, as in losses.py: the computation runs in libvsd.so on
the current HIP stream of the tensors' device.
"""
import ctypes
from typing import NamedTuple

import torch

from . import _lib
from ._lib import VSD_BF16, VSD_F32
from .losses import _device, _row_stride, _workspace
from .vsd import _dtype_code, _ptr, _stream

__all__ = ["BlockMatrix", "quantize_blocks", "block_product", "product_workspace_bytes"]

BLOCK = 128


class BlockMatrix(NamedTuple):
    """A matrix [rows, cols] of 8-bit values with a scale for every block of 1 or 128
    rows x 128 columns."""
    values: torch.Tensor  # [rows, ld] float8_e4m3fn, ld a multiple of 128 >= cols, zeros past cols in the last block
    scales: torch.Tensor  # [ceil(cols / 128), rows] f32, or [ceil(cols / 128), ceil(rows / 128)]
    cols: int

    @property
    def group(self):
        """Rows of a block (a matrix of one row: 1)."""
        return 1 if self.scales.shape[1] == self.values.shape[0] else BLOCK


def _blocks(name, m):
    """(device, VsdBlocks) of a BlockMatrix."""
    val, sc = m.values, m.scales
    if not val.is_cuda or val.dtype != torch.float8_e4m3fn or val.dim() != 2 or val.stride(1) != 1:
        raise ValueError(f"{name}.values must be a [rows, ld] float8_e4m3fn device tensor with unit column stride")
    rows, width = val.shape
    if not 1 <= m.cols <= width or rows < 1:
        raise ValueError(f"{name}: cols={m.cols} outside [1, {width}], or no rows")
    nb, groups = (m.cols + BLOCK - 1) // BLOCK, (rows + BLOCK - 1) // BLOCK
    if width < nb * BLOCK:
        raise ValueError(f"{name}.values must hold whole blocks: {nb * BLOCK} columns for cols={m.cols}, got {width}")
    if (sc.dtype != torch.float32 or sc.device != val.device or sc.dim() != 2 or sc.shape[0] != nb
            or sc.shape[1] not in (rows, groups) or (sc.shape[1] > 1 and sc.stride(1) != 1)):
        raise ValueError(f"{name}.scales must be float32 [{nb}, {rows}] or [{nb}, {groups}] with unit column stride on "
                         f"{val.device}, got {sc.dtype} {tuple(sc.shape)} on {sc.device}")
    ld = val.stride(0) if rows > 1 else (width + BLOCK - 1) // BLOCK * BLOCK
    return val.device, _lib.VsdBlocks(val.data_ptr(), sc.data_ptr(), rows, m.cols, ld,
                                      sc.stride(0) if nb > 1 else sc.shape[1], m.group)


def quantize_blocks(x, group=1, transpose=False, out=None):
    """x [R, C] (bfloat16 or float32, unit column stride), or x^T with transpose, as a
    BlockMatrix: a scale for every block of `group` (1 or 128) rows x 128 columns.

    out: a BlockMatrix of that shape to fill (a group-128 matrix of one row is the
    same as one of group 1)."""
    lib = _lib.load()
    if not x.is_cuda:
        raise ValueError("x must be a device tensor")
    if x.dim() != 2 or x.shape[0] < 1 or x.shape[1] < 1 or (x.stride(1) != 1 and x.shape[1] != 1):
        raise ValueError(f"x must be [R >= 1, C >= 1] with unit column stride, got {tuple(x.shape)} with strides {x.stride()}")
    if group not in (1, BLOCK):
        raise ValueError(f"group={group} is neither 1 nor {BLOCK}")
    kind = _dtype_code(x)
    dev = x.device
    rows, cols = x.shape[::-1] if transpose else x.shape
    nb, groups = (cols + BLOCK - 1) // BLOCK, (rows + group - 1) // group
    with _device(dev):
        if out is None:
            out = BlockMatrix(torch.empty(rows, nb * BLOCK, dtype=torch.float8_e4m3fn, device=dev),
                              torch.empty(nb, groups, dtype=torch.float32, device=dev), cols)
        on, blocks = _blocks("out", out)
        if on != dev or (blocks.rows, blocks.cols) != (rows, cols) or out.scales.shape[1] != groups:
            raise ValueError(f"out must be a BlockMatrix [{rows}, {cols}] of group {group} on {dev}")
        blocks.group = group
        ld = x.stride(0) if x.shape[0] > 1 else x.shape[1]
        _lib.check(lib.vsd_quantize_blocks(x.data_ptr(), x.shape[0], x.shape[1], ld, kind, int(transpose),
                                           ctypes.byref(blocks), _stream(dev)))
    return out


def product_workspace_bytes(a, b, dtype=torch.bfloat16):
    """Workspace bytes of block_product(a, b, dtype)."""
    return _product_bytes(_blocks("a", a)[1], _blocks("b", b)[1], VSD_BF16 if dtype == torch.bfloat16 else VSD_F32)


def _product_bytes(a, b, kind):
    n = ctypes.c_size_t(0)
    _lib.check(_lib.load().vsd_product_workspace_bytes(ctypes.byref(a), ctypes.byref(b), kind, ctypes.byref(n)))
    return n.value


def block_product(a, b, dtype=torch.bfloat16, out=None, workspace=None):
    """a [M, K] @ b [N, K]^T of block matrices (a of group 1), as [M, N] in dtype
    (bfloat16 or float32), rows padded to multiples of 16 bytes.

    The logits of a head held in 8 bits: block_product(quantize_blocks(hidden), head)
    with head = quantize_blocks(weight, group=128).  out: a [M, N] tensor to fill
    (unit column stride, 16-byte rows; it sets dtype)."""
    lib = _lib.load()
    dev, A = _blocks("a", a)
    on, Bm = _blocks("b", b)
    if on != dev:
        raise ValueError(f"a is on {dev}, b on {on}")
    M, N = A.rows, Bm.rows
    with _device(dev):
        if out is None:
            if dtype not in (torch.bfloat16, torch.float32):
                raise ValueError(f"dtype must be bfloat16 or float32, got {dtype}")
            per16 = 16 // dtype.itemsize
            ld = (N + per16 - 1) // per16 * per16
            out = torch.empty(M, ld, dtype=dtype, device=dev)
            if ld != N:
                out = out[:, :N]
        elif (not isinstance(out, torch.Tensor) or tuple(out.shape) != (M, N) or out.device != dev
                or out.dtype not in (torch.bfloat16, torch.float32) or (out.stride(1) != 1 and N != 1)):
            raise ValueError(f"out must be a bfloat16 or float32 tensor [{M}, {N}] on {dev} with unit column stride")
        kind = VSD_BF16 if out.dtype == torch.bfloat16 else VSD_F32
        need = _product_bytes(A, Bm, kind)
        ws = _workspace(need, workspace, dev)
        _lib.check(lib.vsd_block_product(ctypes.byref(A), ctypes.byref(Bm), out.data_ptr(), _row_stride(out),
                                         kind, _ptr(ws), need, _stream(dev)))
    return out
