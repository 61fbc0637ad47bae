"""Block matrices in float64 (include/vsd.h, "Block matrices"): the quantiser by a
table of the type's values, products as they are defined."""
import numpy as np

BLOCK = 128


def _table():
    """The 127 magnitudes of OCP e4m3, in order: 8 subnormals of 2^-9, then 2^(e-7) (1 + m/8)."""
    vals = []
    for code in range(127):
        e, m = code >> 3, code & 7
        vals.append(m * 2.0 ** -9 if e == 0 else 2.0 ** (e - 7) * (1 + m / 8))
    return np.array(vals)


E4M3 = _table()


def to_e4m3(t):
    """The nearest value, ties to the even code; |t| <= 448.25."""
    a = np.minimum(np.abs(t), 448.0)
    hi = np.searchsorted(E4M3, a, side="left")
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    pick_lo = (down < up) | ((down == up) & (lo % 2 == 0))
    return np.copysign(np.where(pick_lo, E4M3[lo], E4M3[hi]), t)


def quantize(x, group, transpose=False):
    """(values, scales [blocks, row groups]) of float32 x; a block that is not finite has
    scale NaN and values of no meaning."""
    x = np.asarray(x, dtype=np.float32)
    x = x.T if transpose else x
    rows, cols = x.shape
    nb, ng = -(-cols // BLOCK), -(-rows // group)
    values = np.zeros((rows, cols))
    scales = np.zeros((nb, ng), dtype=np.float32)
    for g in range(ng):
        for b in range(nb):
            at = np.s_[g * group:(g + 1) * group, b * BLOCK:(b + 1) * BLOCK]
            part = x[at]
            with np.errstate(all="ignore"):
                s = np.float32(np.abs(part).max()) / np.float32(448.0)
                s = np.float32(2.0 ** -126) if s < 2.0 ** -126 else s
                fine = np.isfinite(part).all()
                scales[b, g] = s if fine else np.nan
                if fine:
                    values[at] = to_e4m3((part / s).astype(np.float64))
    return values, scales


def dense(values, scales, cols):
    """The float64 matrix that values [rows, >= cols] and scales stand for."""
    rows = values.shape[0]
    group = 1 if scales.shape[1] == rows else BLOCK
    s = np.repeat(np.asarray(scales, dtype=np.float64).T, group, axis=0)[:rows]
    return np.asarray(values, dtype=np.float64)[:, :cols] * np.repeat(s, BLOCK, axis=1)[:, :cols]
