"""Draws under the deployed rule in float64, straight from the definition (include/vsd.h,
"Draws under the deployed rule"): one row at a time, in the order of the logits."""
import math

import numpy as np


def draw_row(x, u, temp=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log_prob, kept) of one row of float64 logits; settings as float32 holds them."""
    x = np.asarray(x, dtype=np.float64)
    temp, top_p, min_p, u = (float(np.float32(v)) for v in (temp, top_p, min_p, u))
    if not ((temp == 0 or 1e-30 <= temp * (1 + 1e-6) and temp <= 1e30 * (1 + 1e-6)) and top_k >= 0 and 0 < top_p <= 1
            and 0 <= min_p <= 1 and 0 <= u < 1):
        return -1, 0.0, 0
    if np.isnan(x).any():
        return -1, math.nan, 0
    entries = [i for i in range(len(x)) if x[i] > -np.inf]
    if not entries:
        return -1, 0.0, 0
    entries.sort(key=lambda i: (-x[i], i))
    best = x[entries[0]]
    if temp == 0:
        return entries[0], 0.0, 1
    w = {i: 1.0 if x[i] == best else math.exp((x[i] - best) / temp) for i in entries}
    if top_k > 0:
        entries = entries[:top_k]
    if top_p < 1:
        target = top_p * math.fsum(w[i] for i in entries)
        part, n = [], 0
        while n < len(entries):
            part.append(w[entries[n]])
            n += 1
            if math.fsum(part) >= target if n < 64 or n % 64 == 0 else False:
                break
        # back to the shortest prefix
        while n > 1 and math.fsum(part[:n - 1]) >= target:
            n -= 1
        entries = entries[:n]
    entries = [i for i in entries if w[i] >= min_p]
    z = math.fsum(w[i] for i in entries)
    kept = sorted(entries)
    c = np.cumsum(np.array([w[i] for i in kept], dtype=np.longdouble))
    tok = kept[min(int(np.searchsorted(c, np.longdouble(u) * c[-1], side="right")), len(kept) - 1)]
    lp = (0.0 if x[tok] == best else (x[tok] - best) / temp) - math.log(z)
    return tok, lp, len(kept)


def draws(x, u, temp, top_k, top_p, min_p):
    """Arrays (token, log_prob, kept) of rows x; settings are numbers or one per row."""
    R = len(x)
    each = [np.broadcast_to(np.asarray(s), (R,)) for s in (temp, top_k, top_p, min_p)]
    out = [draw_row(x[r], u[r], *(s[r] for s in each)) for r in range(R)]
    return tuple(np.array([o[i] for o in out]) for i in range(3))
