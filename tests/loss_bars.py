"""Bars of the base losses' float32 results against float64, from counted roundings.

u = 2^-24, half a float32 step.  A row's sum s = sum_v exp2((x_v - m) c): a term
whose exponent is a = (x_v - m) c <= 0 has a relative error of at most
3 u |a| ln 2 from its exponent (subtraction, product, c) and 2 u from exp2.  The
weight of a term falls as 2^a, so the mean of |a| over the terms is at most
log2(V) <= 17.  A term passes through one addition per 8-column step of its
thread (eight, and a rescale of two operations) of at least 64 threads, and
through the joins (4 dpp, 4 lanes, at most 16 wavefronts, 3 operations each).
"""
import math

import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 1e-36  # exp2 flushes below 2^-126; the gradients' coefficients stay below 100 here


def sum_rel(V, runs=0):
    """Relative error of s; runs: partial sums joined on top (LM head)."""
    steps = 10 * math.ceil(V / 512) + 3 * (24 + runs)
    return U * (steps + 3 * math.log2(max(V, 2)) * math.log(2) + 2)


def lse_bar(ref, m, V, T, runs=0, dx=0.0):
    """|lse error|: the tail's error, log, m / T (1 / T is rounded too), their sum; dx: of the logits / T."""
    tail = np.abs(ref - m / T)
    return sum_rel(V, runs) + U * (3 * tail + 3 * np.abs(m / T) + np.abs(ref)) + dx


def loss_bar(o, x, idx, p, m, V, T, runs=0, dx=0.0):
    """|loss error| of o = losses(): every member's p |log p| and p |log q| to a few
    roundings (log p itself: value / T_p, maximum, log of a sum of 64 terms, exp), and
    x / T - m / T to four (difference, 1 / T, product, sum)."""
    at = np.where(p > 0, np.take_along_axis(x, np.maximum(idx, 0), 1) / T, 0.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        logp = np.where(p > 0, np.log(p), 0.0)
    mass = p.sum(1)
    logq = np.where(p > 0, np.abs(at - o["lse"][:, None]), 0.0)
    lp_err = U * (80 + 6 * np.abs(logp) + 60)  # teacher values up to 20 / T_p here
    terms = np.sum(p * (np.abs(logp) + logq + 1) * (lp_err + 8 * U), axis=1)
    with np.errstate(divide="ignore", invalid="ignore"):
        tail = np.where(o["live"], o["lse"] - m / T, 0.0)
    gap = np.where(p > 0, np.abs(at - (m / T)[:, None]), 0.0)
    return mass * (sum_rel(V, runs) + 3 * U * np.abs(tail) + 2 * dx) + terms + np.sum(p * 4 * U * gap, axis=1)


def grad_bar(o, x, idx, p, m, V, T, k, kind, runs=0, dx=0.0):
    """|gradient error| per element; k [R] = |scale w / T|."""
    a = np.minimum(np.abs((x - m[:, None]) / T) / math.log(2), 300)
    q = o["q"] * p.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lp_err = U * (150 + 6 * np.abs(np.log(np.maximum(p, 1e-30))))
    mem = np.zeros_like(x)
    for r in range(len(x)):
        on = p[r] > 0
        np.add.at(mem[r], idx[r][on], p[r][on] * (lp_err[r][on] + 64 * U))
    mass_err = np.sum(p * lp_err, axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        soft = np.where(q > 0, q * (sum_rel(V, runs) + 3 * U * a * math.log(2) + 10 * U + 2 * dx), 0.0)
    err = k[:, None] * (soft + o["q"] * mass_err + mem)
    return err * 1.01 + HALF[kind] * (np.abs(o["grad"]) + err) + TINY
