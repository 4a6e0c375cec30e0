"""fp64 statement of the operators over whole rows, written from the formulas in the C header: the norm in front of the projections
and the log probabilities behind the last.  numpy only; test infrastructure."""
from __future__ import annotations

import numpy as np


def rmsnorm(x, weight=None, eps=1e-5, residual=None):
    """fp16 [M, D] (and a residual of fp16 or fp32) -> (h, y), fp64, unrounded."""
    h = x.astype(np.float64)
    if residual is not None:
        h = h + residual.astype(np.float64)
    with np.errstate(all="ignore"):
        y = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
        return h, y if weight is None else y * weight.astype(np.float64)


def rmsnorm_bound(y, D):
    """How far an fp16 y may be off: its own rounding, half a step (2^-11; 2^-25 among the subnormals), and that of the fp32 arithmetic
    in steps of 2^-24 of the value.  h: 1.  The squares and their sum over D channels, added 8 to 32 a thread one after the other and then in
    a tree of up to 10 levels: 1 + 32 + 10, halved by the root.  Mean, eps, root, quotient: up to 8.  Two products: 2."""
    off = (1 + 22 + 8 + 2) * 2.0 ** -24
    return np.abs(y) * (2.0 ** -11 * (1 + off) + off) + 2.0 ** -25


def codes(y):
    """fp64 y [M, D] -> (scale fp32 [M], y / scale fp64): a code is the whole number next to the latter."""
    scale = (np.abs(y).max(axis=1) / 127.0).astype(np.float32)
    with np.errstate(all="ignore"):
        return scale, np.where(scale[:, None] > 0, y / scale.astype(np.float64)[:, None], 0.0)


def logprobs(x, a=1.0, top=0):
    """Logits [M, V] (any float type; exact in fp64) -> (log p fp64 [M, V], entropy [M], top ids [M, top], bound of log p, bound of the entropy).
    Rows that hold NaN or +inf, or nothing but -inf, are NaN.  The bounds say how far an fp32 result may be off, u = 2^-24 being half a step, with
    d = a (x - m) and p the probabilities:
      d: the subtraction, two roundings of a log2 e and of its product:                      4 u |d|, which moves a weight by as much of itself
      the sums S of weights and T of weighted d: V / 256 one after the other at most, 40 in the tree of threads and waves with
      what brings them to one m, 8 for the exponential and the rest:                          u (V / 256 + 48) of the sum of the sizes
      ln S: that over S, the logarithm's own 4 steps:                                        u (V / 256 + 48 + 4 sum p |d| + 8 ln S)
      log p = d - ln S, each of these and the difference:                                    + u (4 |d| + |log p|)
      H = ln S - T / S:                          the former, u (V / 256 + 56) |T / S|, 4 u sum p d^2, and u H for the difference"""
    x = x.astype(np.float64)
    u, V = 2.0 ** -24, x.shape[1]
    with np.errstate(all="ignore"):
        m = x.max(axis=1, keepdims=True)
        d = np.float64(np.float32(a)) * (x - m)
        w = np.exp(d)
        S = w.sum(axis=1, keepdims=True)
        p = w / S
        log_p = d - np.log(S)
        sized = np.where(p > 0, p * np.abs(d), 0.0).sum(axis=1)
        squares = np.where(p > 0, p * d * d, 0.0).sum(axis=1)
        H = np.log(S[:, 0]) + sized
        of_s = u * (V / 256 + 48 + 4 * sized + 8 * np.log(S[:, 0]))
        bound = of_s[:, None] + u * (4 * np.abs(d) + np.abs(log_p)) + 2.0 ** -149
        bound_h = of_s + u * ((V / 256 + 56) * sized + 4 * squares + H)
    bad = ~np.isfinite(m[:, 0])
    log_p[bad], H[bad] = np.nan, np.nan
    order = np.where(np.isnan(x), np.inf, x)
    ids = np.empty((x.shape[0], top), np.int64)
    for i in range(x.shape[0]):
        # NaN first, then by value, of equal ones the lower index
        ids[i] = np.lexsort((np.arange(V), -order[i], ~np.isnan(x[i])))[:top]
    return log_p, H, ids, bound, bound_h
