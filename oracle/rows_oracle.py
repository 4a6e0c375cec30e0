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
