"""fp64 statement of what lies between the q/k/v projections and the output projection, written from the formulas in the
C header: rotary positions, the quantised cache, attention over it.  numpy only; test infrastructure."""
from __future__ import annotations

import numpy as np


def rope_angles(positions: int, rot_dim: int, base=10000.0, scaling="none", factor=1.0, low=0.0, high=0.0, trained=0.0):
    """fp64 [positions, rot_dim / 2]: the angle of every position and pair."""
    f = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])
    if scaling == "linear":
        f = f / factor
    elif scaling == "wavelength":
        out = []
        for x in f:
            turns = trained * x / (2 * np.pi)
            if turns >= high:
                out.append(x)
            elif turns <= low:
                out.append(x / factor)
            else:
                keep = (turns - low) / (high - low)
                out.append((1 - keep) * x / factor + keep * x)
        f = np.array(out)
    return np.arange(positions)[:, None] * f[None, :]


def rope(x: np.ndarray, cos: np.ndarray, sin: np.ndarray, head_dim: int, layout: str) -> np.ndarray:
    """fp16 [M, heads * head_dim]; cos, sin fp32 [M, rot / 2] of the rows' positions.  Products of fp16 and fp32 are exact in
    fp64; the sum goes to fp32 and from there to fp16."""
    M, width = x.shape
    y = x.copy().reshape(M, width // head_dim, head_dim)
    half = cos.shape[1]
    c, s = cos.astype(np.float64), sin.astype(np.float64)
    for i in range(half):
        a_at, b_at = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        xs = x.reshape(y.shape)
        a, b = xs[:, :, a_at].astype(np.float64), xs[:, :, b_at].astype(np.float64)
        ci, si = c[:, i:i + 1], s[:, i:i + 1]
        y[:, :, a_at] = (a * ci - b * si).astype(np.float32).astype(np.float16)
        y[:, :, b_at] = (b * ci + a * si).astype(np.float32).astype(np.float16)
    return y.reshape(M, width)


def quantise(x: np.ndarray, bits: int):
    """fp16 [..., d] -> (codes int, scale fp16 [..., 1], zero [..., 1]); the last axis is one group."""
    top = 2 ** bits - 1
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(x).all(axis=-1, keepdims=True)
        x32 = np.where(bad, np.float32(0), x.astype(np.float32))
        lo = np.minimum(x32.min(axis=-1, keepdims=True), np.float32(0))
        hi = np.maximum(x32.max(axis=-1, keepdims=True), np.float32(0))
        s = np.maximum((hi - lo) / np.float32(top), np.float32(2.0 ** -14)).astype(np.float16)
        s64 = s.astype(np.float64)
        z = np.minimum(np.rint(-lo.astype(np.float64) / s64), top)
        t = np.floor(65504.0 / s64)
        code = np.rint(x32.astype(np.float64) / s64) + z
        code = np.clip(code, np.maximum(0, z - t), np.minimum(top, z + t))
    return code.astype(np.int64), np.where(bad, np.float16(np.nan), s), z


def values(code, s, z) -> np.ndarray:
    """fp64, unrounded."""
    return (code - z) * s.astype(np.float64)


def held(x: np.ndarray, heads: int, bits: int) -> np.ndarray:
    """fp64 [M, heads, d]: what the cache holds of fp16 x [M, heads * d]."""
    return values(*quantise(x.reshape(x.shape[0], heads, x.shape[1] // heads), bits))


def attention(q, k, v, limits, scale):
    """One sequence.  q fp16 [n, q_heads, d], k and v fp64 [tokens, kv_heads, d], limits [n]: row i sees tokens < limits[i]
    (a boolean [n, tokens] serves too).  Returns (y fp64, bound): `bound` is how far an fp16 result may be off if keys and values are
    taken as they are, scores and sums are fp32, and a probability times its value's scale is rounded to fp16 once, to nearest, for
    the product with the codes and not for the sum of the probabilities.  With
      w   the probabilities, a the score's sum of absolute products, e = 2^-11 half a step of fp16, u = 2^-23 a whole step of fp32
          (half of one if every addition rounds to nearest, which nothing says of those within a matrix instruction),
    it adds up, to first order in e and u,
      probabilities rounded for the product:            e sum w |v|
      scores off by D = u ((d / 32 + 36) (a + 10) + 4 max a + 64): sums of d / 32 instructions that add 32 products in any order and may start from
      a value's log2 s over the key's scale (|log2 s| <= 14, 10 in units of a natural logarithm); the scale's factors and the subtraction of the
      reference; logarithm, reciprocal and exponential.  In numerator and denominator alike:
                                                        sum w (exp D - 1) |v - y| / sum w exp(-D)
      the sums over n tokens: products as above, weights of a lane one after the other, and up to 16 steps each that bring
      parts and references together:                    u (n / 32 + 52) sum w |v| + u (n / 4 + 16) |y|
      probabilities among fp16's subnormals, next to a largest of 2^10 at least, whose token's largest value is half its scale
      times the codes' range at least, or whose scale is 2^-14:   n 2^-34 max(max |v|, 2^-7)
      the result's own rounding:                        e |y| + 2^-25"""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    tokens = k.shape[0]
    e, u = 2.0 ** -11, 2.0 ** -23
    y = np.zeros((n, heads, d))
    bound = np.full((n, heads, d), 2.0 ** -25)
    for i in range(n):
        seen = np.flatnonzero(limits[i]) if np.ndim(limits) == 2 else np.arange(min(max(int(limits[i]), 0), tokens))
        if len(seen) == 0:
            continue
        for h in range(heads):
            kk, vv = k[seen, h // group], v[seen, h // group]
            qq = q[i, h].astype(np.float64)
            score = kk @ qq * scale
            a = np.abs(kk) @ np.abs(qq) * abs(scale)
            w = np.exp(score - score.max())
            w /= w.sum()
            y[i, h] = w @ vv
            off, size, out = np.abs(vv - y[i, h]), w @ np.abs(vv), np.abs(y[i, h])
            delta = np.minimum(u * ((d / 32 + 36) * (a + 10) + 4 * a.max() + 64), 100.0)
            b = e * size + (w * np.expm1(delta)) @ off / (w @ np.exp(-delta))
            b += u * ((tokens / 32 + 52) * size + (tokens / 4 + 16) * out)
            b += tokens * 2.0 ** -34 * max(np.abs(vv).max(), 2.0 ** -7)
            bound[i, h] += b + e * (out + b)
    return y, bound
