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
    (a boolean [n, tokens] serves too).  Returns (y fp64, bound): `bound` is how far an fp16 result may be off, from
      w   the probabilities, a the score's sum of absolute products, e = 2^-11 half a step of fp16
      probabilities rounded toward zero to fp16 in numerator and denominator alike:      2 e sum w |v - y|
      values rounded to fp16:                                                            e sum w |v|
      scores off by d = e a + (D + 8) 2^-24 a + 2^-20 (keys rounded to fp16; fp32 sums; scale and exponential),
      in numerator and denominator:                                                      2 sum w d |v - y|
      probabilities below fp16's normal range next to the largest, 2^5 at least:          tokens 2^-29 max |v|
      the result's own rounding:                                                          e |y| + 2^-25"""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    tokens = k.shape[0]
    e = 2.0 ** -11
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
            off = np.abs(vv - y[i, h])
            delta = (e + (d + 8) * 2.0 ** -24) * a + 2.0 ** -20
            bound[i, h] += 2 * e * (w @ off) + e * (w @ np.abs(vv)) + 2 * ((w * delta) @ off)
            bound[i, h] += tokens * 2.0 ** -29 * np.abs(vv).max() + e * np.abs(y[i, h])
    return y, bound
