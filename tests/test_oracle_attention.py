"""The attention oracle held to hand-computed values and identities (CPU)."""
import numpy as np
import pytest

from oracle import attention_oracle as A


def test_rope_quarter_turn_and_kept_channels():
    x = np.arange(1, 9, dtype=np.float16).reshape(1, 8)                # one head of 8, four channels turn
    cos, sin = np.array([[0.0, 1.0]], np.float32), np.array([[1.0, 0.0]], np.float32)
    assert A.rope(x, cos, sin, 8, "half").tolist() == [[-3, 2, 1, 4, 5, 6, 7, 8]]
    assert A.rope(x, cos, sin, 8, "interleaved").tolist() == [[-2, 1, 3, 4, 5, 6, 7, 8]]


def test_rope_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 64)).astype(np.float16)
    ang = A.rope_angles(100, 64)
    dot = lambda m, n: float((A.rope(q, np.cos(ang[m:m + 1]).astype(np.float32), np.sin(ang[m:m + 1]).astype(np.float32), 64, "half").astype(float)
                              * A.rope(k, np.cos(ang[n:n + 1]).astype(np.float32), np.sin(ang[n:n + 1]).astype(np.float32), 64, "half")).sum())
    assert abs(dot(7, 3) - dot(97, 93)) < 64 * 3 * 2.0 ** -10


def test_angles_scaled():
    plain = A.rope_angles(9, 16)
    assert np.allclose(A.rope_angles(9, 16, scaling="linear", factor=4.0), plain / 4)
    w = A.rope_angles(9, 16, scaling="wavelength", factor=8.0, low=1.0, high=4.0, trained=64.0)
    turns = 64.0 * plain[1] / (2 * np.pi)
    assert np.array_equal(w[1][turns >= 4], plain[1][turns >= 4]) and np.allclose(w[1][turns <= 1], plain[1][turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all(w[1][mid] < plain[1][mid]) and np.all(w[1][mid] > plain[1][mid] / 8)


def test_quantiser_by_hand():
    x = np.array([[-1.0, 0.0, 2.0, 0.5]], np.float16)                 # range 3, 4 bits: s = fp16(0.2), z = 5
    code, s, z = A.quantise(x, 4)
    assert s[0, 0] == np.float16(0.2) and z[0, 0] == 5 and code.tolist() == [[0, 5, 15, 8]]   # 0.5 / 0.19995 = 2.5006 -> 3
    code, s, z = A.quantise(np.array([[5.0, 6.0]], np.float16), 4)    # one sign: zero stays in the range
    assert s[0, 0] == np.float16(0.4) and z[0, 0] == 0 and code.tolist() == [[13, 15]]
    code, s, z = A.quantise(np.zeros((1, 4), np.float16), 8)
    assert s[0, 0] == np.float16(2.0 ** -14) and not code.any() and z[0, 0] == 0


@pytest.mark.parametrize("bits", [4, 8])
def test_quantiser_error_and_range(bits):
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((50, 64)) * np.exp(rng.standard_normal((50, 1)) * 3)).astype(np.float16)
    x[0] = 65504
    x[1, ::2], x[1, 1::2] = 65504, -65504
    code, s, z = A.quantise(x, bits)
    assert code.min() >= 0 and code.max() <= 2 ** bits - 1
    val = A.values(code, s, z)
    assert np.abs(val).max() <= 65504
    # half a step, and at the ends what the scale's rounding and the zero's take off
    assert np.all(np.abs(val - x) <= s.astype(float) * (1.0 + 2.0 ** bits * 2.0 ** -11))
    bad = x.copy()
    bad[3, 5], bad[4, 6] = np.nan, np.inf
    val = A.values(*A.quantise(bad, bits))
    assert np.isnan(val[3:5]).all() and np.array_equal(val[5:], A.values(code, s, z)[5:])


def test_attention_as_nested_loops():
    rng = np.random.default_rng(2)
    q = rng.standard_normal((3, 4, 8)).astype(np.float16)
    k, v = rng.standard_normal((2, 5, 2, 8))
    y, bound = A.attention(q, k, v, [0, 2, 5], 0.3)
    assert not y[0].any()
    for i, lim in ((1, 2), (2, 5)):
        for h in range(4):
            num, den = np.zeros(8), 0.0
            for t in range(lim):
                p = np.exp(0.3 * sum(float(q[i, h, c]) * k[t, h // 2, c] for c in range(8)))
                num, den = num + p * v[t, h // 2], den + p
            assert np.allclose(y[i, h], num / den, rtol=1e-12)
    assert np.all(bound > 0) and bound.max() < 0.05
    seen = np.arange(5)[None] < np.array([0, 2, 5])[:, None]
    assert np.array_equal(A.attention(q, k, v, seen, 0.3)[0], y)
