"""What the attention oracle's bound and the tests' 2-norm let through: the kernels' arithmetic, and nothing coarser (CPU)."""
import numpy as np
import pytest

from oracle import attention_oracle as A

# Two roundings to fp16 of independent parts of an answer, of the probabilities and of the answer itself, each 2.05e-4 in the 2-norm: a step of
# 2^-10 times the power of two below a number, over sqrt(12), next to the root mean square of normal numbers.  Together 2.9e-4; a third makes 3.55e-4.
NORM = 3.3e-4


def _case(seed, rows=24, tokens=300, d=64, bits=8, size=1.0):
    rng = np.random.default_rng(seed)
    q = (size * rng.standard_normal((rows, 1, d))).astype(np.float16)
    code, s, z = A.quantise(rng.standard_normal((tokens, 1, d)).astype(np.float16), bits)
    vcode, vs, vz = A.quantise(rng.standard_normal((tokens, 1, d)).astype(np.float16), bits)
    return q, (code, s, z), (vcode, vs, vz), np.full(rows, tokens), d ** -0.5


def _answer(q, k, v, scale, k_as=np.float64, v_as=np.float64, score_as=np.float64, p_as=None, cut=False):
    """fp64 but for what is rounded to the types given; p_as: the probabilities times the values' scales, 2^10 below the largest."""
    kk = A.values(*k).astype(k_as).astype(np.float64)[:, 0]
    vv = A.values(*v).astype(v_as).astype(np.float64)[:, 0]
    score = (q[:, 0].astype(np.float64) @ kk.T * scale).astype(score_as).astype(np.float64)
    w = np.exp(score - score.max(axis=1, keepdims=True))
    total = w.sum(axis=1, keepdims=True)
    if p_as is not None:
        s = v[1].astype(np.float64)[:, 0, 0]
        p = w * s * 2.0 ** 10
        p16 = p.astype(p_as)
        if cut:
            p16 = np.where(p16.astype(np.float64) > p, np.nextafter(p16, p_as(0)), p16)
        w = p16.astype(np.float64) / (s * 2.0 ** 10)
    return (w @ vv / total).astype(np.float16).astype(np.float64)[:, None]


def _compare(got, want, bound):
    return bool(np.all(np.abs(got - want) <= bound)), np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens", [1, 17, 300, 2000])
def test_the_kernels_arithmetic_is_within(bits, tokens):
    for seed in range(3):
        q, k, v, limits, scale = _case(seed, tokens=tokens, bits=bits)
        want, bound = A.attention(q, A.values(*k), A.values(*v), limits, scale)
        ok, norm = _compare(_answer(q, k, v, scale, p_as=np.float16), want, bound)
        assert ok and norm <= NORM, norm
        ok, norm = _compare(_answer(q, k, v, scale), want, bound)          # the result's rounding alone
        assert ok and norm <= 2.4e-4, norm


def test_rounded_scores_are_not():
    """Scores of some tens in fp16 are off by a hundredth."""
    for seed in range(3):
        q, k, v, limits, scale = _case(seed, size=20.0)
        want, bound = A.attention(q, A.values(*k), A.values(*v), limits, scale)
        assert _compare(_answer(q, k, v, scale, p_as=np.float16), want, bound)[0]
        assert not _compare(_answer(q, k, v, scale, p_as=np.float16, score_as=np.float16), want, bound)[0]
        assert not _compare(_answer(q, k, v, scale, k_as=np.float16), want, bound)[0]


def test_further_roundings_are_above_the_norm():
    for seed in range(3):
        q, k, v, limits, scale = _case(seed, rows=64)
        want, bound = A.attention(q, A.values(*k), A.values(*v), limits, scale)
        for kw in (dict(v_as=np.float16), dict(k_as=np.float16, v_as=np.float16), dict(score_as=np.float16), dict(cut=True)):
            assert _compare(_answer(q, k, v, scale, p_as=np.float16, **kw), want, bound)[1] > NORM, kw


def test_the_bound_is_no_wider_than_twice_a_rounding_of_everything():
    """Of ordinary data the bound is made of the two roundings: e (sum w |v| + |y|) is most of it."""
    q, k, v, limits, scale = _case(5)
    want, bound = A.attention(q, A.values(*k), A.values(*v), limits, scale)
    score = q[:, 0].astype(np.float64) @ A.values(*k)[:, 0].T * scale
    w = np.exp(score)
    size = (w / w.sum(axis=1, keepdims=True)) @ np.abs(A.values(*v)[:, 0])
    assert np.all(bound[:, 0] <= 2 * 2.0 ** -11 * (size + np.abs(want[:, 0])) + 2.0 ** -25)
