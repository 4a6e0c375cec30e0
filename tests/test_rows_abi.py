"""Argument checks of the norm and of the log probabilities, without a GPU."""
import pytest

from paper_2506_13472_amd import binding as B
from test_attention_abi import ALIGN, ARG, NULL, SHAPE, W, X, Y, Z, _code


def _norm(**over):
    d = B.RmsNormDesc()
    for k, v in dict(dict(M=4, D=512, residual_type=B.F16, eps=1e-5, x=X, ldx=512, residual=None, ld_residual=0, residual_out=None,
                          ld_residual_out=0, weight=W, y=Y, ldy=512, codes=None, ld_codes=0, scales=None), **over).items():
        setattr(d, k, v)
    return B.rosaq_rmsnorm(d)


def test_rmsnorm_refusals():
    assert B.lib().rosaq_rmsnorm(None, None) == NULL
    stream = dict(residual=Z, ld_residual=512)
    kept = dict(stream, residual_out=Z + 0x400000, ld_residual_out=512)
    codes = dict(codes=Z + 0x800000, ld_codes=512, scales=Z + 0xc00000)
    assert _code(lambda: _norm(x=0)) == NULL and _code(lambda: _norm(y=0)) == NULL
    assert _code(lambda: _norm(residual_out=Z, ld_residual_out=512)) == NULL               # no stream to keep
    assert _code(lambda: _norm(**dict(codes, scales=0))) == NULL and _code(lambda: _norm(**dict(codes, codes=0))) == NULL
    assert _code(lambda: _norm(M=0)) == SHAPE and _code(lambda: _norm(M=-3)) == SHAPE
    for D in (0, -8, 4, 516, 32776, 65536):
        assert _code(lambda: _norm(D=D, ldx=1 << 20, ldy=1 << 20)) == SHAPE, D
    for eps in (-1e-9, float("nan"), float("inf")):
        assert _code(lambda: _norm(eps=eps)) == ARG
    for kind in (B.BF16, 3, -1):
        assert _code(lambda: _norm(residual_type=kind)) == ARG
    for name in ("ldx", "ldy"):
        assert _code(lambda: _norm(**{name: 504})) == SHAPE and _code(lambda: _norm(**{name: 516})) == ALIGN
        assert _code(lambda: _norm(**{name: (1 << 40) + 8})) == SHAPE
    assert _code(lambda: _norm(x=X + 8)) == ALIGN and _code(lambda: _norm(y=Y + 2)) == ALIGN and _code(lambda: _norm(weight=W + 8)) == ALIGN
    assert _code(lambda: _norm(**dict(stream, ld_residual=500))) == SHAPE
    assert _code(lambda: _norm(**dict(stream, residual=Z + 4, residual_type=B.F32))) == ALIGN
    assert _code(lambda: _norm(**dict(stream, ld_residual=514, residual_type=B.F32))) == ALIGN
    assert _code(lambda: _norm(**dict(kept, ld_residual_out=0))) == SHAPE
    assert _code(lambda: _norm(**dict(codes, codes=Z + 4))) == ALIGN and _code(lambda: _norm(**dict(codes, ld_codes=516))) == ALIGN
    assert _code(lambda: _norm(**dict(codes, scales=Z + 2))) == ALIGN


def test_rmsnorm_refuses_overlap():
    stream = dict(residual=Z, ld_residual=512)
    assert _code(lambda: _norm(y=X + 16)) == ARG and _code(lambda: _norm(y=X, ldy=1024)) == ARG         # not the same matrix
    assert _code(lambda: _norm(y=X + 3 * 1024)) == ARG
    assert _code(lambda: _norm(**stream, y=Z + 1024)) == ARG
    assert _code(lambda: _norm(**stream, residual_out=Z + 16, ld_residual_out=512)) == ARG
    assert _code(lambda: _norm(**stream, residual_out=Y, ld_residual_out=512)) == ARG                  # over y
    assert _code(lambda: _norm(**stream, residual_out=Z, ld_residual_out=512, y=Z)) == ARG             # both in place
    assert _code(lambda: _norm(**stream, residual_type=B.F32, y=Z)) == ARG                             # another type in its place
    assert _code(lambda: _norm(**stream, residual_type=B.F32, residual_out=X, ld_residual_out=512)) == ARG
    assert _code(lambda: _norm(weight=Y + 3 * 1024 + 512)) == ARG and _code(lambda: _norm(weight=Y)) == ARG
    assert _code(lambda: _norm(codes=X, ld_codes=1024, scales=Z)) == ARG                               # codes lie nowhere in place
    assert _code(lambda: _norm(codes=Z, ld_codes=512, scales=Z + 2044)) == ARG
    assert _code(lambda: _norm(codes=Z, ld_codes=512, scales=Y + 4)) == ARG
    # columns of one buffer are apart: the call gets to its next complaint
    assert _code(lambda: _norm(ldx=2048, y=X + 1024, ldy=2048, weight=X + 2 * 512)) == ARG
    assert _code(lambda: _norm(ldx=2048, y=X + 1008, ldy=2048)) == ARG and _code(lambda: _norm(ldx=2048, y=X + 2 * 1544, ldy=2048)) == ARG


def _logprobs(ws=W, **over):
    d = B.LogprobsDesc()
    for k, v in dict(dict(M=4, V=1000, type=B.F16, scale=1.0, logits=X, ld=1000, given=2, top=5, tokens=Y, given_out=Z, entropy=Z + 0x1000,
                          top_ids=Z + 0x2000, top_out=Z + 0x3000), **over).items():
        setattr(d, k, v)
    return B.rosaq_logprobs(d, ws)


def test_logprobs_refusals():
    assert B.lib().rosaq_logprobs(None, W, 0, None) == NULL
    assert _code(lambda: _logprobs(ws=W + 128)) == ALIGN
    for name in ("logits", "tokens", "given_out", "top_ids", "top_out"):
        assert _code(lambda: _logprobs(**{name: 0})) == NULL, name
    assert _code(lambda: _logprobs(given=0, top=0, entropy=0)) == NULL
    assert _code(lambda: _logprobs(M=0)) == SHAPE and _code(lambda: _logprobs(V=0)) == SHAPE and _code(lambda: _logprobs(V=(1 << 30) + 1, ld=1 << 31)) == SHAPE
    for given in (-1, 4097):
        assert _code(lambda: _logprobs(given=given)) == SHAPE
    for top in (-1, 65):
        assert _code(lambda: _logprobs(top=top)) == SHAPE
    assert _code(lambda: _logprobs(V=4, top=5)) == SHAPE
    assert _code(lambda: _logprobs(ld=999)) == SHAPE and _code(lambda: _logprobs(ld=(1 << 40) + 1)) == SHAPE
    for scale in (0.0, -1.0, float("nan"), float("inf"), 2e18, 1e-19):
        assert _code(lambda: _logprobs(scale=scale)) == ARG
    for kind in (-1, 3):
        assert _code(lambda: _logprobs(type=kind)) == ARG
    assert _code(lambda: _logprobs(logits=X + 1)) == ALIGN and _code(lambda: _logprobs(logits=X + 2, type=B.F32)) == ALIGN
    for name, at in (("tokens", Y + 4), ("given_out", Z + 2), ("entropy", Z + 0x1001), ("top_ids", Z + 0x2004), ("top_out", Z + 0x3002)):
        assert _code(lambda: _logprobs(**{name: at})) == ALIGN, name
    for over in (dict(entropy=X + 7996), dict(given_out=Y + 60), dict(top_ids=X - 8), dict(top_ids=Z + 24), dict(top_out=Z + 0x1008),
                 dict(top_out=Z + 0x2000 + 156)):
        assert _code(lambda: _logprobs(**over)) == ARG, over


def _logprobs_workspace(M, V, top=5, **over):
    d = B.LogprobsDesc()
    for k, v in dict(dict(M=M, V=V, top=top, scale=1.0), **over).items():
        setattr(d, k, v)
    return B.rosaq_workspace_bytes_logprobs(d)


def test_logprobs_workspace():
    assert _logprobs_workspace(4096, 32000) == 256 and _logprobs_workspace(1, 1000) == 256
    for over in (dict(M=0), dict(V=0), dict(type=5), dict(top=65), dict(scale=0.0)):
        with pytest.raises(B.RosaqError):
            _logprobs_workspace(**dict(dict(M=1, V=1000), **over))
    # 16 bytes of sums and 8 an alternative for every part, of which there are at most 8
    for M, V, top in ((1, 262144, 64), (3, 131071, 5), (8, 100000, 0), (1, 1 << 30, 20)):
        n = _logprobs_workspace(M, V, top)
        part = M * (16 + 8 * top)
        assert n == 256 or (n % part == 0 and 2 <= n // part <= 8)
    assert _logprobs_workspace(1, 262144, 64) > 256
