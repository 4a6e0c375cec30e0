"""Argument checks of the rotary positions, the quantised cache and the attention over it, without a GPU."""
import ctypes as C

import pytest

from paper_2506_13472_amd import binding as B

X, Y, Z, W = 0x100000, 0x900000, 0x1100000, 0x2000000      # never dereferenced: every call fails validation first
NULL, SHAPE, ARG, ALIGN, WORKSPACE = -1, -2, -3, -5, -6


def _code(fn):
    with pytest.raises(B.RosaqError) as e:
        fn()
    assert B.rosaq_last_error() != ""
    return e.value.code


def _cache(**over):
    d = dict(kv_heads=4, head_dim=128, bits=4, page_tokens=64, num_pages=10, data=W)
    d.update(over)
    return B.Cache(**d)


def _angles(**over):
    d = dict(table=X, positions=100, rot_dim=128, layout=0)
    d.update(over)
    return B.RopeAngles(**d)


def test_cache_bytes():
    # 16 tokens of a head: two halves of codes, two times sixteen scales and zeros
    assert B.rosaq_cache_bytes(1, 128, 4, 16, 1) == 2 * 16 * 64 + 128
    assert B.rosaq_cache_bytes(4, 64, 8, 64, 10) == 10 * 4 * 4 * (2 * 16 * 64 + 128)
    assert B.rosaq_cache_bytes(40, 128, 8, 128, 100000) == 100000 * 40 * 8 * (2 * 16 * 128 + 128)      # past 32 bits
    for bad in ((0, 128, 4, 64, 1), (1, 96, 4, 64, 1), (1, 128, 3, 64, 1), (1, 128, 4, 48, 1), (1, 128, 4, 8, 1), (1, 128, 4, 8192, 1),
                (1, 128, 4, 64, 0), (4096, 128, 8, 4096, 1 << 30), (1, 128, 4, -64, 1), (5000, 128, 4, 64, 1)):
        with pytest.raises(B.RosaqError):
            B.rosaq_cache_bytes(*bad)


def test_rope_table_refusals():
    f = B.rosaq_rope_table
    assert _code(lambda: f(0, 10, 128)) == NULL
    assert B.lib().rosaq_rope_table(None, X, 10, None) == NULL
    for rot in (0, 8, 24, 144):
        assert _code(lambda: f(X, 10, rot)) == SHAPE
    for n in (0, -1, (1 << 24) + 1):
        assert _code(lambda: f(X, n, 128)) == SHAPE
    for base in (1.0, 0.0, -5.0, float("nan"), float("inf")):
        assert _code(lambda: f(X, 10, 128, base)) == ARG
    assert _code(lambda: f(X, 10, 128, scaling=3)) == ARG
    assert _code(lambda: f(X, 10, 128, scaling=1, factor=0.0)) == ARG
    assert _code(lambda: f(X, 10, 128, scaling=2, factor=2.0, low=4.0, high=4.0, trained_positions=8.0)) == ARG
    assert _code(lambda: f(X, 10, 128, scaling=2, factor=2.0, low=1.0, high=4.0)) == ARG
    assert _code(lambda: f(X, 10, 128, scaling=2, factor=float("nan"), low=1.0, high=4.0, trained_positions=8.0)) == ARG
    assert _code(lambda: f(X + 4, 10, 128)) == ALIGN


def test_rope_refusals():
    def f(a=None, at=Z, x=X, M=4, ldx=256, heads=2, dim=128, y=Y, ldy=256):
        return B.rosaq_rope(a if a is not None else _angles(), at, x, M, ldx, heads, dim, y, ldy)
    assert B.lib().rosaq_rope(None, Z, X, 4, 256, 2, 128, Y, 256, None) == NULL
    assert _code(lambda: f(at=0)) == NULL and _code(lambda: f(x=0)) == NULL and _code(lambda: f(y=0)) == NULL
    assert _code(lambda: f(_angles(table=0))) == NULL
    assert _code(lambda: f(M=0)) == SHAPE and _code(lambda: f(M=(1 << 26) + 1)) == SHAPE       # M x heads
    assert _code(lambda: f(heads=0)) == SHAPE and _code(lambda: f(heads=4097, ldx=1 << 20, ldy=1 << 20)) == SHAPE
    assert _code(lambda: f(M=1 << 20, heads=256, ldx=1 << 20, ldy=1 << 20)) == SHAPE
    assert _code(lambda: f(dim=96)) == ARG
    assert _code(lambda: f(ldx=248)) == SHAPE and _code(lambda: f(ldy=128)) == SHAPE
    assert _code(lambda: f(ldx=260)) == ALIGN and _code(lambda: f(x=X + 2)) == ALIGN and _code(lambda: f(y=Y + 8)) == ALIGN
    assert _code(lambda: f(at=Z + 2)) == ALIGN
    assert _code(lambda: f(_angles(rot_dim=24))) == SHAPE and _code(lambda: f(_angles(rot_dim=0))) == SHAPE
    assert _code(lambda: f(_angles(rot_dim=128), dim=64, heads=4)) == SHAPE
    assert _code(lambda: f(_angles(positions=0))) == SHAPE and _code(lambda: f(_angles(layout=2))) == ARG
    assert _code(lambda: f(y=X + 16)) == ARG and _code(lambda: f(y=X, ldy=512)) == ARG       # overlapping, not in place


def test_append_refusals():
    def f(c=None, slots=Z, M=4, k=X, ldk=512, v=Y, ldv=512, **kw):
        return B.rosaq_cache_append(c if c is not None else _cache(), slots, M, k, ldk, v, ldv, **kw)
    assert B.lib().rosaq_cache_append(None, Z, 4, X, 512, Y, 512, None, 0, 0, 0, 0, 0, 0, None) == NULL
    assert _code(lambda: f(slots=0)) == NULL and _code(lambda: f(k=0)) == NULL and _code(lambda: f(v=0)) == NULL
    assert _code(lambda: f(_cache(data=0))) == NULL
    assert _code(lambda: f(_cache(data=W + 16))) == ALIGN and _code(lambda: f(slots=Z + 4)) == ALIGN and _code(lambda: f(k=X + 8)) == ALIGN
    assert _code(lambda: f(_cache(bits=3))) == ARG and _code(lambda: f(_cache(head_dim=256))) == ARG
    assert _code(lambda: f(_cache(page_tokens=20))) == SHAPE and _code(lambda: f(_cache(num_pages=0))) == SHAPE
    assert _code(lambda: f(M=0)) == SHAPE and _code(lambda: f(ldk=504)) == SHAPE and _code(lambda: f(ldv=100)) == SHAPE
    assert _code(lambda: f(ldv=516)) == ALIGN
    assert _code(lambda: f(rope=_angles())) == NULL                                           # no positions
    assert _code(lambda: f(rope=_angles(rot_dim=20), positions_ptr=Z)) == SHAPE
    q = dict(q_ptr=X, ldq=1024, q_heads=8, q_out_ptr=Y, ldq_out=1024)
    assert _code(lambda: f(**q)) == NULL                                                      # q without a rotation
    r = dict(rope=_angles(), positions_ptr=Z)
    assert _code(lambda: f(**r, **dict(q, q_out_ptr=0))) == NULL
    assert _code(lambda: f(**r, **dict(q, q_heads=0))) == SHAPE and _code(lambda: f(**r, **dict(q, ldq=512))) == SHAPE
    assert _code(lambda: f(**r, **dict(q, q_out_ptr=X + 16))) == ARG
    assert _code(lambda: f(**r, **dict(q, q_ptr=Z, q_out_ptr=X + 512))) == ARG                # over k, over v
    assert _code(lambda: f(**r, **dict(q, q_ptr=Z, q_out_ptr=Y - 1024))) == ARG
    # columns of one buffer, q turned in place: apart, so that the call gets to its next complaint
    one = dict(k=X + 2048, ldk=2048, v=X + 3200, ldv=2048, **r, **dict(q, q_ptr=X, q_out_ptr=X, ldq=2048, ldq_out=2048))
    assert _code(lambda: f(M=1 << 25, **one)) == SHAPE
    assert _code(lambda: f(**dict(one, q_heads=9, ldq=2048))) == ARG                          # q's last head is k's first
    assert _code(lambda: f(M=1 << 20, **r, **dict(q, q_heads=125, ldq=1 << 15, ldq_out=1 << 15))) == SHAPE


def test_read_refusals():
    def f(c=None, slots=Z, M=4, k=X, ldk=512, v=Y, ldv=512):
        return B.rosaq_cache_read(c if c is not None else _cache(), slots, M, k, ldk, v, ldv)
    assert B.lib().rosaq_cache_read(None, Z, 4, X, 512, Y, 512, None) == NULL
    assert _code(lambda: f(slots=0)) == NULL and _code(lambda: f(k=0, v=0)) == NULL
    assert _code(lambda: f(M=0)) == SHAPE and _code(lambda: f(ldk=0)) == SHAPE and _code(lambda: f(v=Y + 2)) == ALIGN
    assert _code(lambda: f(_cache(kv_heads=0))) == SHAPE
    assert _code(lambda: f(v=X)) == ARG and _code(lambda: f(v=X + 1024 * 3)) == ARG


def _desc(cache=None, **over):
    d = B.AttentionDesc()
    d.cache = C.pointer(cache if cache is not None else _cache())
    for k, v in dict(dict(q_heads=8, M=4, sequences=4, max_rows=1, max_kv=640, prefix_len=0, causal=1, scale=0.1, q=X, ldq=1024, y=Y,
                          ldy=1024, row_start=None, kv_len=Z, pages=Z, page_stride=10, prefix_pages=None), **over).items():
        setattr(d, k, v)
    return d


def test_attention_refusals():
    def f(*a, ws=W, n=1 << 40, **over):
        return B.rosaq_attention(_desc(*a, **over), ws, n)
    assert B.lib().rosaq_attention(None, W, 1, None) == NULL
    d = _desc()
    d.cache = None
    assert B.lib().rosaq_attention(d, W, 1 << 30, None) == NULL
    for name in ("q", "y", "kv_len", "pages"):
        assert _code(lambda: f(**{name: 0})) == NULL, name
    assert _code(lambda: f(prefix_len=5)) == NULL
    assert _code(lambda: f(_cache(data=0))) == NULL and _code(lambda: f(_cache(bits=5))) == ARG
    assert _code(lambda: f(q_heads=6)) == SHAPE and _code(lambda: f(q_heads=0)) == SHAPE
    assert _code(lambda: f(M=0)) == SHAPE and _code(lambda: f(sequences=0)) == SHAPE and _code(lambda: f(sequences=5)) == SHAPE
    assert _code(lambda: f(max_rows=0)) == SHAPE and _code(lambda: f(max_rows=2)) == SHAPE     # two rows need row_start
    assert _code(lambda: f(max_rows=5, row_start=Z)) == SHAPE                                   # more than M
    assert _code(lambda: f(max_kv=-1)) == SHAPE and _code(lambda: f(prefix_len=-1)) == SHAPE
    assert _code(lambda: f(max_kv=(1 << 30) + 1, page_stride=1 << 30)) == SHAPE and _code(lambda: f(page_stride=-1)) == SHAPE
    for s in (float("nan"), float("inf"), -float("inf"), 2e18):
        assert _code(lambda: f(scale=s)) == ARG
    assert _code(lambda: f(causal=2)) == ARG
    assert _code(lambda: f(ldq=1000)) == SHAPE and _code(lambda: f(ldy=1028)) == ALIGN and _code(lambda: f(q=X + 2)) == ALIGN
    assert _code(lambda: f(kv_len=Z + 1)) == ALIGN and _code(lambda: f(row_start=Z + 2)) == ALIGN
    # columns of one buffer are apart, as long as no column is shared: the call gets to its next complaint
    assert _code(lambda: f(ldq=4096, ldy=4096, y=X + 2 * 1024, n=0, max_kv=1 << 20, page_stride=1 << 14)) == WORKSPACE
    assert _code(lambda: f(ldq=4096, ldy=4096, y=X + 2 * 1016)) == ARG and _code(lambda: f(ldq=4096, ldy=4096, y=X + 2 * 3080)) == ARG
    assert _code(lambda: f(y=X)) == ARG and _code(lambda: f(y=X + 2048)) == ARG
    assert _code(lambda: f(M=1 << 20, sequences=1 << 20, max_rows=1 << 20, row_start=Z, q_heads=128, ldq=1 << 14, ldy=1 << 14,
                           y=X + (1 << 40))) == SHAPE                                           # the grid
    split = dict(max_kv=1 << 20, page_stride=1 << 14)
    need = B.rosaq_workspace_bytes_attention(_desc(**split))
    assert need > 256 and need % 4 == 0
    assert _code(lambda: f(n=need - 1, **split)) == WORKSPACE and _code(lambda: f(ws=0, **split)) == WORKSPACE
    assert _code(lambda: f(ws=W + 128, **split)) == ALIGN


def test_workspace_size_needs_no_pointers():
    c = _cache(data=0)
    a = _desc(c, q=0, y=0, kv_len=0, pages=0, page_stride=0, max_kv=1 << 20)
    b = _desc(max_kv=1 << 20, page_stride=1 << 14)
    assert B.rosaq_workspace_bytes_attention(a) == B.rosaq_workspace_bytes_attention(b)
    assert B.rosaq_workspace_bytes_attention(_desc(c, max_kv=0)) >= 256
    with pytest.raises(B.RosaqError):
        B.rosaq_workspace_bytes_attention(_desc(c, q_heads=3))
