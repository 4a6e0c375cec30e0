"""Launches that only large batches take: eight heads a task of rotary positions and cache, a wave for each tile of attention, and
workgroups that eight XCDs do not share evenly.  Sizes follow the rules at many(), shape_launch() and prefix_apart()."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from paper_2506_13472_amd import torch_glue as T
from test_gpu_attention import Batch, _spread, _trig, _values, dev, same_bits
from test_oracle_attention_bound import NORM

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("M,heads,dim,rot", [(2049, 37, 128, 128), (1725, 39, 128, 96), (65536, 1, 128, 16), (2049, 37, 64, 64), (9364, 7, 64, 16),
                                             (2049, 33, 64, 48)])
def test_rope_of_many_heads(layout, M, heads, dim, rot):
    """rows x heads from 2^16 on, a number of heads that eight does not divide, rows without a position."""
    print(f"case rope {layout} {M}x{heads}x{dim} rot {rot}", flush=True)
    assert M * heads >= 1 << 16 and heads % 8
    rng = np.random.default_rng(M + rot)
    x = rng.standard_normal((M, heads * dim)).astype(np.float16)
    at = rng.integers(0, 5000, M).astype(np.int32)
    table, cos, sin = _trig(5000, rot, at)
    want = A.rope(x, cos, sin, dim, layout)
    gone = rng.choice(M, 9, replace=False)
    at[gone] = rng.choice([-1, 5000, np.iinfo(np.int32).max], 9)
    buf = torch.full((M, heads * dim + 16), 7.0, dtype=torch.float16, device="cuda")
    buf[:, :heads * dim] = dev(x)
    xd = buf[:, :heads * dim]
    r = T.Rope(dev(table), layout)
    want[gone] = 5.0
    same_bits(T.rope(r, xd, dev(at), dim, out=torch.full((M, heads * dim), 5.0, dtype=torch.float16, device="cuda")), want)
    T.rope(r, xd, dev(at), dim, out=xd)
    want[gone] = x[gone]
    same_bits(xd, want)
    assert bool((buf[:, heads * dim:] == 7.0).all())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,kv,dim,page,rot,group,layout", [(2531, 13, 128, 16, 128, 3, "half"), (2531, 13, 64, 64, 32, 1, "interleaved"),
                                                            (3641, 9, 128, 4096, 0, 0, "half"), (1201, 29, 64, 128, 64, 2, "half"),
                                                            (2049, 17, 128, 32, 48, 5, "interleaved")])
def test_cache_of_many_heads(bits, M, kv, dim, page, rot, group, layout):
    print(f"case cache int{bits} {M}x{kv}x{dim} page {page} rot {rot} queries {group}", flush=True)
    assert M * 2 * kv >= 1 << 16 and kv % 8
    rng = np.random.default_rng(M * bits)
    k, v = _values(rng, M, kv * dim), _values(rng, M, kv * dim)
    k[5, 3], v[M - 2, -1] = np.nan, np.inf
    pages = (M + 40) // page + 2
    slots = rng.permutation(pages * page)[:M].astype(np.int64)
    told = slots.copy()
    told[[0, 3, M - 1]] = -1, pages * page, -(1 << 40)
    gone = np.zeros(M, bool)
    gone[[0, 3, M - 1]] = True
    cache = T.KvCache(kv, dim, bits, page, pages)
    cache.data.zero_()
    if rot:
        at = rng.integers(0, 3000, M).astype(np.int32)
        table, cos, sin = _trig(3000, rot, at)
        at[7], gone[7] = 3000, True
        q = rng.standard_normal((M, group * kv * dim)).astype(np.float16)
        qd = dev(q)
        got = T.cache_append(cache, dev(told), dev(k), dev(v), rope=T.Rope(dev(table), layout), positions=dev(at), q=qd, q_out=qd)
        want = A.rope(q, cos, sin, dim, layout)
        want[gone] = q[gone]
        same_bits(got, want)
        k = A.rope(k, cos, sin, dim, layout)
    else:
        T.cache_append(cache, dev(told), dev(k), dev(v))
    want = [A.held(x, kv, bits).astype(np.float16).reshape(M, -1) for x in (k, v)]
    for w in want:
        w[gone] = 0                                     # the cache was cleared
    for got, w in zip(T.cache_read(cache, dev(slots)), want):
        same_bits(got, w)
    out = torch.full((M, kv * dim), 3.0, dtype=torch.float16, device="cuda")
    T.cache_read(cache, dev(told), v=out)
    want[1][told != slots] = 3.0
    same_bits(out, want[1])
    other = np.setdiff1d(np.arange(pages * page), slots[~gone])
    for x in T.cache_read(cache, dev(other)):
        assert not x.any()


def _check(b, plan=None, **kw):
    y = b.run(plan, **kw)
    want, bound = b.oracle()
    off = y.cpu().numpy().astype(np.float64).reshape(want.shape) - want
    assert np.isfinite(off).all() and np.all(np.abs(off) <= bound)
    live = bound.any(axis=(1, 2))
    assert np.linalg.norm(off[live]) <= NORM * np.linalg.norm(want[live])
    assert torch.equal(y, b.run(plan, **kw))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("seqs,kv,group,prefix,page", [(64, 32, 1, 0, 64), (70, 32, 2, 0, 16), (131, 17, 3, 0, 4096), (64, 32, 1, 17, 32), (66, 33, 2, 48, 16)])
def test_decode_of_a_wave_for_each_tile(bits, dim, seqs, kv, group, prefix, page):
    """2048 tiles and more of up to 16 steps, no prefix apart: the results are stored as they are."""
    print(f"case alone int{bits} dim {dim} {seqs} sequences heads {kv} x {group} prefix {prefix} page {page}", flush=True)
    lens = _spread(seqs, 300, seqs + bits)
    lens[3], lens[-1] = 0, 300
    b = Batch(seqs, lens, [1] * seqs, kv, group, dim, bits, page, prefix=prefix, pad=3, slack=1)
    assert seqs * kv >= 2048 and b.plan().ws_bytes == 256
    b.append()
    _check(b, single=True)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim,prefix,page", [(64, 131, 32), (128, 131, 16), (128, 600, 64)])
def test_decode_behind_a_prefix_under_64_rows(bits, dim, prefix, page):
    """The prefix is computed for all 64 rows at once, in one row tile a wave, beside a wave for each sequence and head."""
    print(f"case prefix of 64 rows int{bits} dim {dim} prefix {prefix} page {page}", flush=True)
    lens = _spread(64, 200, prefix + bits)
    lens[0], lens[63] = 200, 0
    b = Batch(prefix, lens, [1] * 64, 32, 1, dim, bits, page, prefix=prefix)
    plan = b.plan()
    stages = -(-prefix // 64)                           # a workgroup takes two at least, and there are 256 workgroups for 32 heads
    most = max(1, min(256 // 32, stages // 2))
    parts = 1 + -(-stages // -(-stages // most))
    assert plan.ws_bytes == parts * 64 * 32 * (dim + 2) * 4
    b.append()
    _check(b, plan, single=True)


@pytest.mark.parametrize("bits,dim", [(4, 128), (8, 64)])
@pytest.mark.parametrize("kv", [1, 3])
@pytest.mark.parametrize("rows,group", [(1, 1), (1, 5), (20, 1), (40, 2)])
def test_sequences_that_eight_xcds_do_not_share_evenly(bits, dim, kv, rows, group):
    """67 or 201 pairs of sequence and kv head, dealt to the XCDs in rounds of which the last is short."""
    print(f"case uneven int{bits} dim {dim} heads {kv} x {group} rows {rows}", flush=True)
    lens = [rows + n for n in _spread(67, 560, rows + kv)]
    lens[5], lens[66] = rows, rows + 560
    b = Batch(kv, lens, [rows] * 67, kv, group, dim, bits, 32, pad=1)
    b.append()
    _check(b)
