"""Rotary positions, the quantised cache and the attention over it on the GPU, against the fp64 oracle."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from oracle import rosaq_oracle as O
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def same_bits(got, want):
    """fp16, NaN equal to NaN, the sign of zero aside."""
    got = got.cpu().numpy()
    assert got.shape == want.shape
    ok = (got == want) | (np.isnan(got) & np.isnan(want))
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])


# ---- rotary positions ---------------------------------------------------------------------------

def _trig(positions, rot, at):
    ang = A.rope_angles(positions, rot)
    table = np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)
    return table, table[at, :, 0], table[at, :, 1]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("M,heads,dim,rot,pad", [(1, 1, 64, 64, 0), (1, 32, 128, 128, 0), (5, 3, 128, 16, 8), (37, 7, 64, 48, 0),
                                                 (64, 32, 128, 128, 0), (130, 5, 128, 96, 24), (1003, 1, 64, 16, 0), (700, 40, 128, 64, 0)])
def test_rope(layout, M, heads, dim, rot, pad):
    print(f"case rope {layout} {M}x{heads}x{dim} rot {rot}", flush=True)
    rng = np.random.default_rng(M + rot)
    x = rng.standard_normal((M, heads * dim)).astype(np.float16)
    at = rng.integers(0, 5000, M).astype(np.int32)
    table, cos, sin = _trig(5000, rot, at)
    want = A.rope(x, cos, sin, dim, layout)
    r = T.Rope(dev(table), layout)
    buf = torch.full((M, heads * dim + pad), 7.0, dtype=torch.float16, device="cuda")
    buf[:, :heads * dim] = dev(x)
    xd = buf[:, :heads * dim]
    y = T.rope(r, xd, dev(at), dim)
    same_bits(y, want)
    assert T.rope(r, xd, dev(at), dim, out=xd) is xd                  # in place
    same_bits(xd, want)
    if pad:
        assert bool((buf[:, heads * dim:] == 7.0).all())


def test_rope_rows_without_a_position_stay():
    print("case rope positions outside the table", flush=True)
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 256)).astype(np.float16)
    at = rng.integers(0, 64, 40).astype(np.int32)
    table, cos, sin = _trig(64, 128, at)
    want = A.rope(x, cos, sin, 128, "half")
    at[3], at[4], at[17], at[39] = -1, 64, np.iinfo(np.int32).max, np.iinfo(np.int32).min
    y = torch.full((40, 256), 5.0, dtype=torch.float16, device="cuda")
    T.rope(T.Rope(dev(table)), dev(x), dev(at), 128, out=y)
    want[[3, 4, 17, 39]] = 5.0
    same_bits(y, want)


@pytest.mark.parametrize("kw,okw", [(dict(), dict()), (dict(base=500000.0), dict(base=500000.0)),
                                    (dict(scaling=B.ROPE_SCALE_LINEAR, factor=4.0), dict(scaling="linear", factor=4.0)),
                                    (dict(base=500000.0, scaling=B.ROPE_SCALE_WAVELENGTH, factor=8.0, low=1.0, high=4.0, trained_positions=8192.0),
                                     dict(base=500000.0, scaling="wavelength", factor=8.0, low=1.0, high=4.0, trained=8192.0))])
@pytest.mark.parametrize("positions,rot", [(1, 16), (131, 48), (40001, 128)])
def test_rope_table(kw, okw, positions, rot):
    print(f"case table {okw} {positions} x {rot}", flush=True)
    got = T.rope_table(positions, rot, **kw).cpu().numpy().astype(np.float64)
    ang = A.rope_angles(positions, rot, **okw)
    # half a step of fp32, and what a few roundings of fp64 (pow, product) make of the angle
    for part, want in ((got[..., 0], np.cos(ang)), (got[..., 1], np.sin(ang))):
        assert np.all(np.abs(part - want) <= 2.0 ** -24 * np.abs(want) + 16 * 2.0 ** -53 * (1 + ang))


# ---- the cache ----------------------------------------------------------------------------------

def _values(rng, M, width):
    return (rng.standard_normal((M, width)) * np.exp(rng.standard_normal((M, width // 64)).repeat(64, 1))).astype(np.float16)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,kv,dim,page,rot,q_heads", [(1, 1, 64, 16, 0, 0), (1, 32, 128, 64, 128, 32), (33, 3, 64, 16, 32, 9),
                                                       (64, 32, 128, 64, 128, 32), (257, 5, 128, 128, 64, 5), (500, 8, 64, 4096, 0, 0)])
def test_append_and_read(bits, M, kv, dim, page, rot, q_heads):
    print(f"case cache int{bits} {M}x{kv}x{dim} page {page} rot {rot}", flush=True)
    rng = np.random.default_rng(M * bits)
    k, v = _values(rng, M, kv * dim), _values(rng, M, kv * dim)
    pages = (M + 40) // page + 2
    slots = rng.permutation(pages * page)[:M].astype(np.int64)
    cache = T.KvCache(kv, dim, bits, page, pages)
    cache.data.fill_(0xa5)
    if rot:
        at = rng.integers(0, 3000, M).astype(np.int32)
        table, cos, sin = _trig(3000, rot, at)
        q = rng.standard_normal((M, q_heads * dim)).astype(np.float16)
        got = T.cache_append(cache, dev(slots), dev(k), dev(v), rope=T.Rope(dev(table), "interleaved"), positions=dev(at), q=dev(q))
        same_bits(got, A.rope(q, cos, sin, dim, "interleaved"))
        k = A.rope(k, cos, sin, dim, "interleaved")
    else:
        assert T.cache_append(cache, dev(slots), dev(k), dev(v)) is None
    want_k, want_v = (A.held(x, kv, bits).astype(np.float16).reshape(M, -1) for x in (k, v))
    got_k, got_v = T.cache_read(cache, dev(slots))
    same_bits(got_k, want_k)
    same_bits(got_v, want_v)
    # any order, repeated, one kind alone, none of the cache's slots
    order = rng.integers(0, M, 50)
    some = slots[order].copy()
    some[7], some[11], some[30] = -1, pages * page, np.iinfo(np.int64).min
    out = torch.full((50, kv * dim), 3.0, dtype=torch.float16, device="cuda")
    T.cache_read(cache, dev(some), v=out)
    want = want_v[order].copy()
    want[[7, 11, 30]] = 3.0
    same_bits(out, want)
    # bytes of other tokens are as they were
    other = np.setdiff1d(np.arange(pages * page), slots)
    fresh = T.KvCache(kv, dim, bits, page, pages)
    fresh.data.fill_(0xa5)
    for a, b in zip(T.cache_read(cache, dev(other)), T.cache_read(fresh, dev(other))):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
def test_append_odd_groups(bits, dim):
    """NaN, infinities, constants, one sign, the largest numbers, subnormals, half-way quotients; and a second write over the first."""
    print(f"case cache odd groups int{bits} {dim}", flush=True)
    rng = np.random.default_rng(bits + dim)
    x = rng.standard_normal((24, 2 * dim)).astype(np.float16)
    x[0] = 0
    x[1] = np.float16(-3.3)
    x[2] = 65504
    x[3, ::2], x[3, 1::2] = 65504, -65504
    x[4] = np.abs(x[4]) + 9
    x[5] = -np.abs(x[5]) - 9
    x[6] *= np.float16(2.0 ** -20)
    x[7, 3], x[8, 4], x[9, dim + 1] = np.nan, np.inf, -np.inf
    top = 2 ** bits - 1
    x[10, 0], x[10, 1], x[10, 2:] = 0, top, np.arange(2 * dim - 2) % top + 0.5      # scale 1: every quotient half-way
    x[10, dim], x[10, dim + 1] = 0, top
    x[11, 0] = -65504
    x[12] = -0.0
    cache = T.KvCache(2, dim, bits, 16, 3)
    slots = np.arange(5, 29).astype(np.int64)
    T.cache_append(cache, dev(slots), dev(x[::-1].copy()), dev(x[::-1].copy()))
    T.cache_append(cache, dev(slots), dev(x), dev(x))
    want = A.held(x, 2, bits).astype(np.float16).reshape(24, -1)
    for got in T.cache_read(cache, dev(slots)):
        same_bits(got, want)
    assert np.isfinite(want[2:4]).all()


def test_more_than_a_million_tokens():
    print("case many tokens", flush=True)
    M = (1 << 20) + 37
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((M, 64), generator=g, device="cuda").to(torch.float16) for _ in range(2))
    cache = T.KvCache(1, 64, 4, 64, M // 64 + 1)
    slots = torch.randperm(cache.num_pages * 64, generator=g, device="cuda")[:M]
    T.cache_append(cache, slots, k, v)
    some = torch.cat([torch.arange(M - 100, M, device="cuda"), torch.randint(0, M, (2000,), generator=g, device="cuda")])
    for got, x in zip(T.cache_read(cache, slots), (k, v)):
        same_bits(got[some], A.held(x[some].cpu().numpy(), 1, 4).astype(np.float16).reshape(len(some), -1))


def test_append_skips_tokens_without_slot_or_position():
    print("case cache skipped tokens", flush=True)
    rng = np.random.default_rng(3)
    k, v, q = (rng.standard_normal((20, 128)).astype(np.float16) for _ in range(3))
    at = rng.integers(0, 32, 20).astype(np.int32)
    table, cos, sin = _trig(32, 64, at)
    slots = np.arange(20).astype(np.int64)
    slots[2], slots[9] = -1, 32
    at[5], at[14] = -1, 32
    cache = T.KvCache(2, 64, 8, 16, 2)
    cache.data.zero_()
    q_out = torch.full((20, 128), 2.0, dtype=torch.float16, device="cuda")
    T.cache_append(cache, dev(slots), dev(k), dev(v), rope=T.Rope(dev(table)), positions=dev(at), q=dev(q), q_out=q_out)
    gone = [2, 5, 9, 14]
    want = A.rope(q, cos, sin, 64, "half")
    want[gone] = 2.0
    same_bits(q_out, want)
    got_k, got_v = T.cache_read(cache, dev(np.arange(32).astype(np.int64)))
    for got, x in ((got_k, A.rope(k, cos, sin, 64, "half")), (got_v, v)):
        want = A.held(x, 2, 8).astype(np.float16).reshape(20, -1)
        want[gone] = 0
        same_bits(got, np.concatenate([want, np.zeros((12, 128), np.float16)]))


# ---- attention ----------------------------------------------------------------------------------

class Batch:
    """Sequences in a shuffled cache whose unused memory is poison, and the oracle's answer."""

    def __init__(self, seed, kv_lens, rows, kv, group, dim, bits, page=64, prefix=0, causal=True, pad=0, spread=0.5, slack=0):
        """rows: rows of every sequence."""
        rng = np.random.default_rng(seed)
        self.__dict__.update(kv_lens=kv_lens, rows=rows, kv=kv, group=group, dim=dim, bits=bits, page=page, prefix=prefix, causal=causal)
        own = [-(-n // page) for n in kv_lens]
        pre = -(-prefix // page)
        total = sum(own) + pre + 3
        order = rng.permutation(total).astype(np.int32)
        self.prefix_table = order[:pre]
        self.table = rng.choice([-1, total, -7, np.iinfo(np.int32).max], size=(len(kv_lens), max(own + [1]) + slack)).astype(np.int32)
        at = pre
        for i, n in enumerate(own):
            self.table[i, :n] = order[at:at + n]
            at += n
        slots = [self._slots(self.prefix_table, prefix)] + [self._slots(self.table[i], n) for i, n in enumerate(kv_lens)]
        self.slots = np.concatenate(slots)
        tokens = len(self.slots)
        sigma = np.exp(spread * rng.standard_normal(kv * dim))
        self.k = (rng.standard_normal((tokens, kv * dim)) * sigma).astype(np.float16)
        self.v = rng.standard_normal((tokens, kv * dim)).astype(np.float16)
        self.M = sum(rows) + pad
        self.q = rng.standard_normal((self.M, kv * group * dim)).astype(np.float16)
        self.row_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.cache = T.KvCache(kv, dim, bits, page, total)
        self.cache.data.fill_(0xff)                      # scales and zeros that no one has written are NaN
        self.scale = dim ** -0.5

    def _slots(self, pages, n):
        t = np.arange(n)
        return (pages[t // self.page].astype(np.int64) * self.page + t % self.page) if n else np.zeros(0, np.int64)

    def plan(self, **kw):
        d = dict(max_kv=max(self.kv_lens), max_rows=max(max(self.rows), 1), rows=self.M, prefix_len=self.prefix, causal=self.causal)
        d.update(kw)
        return T.AttentionPlan(self.cache, self.kv * self.group, len(self.kv_lens), **d)

    def append(self):
        if len(self.slots):
            T.cache_append(self.cache, dev(self.slots), dev(self.k), dev(self.v))

    def run(self, plan=None, q=None, out=None, single=False):
        y = torch.full((self.M, self.q.shape[1]), 9.0, dtype=torch.float16, device="cuda") if out is None else out
        T.attention(plan or self.plan(), dev(self.q) if q is None else q, dev(np.array(self.kv_lens, np.int32)), dev(self.table),
                    row_start=None if single else dev(self.row_start),
                    prefix_pages=dev(self.prefix_table) if self.prefix else None, out=y)
        return y

    def oracle(self, hidden=None):
        k, v = A.held(self.k, self.kv, self.bits), A.held(self.v, self.kv, self.bits)
        y, bound = np.full((self.M, self.kv * self.group, self.dim), 9.0), np.zeros((self.M, self.kv * self.group, self.dim))
        at = self.prefix
        q = self.q.reshape(self.M, -1, self.dim)
        for i, (n, r) in enumerate(zip(self.kv_lens, self.rows)):
            kk, vv = np.concatenate([k[:self.prefix], k[at:at + n]]), np.concatenate([v[:self.prefix], v[at:at + n]])
            own = np.clip(n - r + 1 + np.arange(r), 0, n) if self.causal else np.full(r, n)
            seen = np.arange(self.prefix + n)[None] < (self.prefix + own)[:, None]
            if hidden is not None:
                seen &= ~np.concatenate([hidden[:self.prefix], hidden[at:at + n]])[None]
            s = slice(self.row_start[i], self.row_start[i + 1])
            y[s], bound[s] = A.attention(q[s], kk, vv, seen, self.scale)
            at += n
        return y, bound

    def check(self, y, hidden=None):
        want, bound = self.oracle(hidden)
        got = y.cpu().numpy().astype(np.float64).reshape(want.shape)
        assert np.isfinite(got).all()
        over = np.abs(got - want) > bound
        assert not over.any(), (np.argwhere(over)[:5], got[over][:5], want[over][:5], bound[over][:5])
        live = bound.any(axis=(1, 2))
        if live.any() and np.linalg.norm(want[live]) > 0:
            assert np.linalg.norm(got[live] - want[live]) <= 1e-3 * np.linalg.norm(want[live])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,kv,group,page", [([1], 1, 1, 16), ([0, 1, 2, 15, 16, 17], 2, 1, 16), ([31, 32, 33, 63, 64, 65, 127, 128, 129], 3, 4, 32),
                                                ([300, 5, 0, 1000], 2, 7, 64), ([257] * 8, 4, 1, 128), ([2500], 1, 16, 64), ([777, 1], 1, 17, 16),
                                                ([40, 3000], 1, 35, 4096)])
def test_decode(bits, dim, lens, kv, group, page):
    print(f"case decode int{bits} dim {dim} lens {lens} heads {kv} x {group} page {page}", flush=True)
    b = Batch(len(lens) + bits, lens, [1] * len(lens), kv, group, dim, bits, page, pad=2, slack=1)
    b.append()
    b.check(b.run(single=True))
    y, z = b.run(), b.run(single=True)
    assert torch.equal(y, z) and torch.equal(y, b.run())              # either form of the call, and the same again


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,rows,kv,group,causal", [([1], [1], 1, 1, True), ([5, 9], [5, 9], 2, 1, True), ([130], [130], 1, 1, True),
                                                       ([257, 64, 300], [129, 1, 0], 2, 3, True), ([90, 200], [33, 2], 1, 8, False),
                                                       ([10, 0, 3], [40, 2, 5], 2, 2, True), ([500], [77], 3, 5, True),
                                                       ([700], [600], 1, 2, True), ([65, 65], [64, 65], 1, 4, False)])
def test_prompts(bits, dim, lens, rows, kv, group, causal):
    print(f"case prompts int{bits} dim {dim} lens {lens} rows {rows} heads {kv} x {group} causal {causal}", flush=True)
    b = Batch(len(lens) + dim, lens, rows, kv, group, dim, bits, 32, causal=causal, pad=3)
    b.append()
    y = b.run()
    b.check(y)
    assert torch.equal(y, b.run())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("prefix,lens,rows,kv,group,dim", [(1, [1, 2], [1, 1], 1, 1, 128), (37, [5, 0, 64, 33], [1, 1, 1, 1], 2, 2, 64),
                                                           (100, [8, 100, 3], [3, 2, 3], 1, 4, 128), (513, [40] * 40, [1] * 40, 2, 1, 128),
                                                           (2100, [9, 30, 1, 0, 77, 200, 31, 32], [2] * 8, 1, 8, 128), (700, [300], [200], 1, 2, 64),
                                                           (64, [0, 0], [1, 2], 3, 1, 128), (1500, [70, 90, 20], [70, 60, 9], 1, 1, 128)])
def test_shared_prefix(bits, prefix, lens, rows, kv, group, dim):
    print(f"case prefix int{bits} {prefix} lens {lens} rows {rows} heads {kv} x {group} dim {dim}", flush=True)
    b = Batch(prefix + bits, lens, rows, kv, group, dim, bits, 32, prefix=prefix, pad=1)
    b.append()
    y = b.run()
    b.check(y)
    assert torch.equal(y, b.run())


def _spread(n, top, seed):
    return [int(x) for x in np.random.default_rng(seed).integers(0, top + 1, n)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("prefix,lens,rows,kv,group,dim", [(2100, _spread(40, 90, 1), [1] * 40, 2, 1, 128), (2075, _spread(60, 40, 2), [1] * 60, 2, 1, 64),
                                                           (3001, _spread(40, 70, 3), _spread(40, 3, 4), 1, 4, 128), (5000, _spread(24, 9, 5), [2] * 24, 1, 8, 64),
                                                           (200, _spread(64, 40, 6), [1] * 64, 32, 1, 64), (130, _spread(64, 33, 7), [1] * 64, 32, 2, 64),
                                                           (161, _spread(64, 5, 8), [1] * 64, 32, 1, 128), (150, [0] * 70, [1] * 70, 32, 2, 128)])
def test_prefix_computed_once_for_all(bits, prefix, lens, rows, kv, group, dim):
    """Batches that save enough by it: up to 64 rows of a kv head and more, few and many heads, some of the sequences without tokens or rows."""
    print(f"case apart int{bits} {prefix} {len(lens)} sequences heads {kv} x {group} dim {dim}", flush=True)
    b = Batch(prefix + bits, lens, rows, kv, group, dim, bits, 32, prefix=prefix, pad=2)
    plan = b.plan()
    assert plan.ws_bytes >= 2 * b.M * kv * group * (dim + 2) * 4       # at least two parts: the prefix, the sequences' own
    b.append()
    y = b.run(plan)
    b.check(y)
    assert torch.equal(y, b.run(plan))
    b.prefix_table[1] = -1                                              # a page of the prefix that is none
    hidden = np.zeros(len(b.slots), bool)
    hidden[32:64] = True
    b.check(b.run(plan), hidden)


@pytest.mark.parametrize("prefix,rows", [(0, 1), (0, 3), (70, 1), (70, 3), (0, 150)])
def test_bad_pages_are_seen_by_no_row(prefix, rows):
    print(f"case bad pages prefix {prefix} rows {rows}", flush=True)
    lens = [200, 330, 160]
    b = Batch(5, lens, [rows] * 3, 2, 2, 128, 4, 16, prefix=prefix)
    b.append()
    hidden = np.zeros(prefix + sum(lens), bool)
    at = prefix
    for i, n in enumerate(lens):
        for page, bad in ((0, -1), (3, b.cache.num_pages), (4, np.iinfo(np.int32).min)):
            b.table[i, page] = bad
            hidden[at + page * 16:at + min(page * 16 + 16, n)] = True
        at += n
    if prefix:
        b.prefix_table[1] = -1
        hidden[16:32] = True
    b.check(b.run(), hidden)
    b.table[:] = -1
    if prefix:
        b.prefix_table[:] = -1
    assert not b.run().any()


@pytest.mark.parametrize("rows", [1, 4, 140])
def test_nan_stays_with_the_rows_that_see_it(rows):
    """A token of NaN reaches the rows that see it, and neither earlier rows of its sequence nor other sequences or heads."""
    print(f"case NaN rows {rows}", flush=True)
    lens = [150, 260]
    b = Batch(8, lens, [rows] * 2, 2, 2, 128, 8, 32)
    clean_k, clean_v = b.k.copy(), b.v.copy()
    token = lens[0] - 1 - (rows > 1)                       # of sequence 0: the last, or the one before
    b.v[token, 5] = np.inf                                 # head 0's values
    b.k[token, 128 + 9] = np.nan                           # head 1's keys
    b.append()
    y = b.run().cpu().numpy().reshape(b.M, 4, 128)
    sees = np.arange(rows) + lens[0] - rows + 1 > token
    assert np.isnan(y[:rows][sees]).all()
    b.k, b.v = clean_k, clean_v
    want, bound = b.oracle()
    good = np.ones(b.M, bool)
    good[:rows] = ~sees
    assert np.all(np.abs(y[good].astype(np.float64) - want[good]) <= bound[good])


def test_scores_that_grow_and_fall():
    """Scores far apart, growing along the sequence, falling, and equal: the running reference moves, or does not."""
    print("case scores", flush=True)
    for order in ("up", "down", "flat"):
        for rows in (1, 130):
            b = Batch(11, [520], [rows], 1, 1, 128, 8, 64, causal=False)
            size = np.linspace(0, 1, 520) if order == "up" else (np.linspace(1, 0, 520) if order == "down" else np.zeros(520))
            b.q[:] = np.float16(1.0)
            b.k[:] = (size[:, None] * 20 - 6).astype(np.float16)     # scores of -68 to 158
            if order == "flat":
                b.v[:] = np.arange(520)[:, None] % 2
            b.append()
            b.check(b.run())


@pytest.mark.parametrize("rows", [1, 20, 140])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30, 3.0])
def test_scales(rows, scale):
    """A mean, the smallest scores first, and scores of some tens."""
    print(f"case scale {scale} rows {rows}", flush=True)
    b = Batch(19, [300], [rows], 2, 1, 64, 4, 32)
    b.scale = scale
    b.append()
    b.check(b.run(b.plan(scale=scale)))


@pytest.mark.parametrize("rows", [1, 20, 140])
def test_values_and_keys_of_very_different_size(rows):
    """Groups from subnormal to the largest numbers side by side: the scale of each acts on its own token only."""
    print(f"case sizes rows {rows}", flush=True)
    b = Batch(20, [400], [rows], 1, 2, 128, 8, 64)
    size = 2.0 ** np.linspace(-24, 15, 400)[np.random.default_rng(0).permutation(400)]
    b.v = np.clip(np.clip(b.v, -2, 2) * size[:, None], -65504, 65504).astype(np.float16)      # 2 x 2^15 is beyond fp16
    b.k = (np.clip(b.k, -2, 2) * np.minimum(size, 8.0)[::-1, None]).astype(np.float16)
    b.append()
    b.check(b.run())


def test_one_token_outweighs_a_long_tail():
    """60000 tokens of which each weighs 2^-24 of the first: together they count."""
    print("case tail", flush=True)
    n = 60000
    b = Batch(12, [n], [1], 1, 1, 128, 8, 64)
    b.q[:] = np.float16(1.0)
    b.k[:] = 0
    b.k[0] = np.float16(24 * np.log(2) / 128 ** 0.5)
    b.v[:] = np.float16(1.0)
    b.v[0] = np.float16(-1.0)
    b.append()
    b.check(b.run())


def test_bounds_cut_and_rows_behind_stay():
    print("case bounds", flush=True)
    b = Batch(13, [100, 220, 50], [4, 9, 2], 1, 2, 64, 4, 16, causal=False, pad=5)
    b.append()
    lens = list(b.kv_lens)
    y = b.run(b.plan(max_kv=128, max_rows=6))
    b.table[1, 8:] = -1                                     # 220 is cut to 128: the oracle hides the rest
    hidden = np.zeros(sum(lens), bool)
    hidden[100 + 128:100 + 220] = True
    want, bound = b.oracle(hidden)
    want[4 + 6:4 + 9], bound[4 + 6:4 + 9] = 9.0, 0.0         # rows of a sequence beyond max_rows
    got = y.cpu().numpy().astype(np.float64).reshape(want.shape)
    assert np.all(np.abs(got - want) <= bound)
    assert bool((y[15:] == 9.0).all())


def test_strides():
    print("case strides", flush=True)
    b = Batch(14, [70, 33], [1, 2], 2, 2, 128, 4, 16, prefix=20)
    rng = np.random.default_rng(0)
    wide = rng.standard_normal((len(b.slots), 3 * 256 + 16)).astype(np.float16)
    wide[:, 8:264], wide[:, 264:520] = b.k, b.v
    w = dev(wide)
    T.cache_append(b.cache, dev(b.slots), w[:, 8:264], w[:, 264:520])
    buf = torch.full((b.M, 512 * 2 + 24), 4.0, dtype=torch.float16, device="cuda")
    buf[:, 512:1024] = dev(b.q)
    b.check(b.run(q=buf[:, 512:1024], out=buf[:, :512]))              # q and y are columns of one buffer
    assert bool((buf[:, 1024:] == 4.0).all()) and torch.equal(buf[:, 512:1024], dev(b.q))


def test_offsets_beyond_32_bits():
    """Pages at the end of a cache of 5 GB, and slots to match."""
    print("case long offsets", flush=True)
    kv, dim, page = 8, 128, 64
    one = B.rosaq_cache_bytes(kv, dim, 8, page, 1)
    pages = (5 << 30) // one
    b = Batch(15, [90, 200], [1, 1], kv, 1, dim, 8, page)
    b.cache = T.KvCache(kv, dim, 8, page, pages)
    far = np.array([pages - 1, pages - 2, pages // 2 + 1, 0, pages - 3, 7], np.int32)
    b.table[0, :2], b.table[1, :4] = far[:2], far[2:6]
    b.slots = np.concatenate([b._slots(b.table[0], 90), b._slots(b.table[1], 200)])
    b.append()
    b.check(b.run(single=True))
    got, _ = T.cache_read(b.cache, dev(b.slots))
    same_bits(got, A.held(b.k, kv, 8).astype(np.float16).reshape(290, -1))


def test_another_stream_and_a_graph():
    """A decode loop captured once: replays append at new slots, attend over growing lengths, and give what eager calls give."""
    print("case graph", flush=True)
    b = Batch(16, [300, 90], [1, 1], 2, 2, 128, 4, 32, prefix=600, slack=3)
    b.table[:] = np.arange(2 * b.table.shape[1]).reshape(2, -1)
    pages = 2 * b.table.shape[1] + 19
    b.prefix_table = np.arange(pages - 19, pages).astype(np.int32)
    b.cache = T.KvCache(2, 128, 4, 32, pages)
    b.slots = np.concatenate([b._slots(b.prefix_table, 600), b._slots(b.table[0], 300), b._slots(b.table[1], 90)])
    b.append()
    plan = b.plan(max_kv=b.table.shape[1] * 32)
    steps = 4
    rng = np.random.default_rng(1)
    new = rng.standard_normal((steps, 3, 2, 512)).astype(np.float16)
    rope = T.Rope(T.rope_table(2000, 128))
    q, k, v = (torch.zeros((2, n), dtype=torch.float16, device="cuda") for n in (512, 256, 256))
    slots, at = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    lens, table, prefix = dev(np.array([300, 90], np.int32)), dev(b.table), dev(b.prefix_table)
    turned, y = torch.empty_like(q), torch.empty_like(q)

    def step():
        T.cache_append(b.cache, slots, k, v, rope=rope, positions=at, q=q, q_out=turned)
        T.attention(plan, turned, lens, table, prefix_pages=prefix, out=y)

    def feed(i):
        n = np.array([301 + i, 91 + i])
        q.copy_(dev(new[i, 0])); k.copy_(dev(new[i, 1, :, :256])); v.copy_(dev(new[i, 2, :, :256]))
        slots.copy_(dev(np.array([b.table[j, (m - 1) // 32] * 32 + (m - 1) % 32 for j, m in enumerate(n)], np.int64)))
        at.copy_(dev((600 + n - 1).astype(np.int32))); lens.copy_(dev(n.astype(np.int32)))

    eager = []
    for i in range(steps):
        feed(i)
        step()
        eager.append(y.clone())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        feed(0)
        step()
        side.synchronize()
        assert torch.equal(y, eager[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(3):
        for i in range(steps):
            feed(i)
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, eager[i]), (turn, i)
            torch.randn(1000, device="cuda").sum().item()


@pytest.mark.parametrize("lens,rows,kv,group,prefix", [(_spread(40, 90, 1), 1, 2, 1, 2100), ([5000, 3000], 1, 2, 2, 0), ([900], 300, 2, 2, 0)])
def test_two_graphs_share_a_workspace(lens, rows, kv, group, prefix):
    """Replayed in turn, with other work between: every call writes its partial results before it reads them."""
    print(f"case two graphs {len(lens)} x {rows} prefix {prefix}", flush=True)
    b = Batch(21, lens, [rows] * len(lens), kv, group, 128, 4, 64, prefix=prefix)
    b.append()
    plan, n, table, start = b.plan(), dev(np.array(lens, np.int32)), dev(b.table), dev(b.row_start)
    pre = dev(b.prefix_table) if prefix else None
    qs = [dev(b.q), dev(b.q[::-1].copy())]
    ys = [torch.empty_like(q) for q in qs]
    want = [T.attention(plan, q, n, table, row_start=start, prefix_pages=pre).clone() for q in qs]
    b.check(want[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for q, y in zip(qs, ys):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                T.attention(plan, q, n, table, row_start=start, prefix_pages=pre, out=y)
    torch.cuda.synchronize()
    for turn in range(3):
        for i in (0, 1, 1, 0):
            ys[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(ys[i], want[i]), (turn, i)
            plan.ws.fill_(0xff)                          # what a call finds there is of no account
            torch.randn(1000, device="cuda").sum().item()


def test_two_plans_on_two_streams():
    print("case two streams", flush=True)
    b = Batch(17, [4000, 5000], [1, 1], 2, 2, 128, 8, 64)
    b.append()
    want = b.run(single=True)
    torch.cuda.synchronize()
    got = []
    for s in [torch.cuda.Stream() for _ in range(2)]:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(b.run(b.plan(), single=True))
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want)


def test_refusals_of_the_torch_layer():
    print("case torch refusals", flush=True)
    b = Batch(18, [20], [1], 1, 2, 64, 4, 16, prefix=5)
    b.append()
    plan, q, lens, table = b.plan(), dev(b.q), dev(np.array([20], np.int32)), dev(b.table)
    prefix = dev(b.prefix_table)
    for bad in (dict(q=q.float()), dict(q=q[:, :64]), dict(q=q.cpu()), dict(lens=lens.long()), dict(lens=lens.cpu()), dict(table=table[0]),
                dict(table=table.long()), dict(prefix=None), dict(prefix=prefix[:0]), dict(out=torch.empty((1, 64), dtype=torch.float16, device="cuda")),
                dict(row_start=lens)):
        d = dict(dict(q=q, lens=lens, table=table, prefix=prefix, out=None, row_start=None), **bad)
        with pytest.raises(ValueError):
            T.attention(plan, d["q"], d["lens"], d["table"], row_start=d["row_start"], prefix_pages=d["prefix"], out=d["out"])
    with pytest.raises(B.RosaqError):
        T.attention(plan, q, lens, table, prefix_pages=prefix, out=q)
    k = torch.zeros((2, 64), dtype=torch.float16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        T.cache_append(b.cache, slots.int(), k, k)
    with pytest.raises(ValueError):
        T.cache_append(b.cache, slots[:1], k, k)
    with pytest.raises(ValueError):
        T.cache_append(b.cache, slots, k, k, q=k)
    with pytest.raises(ValueError):
        T.cache_read(b.cache, slots, k=k.float())
    with pytest.raises(ValueError):
        T.Rope(torch.zeros((4, 32, 2), device="cuda"), "pairs")
    with pytest.raises(ValueError):
        T.rope(T.Rope(torch.zeros((4, 32, 2), device="cuda")), k, slots, 64)


# ---- together -----------------------------------------------------------------------------------

def test_attention_block_between_the_linear_layers():
    """q/k/v projections (rosaq_linear_batch), positions and cache, attention, head-wise output projection: a prompt, then two
    decode steps, every stage against the oracle on what the stage before gave."""
    print("case block", flush=True)
    from test_gpu_parity import check_output, make_case
    D, heads, n = 512, 4, 45
    lay, Q, lam = make_case(5, 64, D, D, 300, O.MODE_HEADWISE)
    rng = np.random.default_rng(6)
    Ws = [(rng.standard_normal((D, D)) * 0.05).astype(np.float16) for _ in range(3)]
    qkv = [B.rosaq_pack_weights(W, Q, lam, 128, 4, B.Q_HEADWISE) for W in Ws]
    o = B.rosaq_pack_weights(lay["W"], Q, lam, 128, 4, B.Q_HEADWISE)
    o_ref = O.pack(lay["W"], Q, lam, 128, 4, O.MODE_HEADWISE)
    cache = T.KvCache(heads, 128, 8, 16, 6)
    rope = T.Rope(T.rope_table(128, 128))
    cos, sin = (rope.table[..., i].cpu().numpy() for i in range(2))
    pages = np.array([[4, 1, 5, 0]], np.int32)
    slot_of = lambda t: pages[0][t // 16].astype(np.int64) * 16 + t % 16
    k_seen, v_seen = np.zeros((0, D), np.float16), np.zeros((0, D), np.float16)
    done = 0
    for rows in (n, 1, 1):
        x = dev(rng.standard_normal((rows, D)).astype(np.float16))
        q, k, v = T.linear_batch(qkv, x)
        at = np.arange(done, done + rows)
        turned = T.cache_append(cache, dev(slot_of(at)), k, v, rope=rope, positions=dev(at.astype(np.int32)), q=q)
        done += rows
        plan = T.AttentionPlan(cache, heads, 1, max_kv=64, max_rows=rows)
        y = T.attention(plan, turned, dev(np.array([done], np.int32)), dev(pages),
                        row_start=dev(np.array([0, rows], np.int32)) if rows > 1 else None)
        out = T.linear(o, y)
        q, k, v, y_np = (t.cpu().numpy() for t in (q, k, v, y))
        same_bits(turned, A.rope(q, cos[at], sin[at], 128, "half"))
        k_seen = np.concatenate([k_seen, A.rope(k, cos[at], sin[at], 128, "half")])
        v_seen = np.concatenate([v_seen, v])
        want, bound = A.attention(turned.cpu().numpy().reshape(rows, heads, 128), A.held(k_seen, heads, 8), A.held(v_seen, heads, 8),
                                  at + 1, 128 ** -0.5)
        assert np.all(np.abs(y_np.reshape(want.shape).astype(np.float64) - want) <= bound)
        check_output(out.cpu().numpy(), y_np, Q, o_ref)
