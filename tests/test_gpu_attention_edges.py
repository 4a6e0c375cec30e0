"""Calls of the attention block that an ordinary batch does not make: results that the calls allocate for rows without a position
or slot, tables without a column, queries that are no numbers, very long sequences, calls of very many outputs."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T
from test_gpu_attention import Batch, dev, same_bits

pytestmark = pytest.mark.gpu


# ---- more outputs than a grid of one dimension holds ---------------------------------------------

@pytest.mark.parametrize("parts,M,kv,tokens", [(2, (1 << 20) + 5, 64, 512), (17, (1 << 19) + 3, 32, 4352)])
def test_joins_of_very_many_outputs(parts, M, kv, tokens):
    """M x heads past 2^26 (up to 16 parts) and 2^24 (more of them); one sequence has the last row, all others are no one's."""
    print(f"case join of {M} x {kv} outputs, {parts} parts", flush=True)
    need = M * kv * 64 * 4 + parts * M * kv * 66 * 4 + (4 << 30)
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip(f"needs {need >> 30} GiB of device memory")
    b = Batch(1, [tokens], [1], kv, 1, 64, 4, 64)
    b.append()
    plan = b.plan(rows=M)
    assert plan.ws_bytes == parts * M * kv * 66 * 4
    q, y = (torch.empty((M, kv * 64), dtype=torch.float16, device="cuda") for _ in range(2))
    q[-1] = dev(b.q[0])
    y[-2:] = 9.0
    T.attention(plan, q, dev(np.array([tokens], np.int32)), dev(b.table), row_start=dev(np.array([M - 1, M], np.int32)), out=y)
    b.check(y[-1:])
    assert bool((y[-2] == 9.0).all())
    del plan, q, y
    torch.cuda.empty_cache()


# ---- results that the calls allocate -------------------------------------------------------------

def _stale(rows, width):
    """Leaves NaN where the allocator will put the next matrix of this shape."""
    t = torch.full((rows, width), float("nan"), dtype=torch.float16, device="cuda")
    at = t.data_ptr()
    del t
    return at


def test_rows_without_a_position_or_slot_are_zero_where_the_call_allocates():
    print("case allocated results", flush=True)
    rng = np.random.default_rng(0)
    x = rng.standard_normal((33, 256)).astype(np.float16)
    at = np.arange(33, dtype=np.int32)
    at[[4, 32]] = -1
    ang = A.rope_angles(33, 128)
    table = np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)
    want = A.rope(x, table[at, :, 0], table[at, :, 1], 128, "half")
    want[[4, 32]] = 0
    r = T.Rope(dev(table))
    cache = T.KvCache(2, 128, 8, 16, 3)
    slots = np.arange(33, dtype=np.int64)
    slots[7] = -1
    xd, ad, sd = dev(x), dev(at), dev(slots)

    where = _stale(33, 256)
    y = T.rope(r, xd, ad, 128)
    assert y.data_ptr() == where
    same_bits(y, want)
    del y

    where = _stale(33, 256)
    y = T.cache_append(cache, sd, xd, xd, rope=r, positions=ad, q=xd)
    assert y.data_ptr() == where
    skipped = want.copy()
    skipped[7] = 0
    same_bits(y, skipped)
    del y

    T.cache_append(cache, sd, xd, xd)
    del xd
    _stale(33, 256)
    k, v = T.cache_read(cache, sd)
    held = A.held(x, 2, 8).astype(np.float16).reshape(33, 256)
    held[7] = 0
    same_bits(k, held)
    same_bits(v, held)


# ---- tables without a column ---------------------------------------------------------------------

def test_page_table_cut_to_no_column():
    """No sequence has tokens of its own yet: the table, cut to the pages in use, has no column."""
    print("case no column", flush=True)
    b = Batch(3, [0, 0, 0], [1, 1, 1], 2, 2, 64, 4, 32, prefix=70)
    b.append()
    plan = b.plan(max_kv=500)
    y = torch.full((3, 256), 9.0, dtype=torch.float16, device="cuda")
    T.attention(plan, dev(b.q), dev(np.array([0, 9, 0], np.int32)), torch.empty((3, 0), dtype=torch.int32, device="cuda"),
                prefix_pages=dev(b.prefix_table), out=y)
    b.check(y)


# ---- queries that are no numbers -----------------------------------------------------------------

@pytest.mark.parametrize("bits,dim", [(4, 64), (4, 128), (8, 64), (8, 128)])
@pytest.mark.parametrize("rows", [1, 3, 20, 140])
@pytest.mark.parametrize("odd", [-np.inf, np.inf, np.nan])
def test_queries_that_are_no_numbers(bits, dim, rows, odd):
    """A score of -inf alone leaves nothing to divide by: the row is NaN, not zero.  Its neighbours and rows that see nothing are as ever."""
    print(f"case odd queries int{bits} {dim} rows {rows} {odd}", flush=True)
    b = Batch(4, [rows, rows + 70, 0], [rows, rows, rows], 1, 2, dim, bits, 16)
    b.k[:, 5] = np.abs(b.k[:, 5]) + 1          # one sign: every score has the same
    b.append()
    hit = [(0, 1), (rows - 1, 0), (rows, 1), (3 * rows - 1, 0)]
    q = b.q.reshape(b.M, 2, dim).copy()
    for row, head in hit:
        q[row, head, 5] = odd
    y = b.run(q=dev(q.reshape(b.M, -1))).cpu().numpy().astype(np.float64).reshape(b.M, 2, dim)
    want, bound = b.oracle()
    for row, head in hit[:3]:
        assert np.isnan(y[row, head]).all(), (row, head)
        y[row, head] = want[row, head]
    assert np.all(np.abs(y - want) <= bound) and not y[2 * rows:].any()


# ---- many tokens of little weight ----------------------------------------------------------------

@pytest.mark.parametrize("rows,seqs", [(1, 1040), (20, 512), (70, 512)])
def test_many_tokens_of_little_weight(rows, seqs):
    """Two million tokens of weight 2^-31 each beside one of 1: a thousandth of the answer, which the sum of the products must not
    lose where the sum of the weights has it.  One part, so that all tokens of a row share a reference.  What a weight may lose is half a
    step of fp16's subnormals, 2^-25, next to a largest of 2^10 at least, twice that against the largest value (the scale of a token is half its
    largest value over the codes' at most)."""
    n = 1 << 21
    print(f"case {n} tokens of little weight, {rows} rows", flush=True)
    cache = T.KvCache(1, 64, 4, 4096, n // 4096)
    slots = torch.arange(n, device="cuda")
    k, v = (torch.zeros((n, 64), dtype=torch.float16, device="cuda") for _ in range(2))
    k[0, 0] = 1.0
    v[0, 1] = 1.0
    v[1:, 2] = 1.0
    T.cache_append(cache, slots, k, v)
    del k, v
    M = seqs * rows
    q = torch.zeros((M, 64), dtype=torch.float16, device="cuda")
    q[:, 0] = 21.484375
    plan = T.AttentionPlan(cache, 1, seqs, max_kv=n, max_rows=rows, rows=M, causal=False, scale=1.0)
    assert plan.ws_bytes == 256                                     # one part
    pages = torch.arange(n // 4096, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    y = T.attention(plan, q, torch.full((seqs,), n, dtype=torch.int32, device="cuda"), pages,
                    row_start=torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * rows).cpu().numpy().astype(np.float64)
    one = 15 * float(np.float16(1 / 15))
    w = np.exp(-21.484375 * one)
    total = 1 + (n - 1) * w
    assert 1e-3 > (total - 1) > 9e-4
    want = np.zeros(64)
    want[1], want[2] = one / total, (n - 1) * w * one / total
    # the fp32 sums of the weights: 2^21 terms over four lanes' registers and waves, each sum off by half a step of what it has
    assert np.all(np.abs(y - want) <= n * 2.0 ** -34 + 2.0 ** -11 * np.abs(want) + 2.0 ** -25)


# ---- means of the largest numbers ----------------------------------------------------------------

@pytest.mark.parametrize("tokens", [100, 600])
@pytest.mark.parametrize("rows", [16, 40, 140])
def test_means_of_the_largest_numbers(rows, tokens):
    """Values of 178 x 368 = 65504 and its negative, which the cache holds exactly: their mean is finite, whatever the probabilities' rounding
    adds up to (up to 2^-11, and from 2^-12 on the sum is nearer to 2^16).  Directly stored and joined."""
    print(f"case largest numbers, {rows} rows, {tokens} tokens", flush=True)
    seqs = 6
    b = Batch(2, [tokens] * seqs, [rows] * seqs, 2, 1, 64, 8, 64, causal=False)
    b.k[:] = 0
    b.k[np.arange(len(b.k)) % tokens % 32 == 0, ::64] = 1.0       # one token of every 32, to which the others' weights are rounded
    b.v[:] = 65504
    b.v[:, 1] = -28336                              # scale 368, zero 77
    b.v[:, 64:] = -b.v[:, :64]                      # zero 178
    b.q[:] = 0
    b.q[:, ::64] = np.linspace(0.05, 2.0, b.M)[:, None].astype(np.float16)
    b.scale = 1.0
    held = A.held(b.v, 2, 8)
    assert held.max() == 65504 and held.min() == -65504
    b.append()
    b.check(b.run(b.plan(scale=1.0)))
