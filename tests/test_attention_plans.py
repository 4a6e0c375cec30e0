"""How the attention's host side takes calls, without a GPU: every call ends at the workspace that it is not given."""
import ctypes as C

import pytest

from paper_2506_13472_amd import binding as B
from test_attention_abi import W, WORKSPACE, Z, _code, _desc


def test_page_table_cut_to_no_column():
    """Where no sequence has tokens of its own the table, cut to the pages in use, is empty, and an empty tensor has no address."""
    long = dict(max_kv=1 << 20, prefix_len=5, prefix_pages=Z)
    assert _code(lambda: B.rosaq_attention(_desc(pages=0, page_stride=0, **long), W, 0)) == WORKSPACE
    assert _code(lambda: B.rosaq_attention(_desc(pages=0, page_stride=1, **long), W, 0)) == -1
    assert _code(lambda: B.rosaq_attention(_desc(pages=0, page_stride=-1, **long), W, 0)) == -2


def _parts(kv, group, dim, bits, M, sequences, max_rows, max_kv, prefix_len):
    """The number of parts of a row, from the size of the workspace: a sum a channel, a reference and a sum of weights, in fp32."""
    cache = B.Cache(kv_heads=kv, head_dim=dim, bits=bits, page_tokens=32, num_pages=10, data=None)
    d = B.AttentionDesc()
    d.cache = C.pointer(cache)
    d.q_heads, d.M, d.sequences, d.max_rows, d.max_kv, d.prefix_len, d.causal, d.scale = kv * group, M, sequences, max_rows, max_kv, prefix_len, 1, 0.1
    n = B.rosaq_workspace_bytes_attention(d)
    row = M * kv * group * (dim + 2) * 4
    assert n == 256 or n % row == 0
    return 1 if n == 256 else n // row


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("prefix,seqs,rows,max_kv,kv,group,dim,own,shared", [
    (2100, 40, 1, 90, 2, 1, 128, 1, 11), (2075, 60, 1, 40, 2, 1, 64, 1, 11), (3001, 40, 3, 70, 1, 4, 128, 1, 16), (5000, 24, 2, 9, 1, 8, 64, 1, 27),
    (200, 64, 1, 40, 32, 1, 64, 1, 2), (130, 64, 1, 33, 32, 2, 64, 1, 1), (161, 64, 1, 5, 32, 1, 128, 1, 1), (150, 70, 1, 0, 32, 2, 128, 1, 1)])
def test_prefix_apart_has_its_own_parts(bits, prefix, seqs, rows, max_kv, kv, group, dim, own, shared):
    """The sequences' own tokens are one part here; the prefix is in as many as its stages of 64 tokens, two of them each at least, and the
    workgroups for its rows (256 for up to 64 of them, 512) allow.  One row a sequence more than a tile holds, and all is one sequence's again."""
    M = seqs * rows + 2
    assert _parts(kv, group, dim, bits, M, seqs, rows, max_kv, prefix) == own + shared
    tile_rows = 16 // group
    together = _parts(kv, group, dim, bits, seqs * (tile_rows + 1), seqs, tile_rows + 1, max_kv, prefix)
    assert together != own + shared


def test_a_prefix_that_saves_little_stays_with_its_sequences():
    assert _parts(32, 1, 128, 4, 64, 64, 1, 256, 64) == 1          # 63 x 32 x 2 steps saved, 64 x 32 results to join and 3000
    assert _parts(32, 1, 128, 4, 64, 64, 1, 256, 65) == 2
    assert _parts(8, 4, 128, 8, 1, 1, 1, 256, 4096) == 17          # one sequence shares with no one: 136 steps, eight a workgroup

