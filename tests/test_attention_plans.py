"""How the attention's host side takes calls, without a GPU: every call ends at the workspace that it is not given."""
import pytest

from paper_2506_13472_amd import binding as B
from test_attention_abi import W, WORKSPACE, Z, _code, _desc


def test_page_table_cut_to_no_column():
    """Where no sequence has tokens of its own the table, cut to the pages in use, is empty, and an empty tensor has no address."""
    long = dict(max_kv=1 << 20, prefix_len=5, prefix_pages=Z)
    assert _code(lambda: B.rosaq_attention(_desc(pages=0, page_stride=0, **long), W, 0)) == WORKSPACE
    assert _code(lambda: B.rosaq_attention(_desc(pages=0, page_stride=1, **long), W, 0)) == -1
    assert _code(lambda: B.rosaq_attention(_desc(pages=0, page_stride=-1, **long), W, 0)) == -2
