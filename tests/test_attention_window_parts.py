"""How a call with a window over up to 16 rows is divided, by the evenness of its workgroups over 256 compute units.  Without a GPU."""
import ctypes as C

import pytest

from paper_2506_13472_amd import binding as B
from test_attention_abi import _cache


def _parts(window, sequences, kv, max_kv, bits, sinks=4):
    cache = _cache(kv_heads=kv, bits=bits, data=0)
    d = B.AttentionDesc()
    d.cache = C.pointer(cache)
    d.q_heads, d.M, d.sequences, d.max_rows, d.max_kv, d.prefix_len, d.causal, d.scale = 4 * kv, sequences, sequences, 1, max_kv, 0, 1, 0.1
    n = B.rosaq_workspace_bytes_attention_window(d, window, sinks) if window else B.rosaq_workspace_bytes_attention(d)
    row = sequences * 4 * kv * (128 + 2) * 4
    assert n == 256 or n % row == 0
    return 1 if n == 256 else n // row


@pytest.mark.parametrize("bits,most", [(4, 1.15), (8, 1.31)])
def test_no_compute_unit_has_far_more_than_the_average(bits, most):
    for groups in list(range(64, 1100, 3)) + [257, 264, 320, 392, 513, 520, 640, 769, 776, 1024, 1025, 2047]:
        n = groups * _parts(4096, groups, 1, 65536, bits)
        assert -(-n // 256) * 256 <= most * n, groups


@pytest.mark.parametrize("bits", [4, 8])
def test_few_steps_take_one_round(bits):
    for groups in (97, 264, 320, 520, 776):
        assert _parts(2000, groups, 1, 65536, bits) == max((768 if bits == 4 else 512) // groups, 1)


@pytest.mark.parametrize("bits", [4, 8])
def test_one_round_where_it_is_even(bits):
    """As many workgroups as are resident at a time: three a compute unit with 4 bits, two with 8."""
    resident = 768 if bits == 4 else 512
    for groups in (64, 128, 256):
        assert groups * _parts(4096, groups // 8, 8, 65536, bits) == resident
    for groups in (512, 768, 1024):
        assert _parts(4096, groups // 8, 8, 65536, bits) == 1
