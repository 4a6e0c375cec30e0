"""Attention with a window: refusals, and the division into parts, without a GPU."""
import ctypes as C
import types

import pytest

from paper_2506_13472_amd import binding as B
from test_attention_abi import ALIGN, ARG, NULL, SHAPE, W, WORKSPACE, X, _cache, _code, _desc


def test_refusals():
    def f(window=100, sinks=4, ws=W, n=1 << 40, **over):
        return B.rosaq_attention_window(_desc(**over), window, sinks, ws, n)
    assert B.lib().rosaq_attention_window(None, 100, 4, W, 1, None) == NULL
    for window in (0, -1, (1 << 30) + 1):
        assert _code(lambda: f(window=window)) == SHAPE
        with pytest.raises(B.RosaqError):
            B.rosaq_workspace_bytes_attention_window(_desc(), window, 4)
    for sinks in (-1, (1 << 30) + 1):
        assert _code(lambda: f(sinks=sinks)) == SHAPE
        with pytest.raises(B.RosaqError):
            B.rosaq_workspace_bytes_attention_window(_desc(), 100, sinks)
    assert _code(lambda: f(causal=0)) == ARG and _code(lambda: f(prefix_len=5, prefix_pages=W)) == ARG
    # what rosaq_attention refuses
    assert _code(lambda: f(q=0)) == NULL and _code(lambda: f(q_heads=6)) == SHAPE and _code(lambda: f(y=X)) == ARG
    assert _code(lambda: f(kv_len=W + 1)) == ALIGN and _code(lambda: f(max_rows=2)) == SHAPE
    long = dict(window=1 << 20, max_kv=1 << 20, page_stride=1 << 14)
    need = B.rosaq_workspace_bytes_attention_window(_desc(max_kv=1 << 20, page_stride=1 << 14), 1 << 20, 4)
    assert need > 256
    assert _code(lambda: f(n=need - 1, **long)) == WORKSPACE and _code(lambda: f(ws=0, **long)) == WORKSPACE and _code(lambda: f(ws=W + 128, **long)) == ALIGN


def _parts(window, sinks, kv, group, M, sequences, max_rows, max_kv):
    cache = _cache(kv_heads=kv, data=0)
    d = B.AttentionDesc()
    d.cache = C.pointer(cache)
    d.q_heads, d.M, d.sequences, d.max_rows, d.max_kv, d.prefix_len, d.causal, d.scale = kv * group, M, sequences, max_rows, max_kv, 0, 1, 0.1
    n = B.rosaq_workspace_bytes_attention_window(d, window, sinks) if window else B.rosaq_workspace_bytes_attention(d)
    row = M * kv * group * (128 + 2) * 4
    assert n == 256 or n % row == 0
    return 1 if n == 256 else n // row


def test_parts_go_by_the_window():
    # one sequence's row, in parts of eight steps of 32 tokens or more.  A window of 4096 behind any text begins inside a step: 129 steps, one of sinks
    assert _parts(4096, 0, 1, 1, 1, 1, 1, 1 << 20) == 15            # 16 parts take 9 steps, and 15 of those hold 129
    assert _parts(4096, 32, 1, 1, 1, 1, 1, 1 << 20) == 15
    assert _parts(1, 0, 1, 1, 1, 1, 1, 1 << 20) == 1
    # never more than the whole text takes
    for window, sinks in ((1 << 30, 0), (1000, 1 << 30), (1 << 30, 1 << 30), (5000, 0)):
        for M, rows in ((1, 1), (40, 40), (300, 300)):
            assert _parts(window, sinks, 2, 1, M, 1, rows, 5000) == _parts(0, 0, 2, 1, M, 1, rows, 5000)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16, 17])
@pytest.mark.parametrize("max_rows", [1, 2, 7, 16, 17, 64, 65, 128, 129, 400])
@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 4), (32, 32), (33, 33), (64, 0), (1000, 5), (3000, 300)])
def test_parts_hold_all_steps(group, max_rows, window, sinks):
    """The steps of every tile, as the kernels walk them, against what the plan has room for: its parts times their steps are
    not seen from outside, so they are found again from the rules: fill / groups workgroups a tile, eight steps or two stages in each at least."""
    max_kv, rows = 6000, max_rows * group
    few = rows <= 16
    step, tile_rows = (32, 16) if few else (64, 64 if rows <= 64 else 128)
    tiles = -(-rows // tile_rows)
    apart = min(-(-(tile_rows - 1) // group), max_rows - 1)
    bound = min(-(-max_kv // step), -(-sinks // step) + -(-(window + apart + step - 1) // step))
    most = 0
    for n in (max_rows, max_rows + 1, 2999, 3000, 3007, 3040, 5999, 6000):
        for t in range(tiles):
            first, last = t * tile_rows // group, (min((t + 1) * tile_rows, rows) - 1) // group
            low = max(n - max_rows + first + 1 - window, 0)
            start = low // step * step
            over = -(-sinks // step) if sinks < start else 0
            start = 0 if sinks >= start else start
            most = max(most, over + -(-max(n - max_rows + last + 1 - start, 0) // step))
    assert most <= bound
    parts = min(max((768 if few else 512) // tiles, 1), max(1, bound // (8 if few else 2)))
    steps = -(-bound // parts)
    assert _parts(window, sinks, 1, group, max_rows, 1, max_rows, max_kv) == -(-bound // steps)


@pytest.mark.parametrize("seqs,kv,rows", [(1, 1, 1), (3, 2, 1), (16, 8, 1), (64, 8, 2), (5, 2, 12), (2, 4, 100)])
def test_parts_of_a_window_over_everything_are_those_without_one(seqs, kv, rows):
    for max_kv in (1, 64, 300, 512, 640, 1024, 1100, 5000):
        want = _parts(0, 0, kv, 1, seqs * rows, seqs, rows, max_kv)
        for window, sinks in ((max_kv, 0), (1 << 30, 0), (1, max_kv), (max_kv, max_kv)):
            assert _parts(window, sinks, kv, 1, seqs * rows, seqs, rows, max_kv) == want


def test_few_steps_stay_whole():
    # a window of w that begins anywhere in a step of 32 tokens takes up to (w + 31) / 32, rounded up, of them, and four sinks one: 560 take 19 + 1, 1024 33 + 1
    for window, whole in ((100, True), (500, True), (560, False), (640, False)):
        assert (_parts(window, 4, 8, 4, 4, 4, 1, 4000) == 1) == whole
    for window, whole in ((640, True), (1024, True), (1100, False)):
        assert (_parts(window, 4, 8, 4, 16, 16, 1, 4000) == 1) == whole


def test_torch_plan_refusals():
    torch = pytest.importorskip("torch")
    from paper_2506_13472_amd import torch_glue as T
    cache = types.SimpleNamespace(args=_cache(kv_heads=2, head_dim=64, data=0), head_dim=64, data=torch.empty(1))
    with pytest.raises(ValueError, match="window is missing"):
        T.AttentionPlan(cache, q_heads=2, sequences=1, max_kv=64, sinks=4)
    for kw in (dict(window=0), dict(window=8, sinks=-1), dict(window=8, prefix_len=3), dict(window=8, causal=False)):
        with pytest.raises(B.RosaqError):
            T.AttentionPlan(cache, q_heads=2, sequences=1, max_kv=64, **kw)
    assert T.AttentionPlan(cache, q_heads=2, sequences=1, max_kv=64, window=8).sinks == 0
