"""Numbers that the C ABI's int32 does not hold are refused, not cut to their low 32 bits.  Without a GPU."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T
from test_attention_abi import SHAPE, W, _cache, _desc

FAR = (1 << 32) + 1, 1 << 32, (1 << 31) + 7, -(1 << 32) + 8          # cut, these are 1, 0, a number below zero, and 8


def _code(fn):
    with pytest.raises(B.RosaqError, match="int32") as e:
        fn()
    return e.value.code


@pytest.mark.parametrize("far", FAR)
def test_window_and_sinks(far):
    for window, sinks in ((far, 4), (100, far)):
        assert _code(lambda: B.rosaq_attention_window(_desc(), window, sinks, W, 1 << 40)) == SHAPE
        assert _code(lambda: B.rosaq_workspace_bytes_attention_window(_desc(), window, sinks)) == SHAPE


@pytest.mark.parametrize("far", FAR)
def test_plan(far):
    cache = types.SimpleNamespace(args=_cache(kv_heads=2, head_dim=64, data=0), head_dim=64, data=torch.empty(1))
    good = dict(q_heads=2, sequences=1, max_kv=64)
    T.AttentionPlan(cache, **good)
    for name in ("q_heads", "sequences", "max_kv", "max_rows", "rows", "prefix_len", "window"):
        assert _code(lambda: T.AttentionPlan(cache, **dict(good, **{name: far}))) == SHAPE, name
    assert _code(lambda: T.AttentionPlan(cache, **good, window=8, sinks=far)) == SHAPE


def test_cache():
    good = dict(kv_heads=1, head_dim=64, bits=4, page_tokens=16, num_pages=3)
    for name in good:
        for far in FAR:
            assert _code(lambda: B.rosaq_cache_bytes(**dict(good, **{name: far}))) == SHAPE
    assert _code(lambda: T.KvCache(1, 64, 4, 16, (1 << 32) + 3, device="cpu")) == SHAPE


def _far_matrices(dtype):
    """Shapes past int32, of tensors that have no memory."""
    return [torch.empty(shape, dtype=dtype, device="meta") for shape in ((1, (1 << 32) + 8), ((1 << 32) + 1, 8))]


def test_norm():
    for x in _far_matrices(torch.float16):
        assert _code(lambda: T.rmsnorm(x)) == SHAPE
        codes, scales = torch.empty(x.shape, dtype=torch.int8, device="meta"), torch.empty(x.shape[0], device="meta")
        assert _code(lambda: T.rmsnorm_codes(x, codes=codes, scales=scales)) == SHAPE


def test_logprobs():
    for x in _far_matrices(torch.float32):
        assert _code(lambda: T.logprobs(x)) == SHAPE
        assert _code(lambda: T.logprobs_buffers(x)) == SHAPE
    x = torch.empty((1, 50), device="meta")
    for top in FAR[:3]:
        assert _code(lambda: T.logprobs_buffers(x, top=top)) == SHAPE
        assert _code(lambda: T.logprobs(x, top=top)) == SHAPE
        assert _code(lambda: T.logprobs_buffers(x, given=top)) == SHAPE
    tokens = torch.empty((1, (1 << 32) + 1), dtype=torch.int64, device="meta")
    assert _code(lambda: T.logprobs(x, tokens)) == SHAPE
