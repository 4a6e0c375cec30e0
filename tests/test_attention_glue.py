"""What the torch calls of the attention block refuse before anything reaches the library, without a GPU."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2506_13472_amd import torch_glue as T


def _plan(prefix_len):
    cache = types.SimpleNamespace(page_tokens=16, data=torch.empty(256, dtype=torch.uint8))
    return types.SimpleNamespace(desc=types.SimpleNamespace(), cache=cache, M=3, width=128, sequences=3, prefix_len=prefix_len,
                                 ws=torch.empty(256, dtype=torch.uint8), ws_bytes=256)


def _call(plan, **kw):
    q = torch.zeros((3, 128), dtype=torch.float16)
    return T.attention(plan, q, torch.ones(3, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), **kw)


def test_prefix_pages_and_the_plan_have_to_agree():
    pages = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="no prefix"):        # read by no one: the answer would leave the prefix out
        _call(_plan(0), prefix_pages=pages)
    with pytest.raises(ValueError, match="missing"):
        _call(_plan(20))
    with pytest.raises(ValueError, match="fewer tokens"):
        _call(_plan(33), prefix_pages=pages)
    for plan, kw in ((_plan(0), {}), (_plan(0), dict(prefix_pages=pages[:0])), (_plan(32), dict(prefix_pages=pages))):
        with pytest.raises(ValueError, match="lie on a GPU"):      # all else is right
            _call(plan, **kw)
