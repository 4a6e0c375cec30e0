"""Which check of the torch calls of norm and log probabilities refuses a call, each by its own words.  Without a GPU: that a call's tensors
do not lie on one is said last."""
import pytest

torch = pytest.importorskip("torch")

from paper_2506_13472_amd import torch_glue as T

half = torch.float16
X = torch.zeros((4, 64), dtype=half)


@pytest.mark.parametrize("match,kw", [
    ("x must be", dict(x=X.float())), ("x must be", dict(x=X.t())),
    ("weight must", dict(weight=torch.zeros(32, dtype=half))), ("weight must", dict(weight=torch.zeros(64))),
    ("weight must", dict(weight=torch.zeros(128, dtype=half)[::2])),
    ("residual_out without", dict(residual_out=X)), ("residual must be fp16 or fp32", dict(residual=X.bfloat16())),
    ("residual must be a", dict(residual=X[:3])), ("residual must be a", dict(residual=X.t())),
    ("residual_out must", dict(residual=X.float(), residual_out=X)), ("residual_out must", dict(residual=X, residual_out=X[:2])),
    ("out must", dict(out=X.float())), ("out must", dict(out=torch.zeros((64, 4), dtype=half).t())), ("out must", dict(out=X[:, :32])),
    ("lie on a GPU", {}), ("lie on a GPU", dict(weight=torch.zeros(64, dtype=half), residual=X.float(), out=X.clone()))])
def test_rmsnorm(match, kw):
    kw = dict(dict(x=X), **kw)
    with pytest.raises(ValueError, match=match):
        T.rmsnorm(**kw)
    if "out" not in kw:
        with pytest.raises(ValueError, match=match):
            T.rmsnorm_codes(**kw)


@pytest.mark.parametrize("match,kw", [
    ("codes must", dict(codes=torch.zeros((4, 64), dtype=torch.uint8))), ("codes must", dict(codes=torch.zeros((4, 32), dtype=torch.int8))),
    ("codes must", dict(codes=torch.zeros((64, 4), dtype=torch.int8).t())), ("scales must", dict(scales=torch.zeros(3))),
    ("scales must", dict(scales=torch.zeros(4, dtype=half))), ("scales must", dict(scales=torch.zeros(8)[::2])),
    ("out must", dict(out=X.float())), ("lie on a GPU", dict(out=X.clone()))])
def test_rmsnorm_codes(match, kw):
    with pytest.raises(ValueError, match=match):
        T.rmsnorm_codes(X, **kw)


def _buffers(**over):
    d = dict(given=torch.zeros((4, 2)), entropy=torch.zeros(4), top_ids=torch.zeros((4, 3), dtype=torch.int64), top=torch.zeros((4, 3)))
    return T.LogProbs(**dict(d, **over))


TOKENS = torch.zeros((4, 2), dtype=torch.int64)


@pytest.mark.parametrize("match,kw", [
    ("tokens must be \\[4, given\\]", dict(tokens=TOKENS[:3])), ("tokens must be \\[4, given\\]", dict(tokens=TOKENS[None])),
    ("tokens must be a contiguous", dict(tokens=TOKENS.int())), ("tokens must be a contiguous", dict(tokens=TOKENS.t().contiguous().t())),
    ("out.given is missing", dict(out=_buffers(given=None))), ("out.top_ids is missing", dict(out=_buffers(top_ids=None))),
    ("out.top is missing", dict(out=_buffers(top=None))),
    ("out.given must", dict(out=_buffers(given=torch.zeros((4, 1))))), ("out.given must", dict(out=_buffers(), tokens=None)),
    ("out.entropy must", dict(out=_buffers(entropy=torch.zeros((4, 1))))), ("out.entropy must", dict(out=_buffers(entropy=torch.zeros(8)[::2]))),
    ("out.top_ids must", dict(out=_buffers(top_ids=torch.zeros((4, 3), dtype=torch.int32)))), ("out.top_ids must", dict(out=_buffers(), top=0)),
    ("out.top must", dict(out=_buffers(top=torch.zeros((4, 3), dtype=half)))), ("out.top must", dict(out=_buffers(top=torch.zeros((3, 4)).t()))),
    ("lie on a GPU", dict(out=_buffers())), ("lie on a GPU", {})])
def test_logprobs(match, kw):
    kw = dict(dict(logits=torch.zeros((4, 50), dtype=half), tokens=TOKENS, top=3), **kw)
    with pytest.raises(ValueError, match=match):
        T.logprobs(**kw)
