"""What the torch calls of the norm and of the log probabilities refuse before anything reaches the library, without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2506_13472_amd import torch_glue as T

half = torch.float16


def test_rmsnorm():
    x = torch.zeros((4, 64), dtype=half)
    for match, args, kw in (("lie on a GPU", (x,), {}), ("x must be", (x.float(),), {}), ("x must be", (x.t(),), {}),
                            ("weight", (x, torch.zeros(32, dtype=half)), {}), ("weight", (x, torch.zeros(64)), {}),
                            ("residual_out without", (x,), dict(residual_out=x)), ("residual must be fp16 or fp32", (x,), dict(residual=x.bfloat16())),
                            ("residual must be a", (x,), dict(residual=x[:3])), ("residual_out must", (x,), dict(residual=x.float(), residual_out=x)),
                            ("out must", (x,), dict(out=x.float())), ("out must", (x,), dict(out=torch.zeros((64, 4), dtype=half).t()))):
        with pytest.raises(ValueError) as e:
            T.rmsnorm(*args, **kw)
        assert match in str(e.value) or "lie on a GPU" in str(e.value)      # a CPU tensor is refused as such at the latest


def test_logprobs():
    x = torch.zeros((4, 50), dtype=half)
    for bad in (x, x.float(), x.bfloat16()):
        with pytest.raises(ValueError, match="lie on a GPU"):
            T.logprobs(bad)
    with pytest.raises(ValueError, match="fp16, bf16 or fp32"):
        T.logprobs(x.double())
    with pytest.raises(ValueError, match="unit column stride"):
        T.logprobs(torch.zeros((50, 4), dtype=half).t())


def test_buffers():
    x = torch.zeros((4, 50), dtype=half)
    out = T.logprobs_buffers(x, given=2, top=3)
    assert [tuple(t.shape) for t in out] == [(4, 2), (4,), (4, 3), (4, 3)] and out.top_ids.dtype is torch.int64 and out.workspace.numel() == 256
    assert T.logprobs_buffers(x, entropy=False) == (None, None, None, None)


def test_buffers_refusals():
    x = torch.zeros((4, 50), dtype=half)
    for bad in (x.double(), x.long(), x[0], x[None]):
        with pytest.raises(ValueError, match="in fp16, bf16 or fp32"):
            T.logprobs_buffers(bad)
        with pytest.raises(ValueError, match="in fp16, bf16 or fp32"):
            T.logprobs(bad)
    for kw in (dict(given=-1), dict(top=-2)):
        with pytest.raises(ValueError, match="below zero"):
            T.logprobs_buffers(x, **kw)
