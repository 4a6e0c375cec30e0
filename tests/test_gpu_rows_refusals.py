"""Which check of the torch calls of norm and log probabilities refuses a call with tensors on the GPU, each by its own words."""
import pytest

torch = pytest.importorskip("torch")

from paper_2506_13472_amd import torch_glue as T

pytestmark = pytest.mark.gpu

half = torch.float16


def test_rmsnorm():
    x = torch.zeros((4, 64), dtype=half, device="cuda")
    codes, scales = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    for match, kw in (("weight must", dict(weight=x[0].float())), ("weight must", dict(weight=x[0, :32])), ("weight must", dict(weight=x[0].cpu())),
                      ("residual_out without", dict(residual_out=x)), ("residual must be fp16 or fp32", dict(residual=x.bfloat16())),
                      ("residual must be a", dict(residual=x[:3])), ("one GPU", dict(residual=x.cpu())),
                      ("residual_out must", dict(residual=x.float(), residual_out=x.clone())), ("one GPU", dict(residual=x, residual_out=x.cpu())),
                      ("out must", dict(out=x.float())), ("one GPU", dict(out=x.cpu()))):
        print(f"case rmsnorm refusal {match} {list(kw)}", flush=True)
        with pytest.raises(ValueError, match=match):
            T.rmsnorm(x, **kw)
    for match, kw in (("codes must", dict(codes=codes.to(torch.uint8))), ("one GPU", dict(codes=codes.cpu())),
                      ("scales must", dict(codes=codes, scales=scales[:3])), ("scales must", dict(codes=codes, scales=scales.cpu()))):
        with pytest.raises(ValueError, match=match):
            T.rmsnorm_codes(x, **kw)


def test_logprobs():
    x = torch.zeros((4, 50), dtype=half, device="cuda")
    tokens = torch.zeros((4, 2), dtype=torch.int64, device="cuda")
    good = lambda: T.logprobs_buffers(x, given=2, top=3)
    cpu = T.logprobs_buffers(x.cpu(), given=2, top=3)
    wrong = good()
    wrong.workspace = cpu.workspace
    for match, kw in (("tokens must be a contiguous", dict(tokens=tokens.int())), ("one GPU", dict(tokens=tokens.cpu())),
                      ("out.given is missing", dict(out=T.logprobs_buffers(x, top=3))), ("out.given must", dict(out=good(), tokens=tokens[:, :1].contiguous())),
                      ("out.top_ids must", dict(out=good(), top=2)), ("one GPU", dict(out=cpu)), ("one GPU", dict(out=wrong))):
        print(f"case logprobs refusal {match} {list(kw)}", flush=True)
        with pytest.raises(ValueError, match=match):
            T.logprobs(x, **dict(dict(tokens=tokens, top=3), **kw))
    assert T.logprobs(x, tokens, top=3, out=good()).top_ids.tolist() == [[0, 1, 2]] * 4
