"""Log probabilities of logits whose difference fp32 does not hold, on the GPU."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_logprobs import TYPES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 300, 70000])
def test_logits_at_both_ends_of_the_range(V, kind):
    """A difference of logits beyond fp32 whose product with the scale is not."""
    big = 3.4028234663852886e38 if kind == "f32" else 3.3895313892515355e38
    x = torch.full((4, V), -big, dtype=torch.float64)
    x[0, 1], x[1, 2:4], x[2, 0] = big, big, big / 2
    x[3] = -np.inf
    x[3, 1], x[3, 4] = big, -big
    x = x.to(TYPES[kind]).cuda()
    tokens = torch.tensor([[0, 1, 4]] * 4, device="cuda")
    for a in (1.0, 0.5, 0.25, 1e-3, 2.0 ** -40, 2.0 ** -60):
        print(f"case logprobs {V} {kind} scale {a}", flush=True)
        got = check(x, tokens, min(V, 5), a)
        assert bool(torch.isfinite(got.given[:3]).all()) == (a < 1) and float(got.given[3, 0]) == -np.inf
