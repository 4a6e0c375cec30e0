"""Attention with a window where its workgroups are divided further than one round of them, on the GPU."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attention import _spread
from test_gpu_attention_window import Windowed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,dim,seqs,kv", [(4, 128, 33, 8), (8, 128, 33, 8), (8, 64, 65, 8), (4, 64, 25, 8)])
def test_more_parts_than_one_round(bits, dim, seqs, kv):
    print(f"case window of {seqs} sequences x {kv} heads, int{bits} dim {dim}", flush=True)
    lens = _spread(seqs, 2900, 5)
    lens[:3] = [2900, 1, 0]
    b = Windowed(bits + dim, lens, [1] * seqs, kv, 1, dim, bits, 2500, 4)
    b.append()
    b.give_back()
    plan = b.plan(max_kv=4000)
    row = b.M * kv * (dim + 2) * 4
    assert plan.ws_bytes // row >= 2
    plan.ws.fill_(0xff)
    y = b.run(plan, single=True)
    b.check(y)
    assert torch.equal(y, b.run(plan))
