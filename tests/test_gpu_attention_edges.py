"""Calls of the attention block that an ordinary batch does not make: results that the calls allocate for rows without a position
or slot, tables without a column, queries that are no numbers, very long sequences, calls of very many outputs."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T
from test_gpu_attention import Batch, dev, same_bits

pytestmark = pytest.mark.gpu


# ---- more outputs than a grid of one dimension holds ---------------------------------------------

@pytest.mark.parametrize("parts,M,kv,tokens", [(2, (1 << 20) + 5, 64, 512), (17, (1 << 19) + 3, 32, 4352)])
def test_joins_of_very_many_outputs(parts, M, kv, tokens):
    """M x heads past 2^26 (up to 16 parts) and 2^24 (more of them); one sequence has the last row, all others are no one's."""
    print(f"case join of {M} x {kv} outputs, {parts} parts", flush=True)
    need = M * kv * 64 * 4 + parts * M * kv * 66 * 4 + (4 << 30)
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip(f"needs {need >> 30} GiB of device memory")
    b = Batch(1, [tokens], [1], kv, 1, 64, 4, 64)
    b.append()
    plan = b.plan(rows=M)
    assert plan.ws_bytes == parts * M * kv * 66 * 4
    q, y = (torch.empty((M, kv * 64), dtype=torch.float16, device="cuda") for _ in range(2))
    q[-1] = dev(b.q[0])
    y[-2:] = 9.0
    T.attention(plan, q, dev(np.array([tokens], np.int32)), dev(b.table), row_start=dev(np.array([M - 1, M], np.int32)), out=y)
    b.check(y[-1:])
    assert bool((y[-2] == 9.0).all())
    del plan, q, y
    torch.cuda.empty_cache()
