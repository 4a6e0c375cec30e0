"""Where the benchmark's decode step takes its norms (CPU, the calls recorded)."""
import pytest

torch = pytest.importorskip("torch")

import bench
from test_bench_decode import Recorder


@pytest.mark.parametrize("chained", [True, False])
def test_norms_stand_in_front_of_both_halves(chained):
    lay = {n: n for n in ("o", "gate", "up", "down")}
    x, ws = torch.zeros((4, 8), dtype=torch.float16), torch.zeros(8, dtype=torch.uint8)
    got = []
    r = Recorder(got)
    bench.decode_layer(r, r, lay, None, x, x, x, x, x, ws, chained, lambda: got.append(("attend",)), lambda: got.append(("norm",)))
    ffn = [("rosaq_mlp_swiglu", "gate", "up", "down")] if chained else [("rosaq_linear_swiglu", "gate", "up"), ("linear", "down")]
    assert [c for c in got if c[0] != "current_stream_ptr"] == \
        [("norm",), ("rosaq_linear_batch",), ("attend",), ("linear", "o"), ("norm",)] + ffn
