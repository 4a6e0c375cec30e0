"""The decode step that the benchmark times with attention is the one without it and what lies between (CPU, the calls recorded)."""
import pytest

torch = pytest.importorskip("torch")

import bench


class Recorder:
    def __init__(self, calls):
        self.calls = calls

    def __getattr__(self, name):
        def call(*args, **kw):
            self.calls.append((name,) + tuple(a for a in args if isinstance(a, str)))
            return 0
        return call


@pytest.mark.parametrize("chained", [True, False])
def test_attention_changes_nothing_else_of_a_layer(chained):
    lay = {n: n for n in ("o", "gate", "up", "down")}
    x, ws = torch.zeros((4, 8), dtype=torch.float16), torch.zeros(8, dtype=torch.uint8)

    def calls(attend):
        got = []
        r = Recorder(got)
        bench.decode_layer(r, r, lay, None, x, x, x, x, x, ws, chained, (lambda: got.append(("attend",))) if attend else None)
        return [c for c in got if c[0] != "current_stream_ptr"]

    ffn = [("rosaq_mlp_swiglu", "gate", "up", "down")] if chained else [("rosaq_linear_swiglu", "gate", "up"), ("linear", "down")]
    assert calls(False) == [("rosaq_linear_batch",), ("linear", "o")] + ffn
    assert calls(True) == [("rosaq_linear_batch",), ("attend",), ("linear", "o")] + ffn
