"""The norm's tests again with a comparison that sees NaN: a difference that is NaN is above no bound, and below none either."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import rows_oracle as R
import test_gpu_rmsnorm as N

pytestmark = pytest.mark.gpu


def near(y, want):
    got = y.cpu().numpy().astype(np.float64)
    ok = np.abs(got - want) <= R.rmsnorm_bound(want, want.shape[1])
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])


@pytest.fixture(autouse=True)
def _near(monkeypatch):
    monkeypatch.setattr(N, "close", near)


@pytest.mark.parametrize("residual", ["", "f16", "f32"])
@pytest.mark.parametrize("D", [8, 128, 136, 512, 520, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 16392, 32768])
def test_widths(D, residual):
    N.test_widths(D, residual)


@pytest.mark.parametrize("M,D", [(700, 4096), (3001, 136), (20000, 128), (1030, 64)])
def test_many_rows(M, D):
    N.test_many_rows(M, D)


@pytest.mark.parametrize("D", [128, 1000, 4096, 16392])
@pytest.mark.parametrize("residual", ["f16", "f32"])
def test_in_place(D, residual):
    N.test_in_place(D, residual)


def test_other_calls():
    N.test_no_weights_and_large_eps()
    N.test_stream_of_large_and_tiny_numbers()
    N.test_graph_and_another_stream()


def test_near_sees_nan():
    want = np.ones((2, 8))
    near(torch.ones((2, 8)), want)
    for bad in (float("nan"), float("inf"), 1.01):
        y = torch.ones((2, 8))
        y[1, 3] = bad
        with pytest.raises(AssertionError):
            near(y, want)
