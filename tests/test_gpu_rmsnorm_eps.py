"""The norm with an eps that fp32 does not hold, on the GPU."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import rows_oracle as R
from paper_2506_13472_amd import torch_glue as T
from test_gpu_rmsnorm import coded, data, dev
from test_gpu_rmsnorm_finite import near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("residual", ["", "f16", "f32"])
@pytest.mark.parametrize("D", [64, 4096])
def test_eps_that_fp32_does_not_hold(D, residual):
    """A row of zeros is zero with any eps above 0, and other rows are what they are with it."""
    for eps in (5e-324, 1e-310, 1e-60, 1e-46, 1e-45, 1e-40, 1.2e-38, 1e39, 1e300):
        print(f"case rmsnorm {D} {residual} eps {eps}", flush=True)
        x, w, r = data(3, D, residual)
        x[1] = 0
        if residual:
            r[1] = 0
        x[2], w[5] = np.float16(2.0 ** -24), 0
        h, y = R.rmsnorm(x, w, eps, r)
        assert np.isfinite(y).all() and not y[1].any()
        kept = lambda: None if r is None else torch.empty_like(dev(r))
        near(T.rmsnorm(dev(x), dev(w), eps, None if r is None else dev(r), kept()), y)
        out = torch.empty_like(dev(x))
        codes, scales = T.rmsnorm_codes(dev(x), dev(w), eps, None if r is None else dev(r), kept(), out=out)
        near(out, y)
        assert not bool(codes[1].any()) and float(scales[1]) == 0
        if eps < 1:                            # with large ones all values, and so the scales, are below fp32's range
            coded(codes, scales, y)


def test_infinite_weights_and_eps_above_fp32():
    """What eps takes from a value is finite, and infinite weights make infinities of it."""
    print("case rmsnorm infinite weights", flush=True)
    x, w, r = data(4, 128, "f32")
    x[x == 0], w[7] = 1, np.inf
    for res in (None, (x * np.float16(0.5)).astype(np.float16), (x * np.float32(0.5)).astype(np.float32)):
        y = T.rmsnorm(dev(x), dev(w), 1e39, None if res is None else dev(res)).cpu().numpy()
        assert np.array_equal(y[:, 7], np.sign(x[:, 7]) * np.inf) and not np.delete(y, 7, axis=1).any()
