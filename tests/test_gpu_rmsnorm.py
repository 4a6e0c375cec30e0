"""The norm in front of the projections on the GPU, against the fp64 oracle."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import rows_oracle as R
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T

pytestmark = pytest.mark.gpu

TYPES = {"f16": np.float16, "f32": np.float32}


def dev(x, pad=0):
    """On the GPU, as columns of a wider buffer where pad is given."""
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    if not pad:
        return t
    buf = torch.full((x.shape[0], x.shape[1] + pad), 7, dtype=t.dtype, device="cuda")
    buf[:, :x.shape[1]] = t
    return buf[:, :x.shape[1]]


def data(M, D, residual, seed=0):
    rng = np.random.default_rng(seed + 7 * M + D)
    x = rng.standard_normal((M, D)).astype(np.float16)
    w = (1 + 0.3 * rng.standard_normal(D)).astype(np.float16)
    r = (rng.standard_normal((M, D)) * np.exp(rng.standard_normal(D))).astype(TYPES[residual]) if residual else None
    return x, w, r


def close(y, want):
    got = y.cpu().numpy().astype(np.float64)
    far = np.abs(got - want) > R.rmsnorm_bound(want, want.shape[1])
    assert not far.any(), (np.argwhere(far)[:5], got[far][:5], want[far][:5])


def kept(out, x, r):
    """The sum, rounded to fp32 and from there to the stream's type."""
    want = (x.astype(np.float32) + r.astype(np.float32)).astype(r.dtype)
    assert np.array_equal(out.cpu().numpy(), want)


def coded(codes, scales, y):
    scale, at = R.codes(y)
    got = scales.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - np.abs(y).max(1) / 127) <= 2.0 ** -24 * (1 + 1e-6) * got)        # one rounding to fp32
    at = y / np.where(got > 0, got, 1.0)[:, None]
    # the nearest whole number, where fp64 sums in another order do not decide
    assert np.all(np.abs(codes.cpu().numpy() - at) <= 0.5 + 1e-9)


@pytest.mark.parametrize("residual", ["", "f16", "f32"])
@pytest.mark.parametrize("D", [8, 64, 128, 136, 512, 520, 1000, 2048, 2056, 4096, 4104, 5120, 8192, 8200, 16384, 16392, 32768])
def test_widths(D, residual):
    for M, pad in ((1, 0), (5, 8), (18, 0)):
        print(f"case rmsnorm {M} x {D} {residual} pad {pad}", flush=True)
        x, w, r = data(M, D, residual)
        h, y = R.rmsnorm(x, w, 1e-5, r)
        xd, rd = dev(x, pad), None if r is None else dev(r, pad)
        out = dev(np.full((M, D), 3, np.float16), pad)
        total = None if r is None else torch.empty_like(rd)
        assert T.rmsnorm(xd, dev(w), 1e-5, rd, total, out) is out
        close(out, y)
        if r is not None:
            kept(total, x, r)
            assert np.array_equal(rd.cpu().numpy(), r)
        codes, scales = T.rmsnorm_codes(xd, dev(w), 1e-5, rd, total)
        coded(codes, scales, y)
        if pad:
            for t in (xd, out) + (() if r is None else (rd,)):
                assert bool((t._base[:, D:] == 7).all())


@pytest.mark.parametrize("M,D", [(700, 4096), (3001, 136), (20000, 128), (257, 5120), (1030, 64)])
def test_many_rows(M, D):
    print(f"case rmsnorm {M} x {D}", flush=True)
    x, w, r = data(M, D, "f16")
    h, y = R.rmsnorm(x, w, 1e-6, r)
    rd, both = dev(r), dev(np.zeros((M, D), np.float16))
    codes, scales = T.rmsnorm_codes(dev(x), dev(w), 1e-6, rd, torch.empty_like(rd), out=both)
    close(both, y)
    coded(codes, scales, y)
    close(T.rmsnorm(dev(x), dev(w), 1e-6, rd), y)              # the stream is kept in its place
    kept(rd, x, r)


@pytest.mark.parametrize("D", [128, 1000, 4096, 16392])
@pytest.mark.parametrize("residual", ["f16", "f32"])
def test_in_place(D, residual):
    print(f"case rmsnorm in place {D} {residual}", flush=True)
    x, w, r = data(9, D, residual, 3)
    h, y = R.rmsnorm(x, w, 1e-5, r)
    xd, rd = dev(x, 16), dev(r, 16)
    assert T.rmsnorm(xd, dev(w), residual=rd, out=xd) is xd
    close(xd, y)
    kept(rd, x, r)
    if residual == "f16":                                      # each in the other's place
        xd, rd = dev(x), dev(r)
        T.rmsnorm(xd, dev(w), residual=rd, residual_out=xd, out=rd)
        close(rd, y)
        kept(xd, x, r)


def test_no_weights_and_large_eps():
    x, w, r = data(6, 256, "f32", 5)
    print("case rmsnorm without weights", flush=True)
    close(T.rmsnorm(dev(x), eps=0.0), R.rmsnorm(x, eps=0.0)[1])
    close(T.rmsnorm(dev(x), dev(w), eps=1e6), R.rmsnorm(x, w, 1e6)[1])
    codes, scales = T.rmsnorm_codes(dev(x), eps=1e-5)
    coded(codes, scales, R.rmsnorm(x, eps=1e-5)[1])


def test_stream_of_large_and_tiny_numbers():
    """Squares that fp32 does not hold, sums that fp16 does not hold."""
    print("case rmsnorm of large and tiny numbers", flush=True)
    x, w, r = data(4, 264, "f32", 6)
    r[0] *= np.float32(1e30)
    r[1] *= np.float32(1e-30)
    r[2] *= np.float32(1e38 / np.abs(r[2]).max())
    x[1] = 0
    h, y = R.rmsnorm(x, w, 0.0, r)
    rd = dev(r)
    close(T.rmsnorm(dev(x), dev(w), 0.0, rd, torch.empty_like(rd)), y)
    coded(*T.rmsnorm_codes(dev(x), dev(w), 0.0, rd, torch.empty_like(rd)), y)
    big = np.full((2, 64), 60000, np.float16)
    rd = dev(big)
    got = T.rmsnorm(dev(big), eps=0.0, residual=rd)
    assert bool(torch.isinf(rd).all()) and bool((got == 1.0).all())


def test_zeros_infinities_and_nan():
    print("case rmsnorm of zeros, infinities, NaN", flush=True)
    x = np.ones((5, 136), np.float16)
    x[0] = 0
    x[1, 77] = np.inf
    x[2, 3] = np.nan
    x[3, 0], x[3, 1] = np.inf, -np.inf
    y = T.rmsnorm(dev(x), eps=1e-5).cpu().numpy()
    assert not y[0].any() and np.isnan(y[1, 77]) and not np.delete(y[1], 77).any() and np.isnan(y[2]).all()
    assert np.isnan(y[3, :2]).all() and not y[3, 2:].any() and np.all(np.abs(y[4] - 1) < 1e-3)
    codes, scales = (t.cpu().numpy() for t in T.rmsnorm_codes(dev(x), eps=1e-5))
    assert scales[0] == 0 and np.isnan(scales[1:4]).all() and not codes[:4].any() and (codes[4] == 127).all()
    assert np.isnan(T.rmsnorm(dev(x[:1]), eps=0.0).cpu().numpy()).all()


def test_graph_and_another_stream():
    """Captured on a side stream and replayed with the program's own work between: every replay adds to the stream once more."""
    print("case rmsnorm in a graph", flush=True)
    x, w, r = data(33, 4096, "f32", 8)
    xd, wd, rd = dev(x), dev(w), dev(r)
    y, codes, scales = torch.empty_like(xd), torch.empty((33, 4096), dtype=torch.int8, device="cuda"), torch.empty(33, device="cuda")
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        T.rmsnorm_codes(xd, wd, 1e-5, rd, codes=codes, scales=scales, out=y)
    for i in range(4):
        g.replay()
        torch.cuda.synchronize()
        total = (x.astype(np.float32) + r).astype(np.float32)
        h, want = R.rmsnorm(x, w, 1e-5, r)
        close(y, want)
        coded(codes, scales, want)
        kept(rd, x, r)
        r = total
        x = (x * np.float16(0.5)).astype(np.float16)
        xd.mul_(0.5)
    with torch.cuda.stream(side):
        eager = T.rmsnorm(xd, wd, 1e-5, rd)
    side.synchronize()
    close(eager, R.rmsnorm(x, w, 1e-5, r)[1])


def test_refusals_of_the_torch_call():
    x = torch.zeros((4, 64), dtype=torch.float16, device="cuda")
    for bad in (dict(weight=torch.zeros(32, dtype=torch.float16, device="cuda")), dict(weight=torch.zeros(64, device="cuda")),
                dict(residual=torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")), dict(residual_out=x.clone()),
                dict(residual=torch.zeros((4, 64), device="cuda"), residual_out=x.clone()), dict(out=x.float()),
                dict(residual=torch.zeros((4, 64), dtype=torch.float16)), dict(residual=torch.zeros((3, 64), dtype=torch.float16, device="cuda"))):
        with pytest.raises(ValueError):
            T.rmsnorm(x, **bad)
    with pytest.raises(ValueError):
        T.rmsnorm_codes(x, codes=torch.zeros((4, 64), dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        T.rmsnorm_codes(x, scales=torch.zeros(3, device="cuda"))
    with pytest.raises(B.RosaqError):
        T.rmsnorm(x[:, :36].contiguous())
