"""Log probabilities, entropy and alternatives on the GPU, against the fp64 oracle."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import rows_oracle as R
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def rows(M, V, kind, seed=0, pad=0, shift=0, masked=0.0):
    """Logits of a type as columns of a buffer whose rows are `pad` longer, `shift` elements in."""
    rng = np.random.default_rng(seed + 31 * M + V)
    x = rng.standard_normal((M, V)) * 2.0 + 2.0 * rng.standard_normal(V)
    x[np.arange(M), rng.integers(0, V, M)] += 9.0
    if masked:
        x[:, rng.random(V) < masked] = -np.inf
        x[:, rng.integers(0, V)] = 0.5
    buf = torch.full((M * (V + pad) + shift + 64,), 300.0, dtype=TYPES[kind], device="cuda")
    view = torch.as_strided(buf, (M, V), (V + pad, 1), shift)
    view.copy_(torch.from_numpy(x).cuda())
    return view


def check(x, tokens=None, top=0, a=1.0, out=None):
    got = T.logprobs(x, tokens, top=top, scale=a, out=out)
    log_p, H, ids, bound, bound_h = R.logprobs(x.float().cpu().numpy(), a, top)

    def near(name, y, want, by):
        y = y.cpu().numpy().astype(np.float64)
        with np.errstate(invalid="ignore", over="ignore"):
            # of logits at both ends of fp32's range the difference, -6.8e38, is -inf in fp32, which the result is: its nearest number
            ok = (np.abs(y - want) <= by) | (y == want.astype(np.float32)) | (np.isnan(y) & np.isnan(want))
        assert ok.all(), (name, np.argwhere(~ok)[:5], y[~ok][:5], want[~ok][:5])
    near("entropy", got.entropy, H, bound_h)
    if tokens is not None:
        t = tokens.cpu().numpy().reshape(len(H), -1)
        at = np.clip(t, 0, x.shape[1] - 1)
        want = np.take_along_axis(log_p, at, 1)
        want[t >= x.shape[1]] = np.nan
        want[t < 0] = 0.0
        near("given", got.given, want, np.take_along_axis(bound, at, 1))
    if top:
        assert np.array_equal(got.top_ids.cpu().numpy(), ids)
        near("top", got.top, np.take_along_axis(log_p, ids, 1), np.take_along_axis(bound, ids, 1))
    return got


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 511, 1000, 2048, 2051, 4096, 8191, 32000, 50257, 131071])
def test_widths(V, kind):
    for M, pad, shift, top in ((1, 0, 0, 1), (3, 0, 0, 5), (3, 3, 1, 64), (2, 8, 7, 20)):
        print(f"case logprobs {M} x {V} {kind} pad {pad} shift {shift} top {top}", flush=True)
        x = rows(M, V, kind, top, pad, shift)
        rng = np.random.default_rng(V)
        check(x, torch.from_numpy(rng.integers(0, V, (M, 3))).cuda(), min(top, V), 1.0 if top < 20 else 0.7)


@pytest.mark.parametrize("kind", ["f16", "f32"])
@pytest.mark.parametrize("M,V", [(600, 3001), (64, 32000), (2100, 300)])
def test_many_rows(M, V, kind):
    print(f"case logprobs {M} x {V} {kind}", flush=True)
    x = rows(M, V, kind, 1)
    tokens = torch.randint(0, V, (M,), device="cuda")
    tokens[::7] = -100
    check(x, tokens, 5)
    check(x, None, 0, 1.25)


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("left", [1, 2, 19, 20, 21, 400])
def test_masked_vocabularies(left, kind):
    """Few tokens allowed: the other alternatives are the lowest of -inf."""
    print(f"case logprobs {left} allowed {kind}", flush=True)
    rng = np.random.default_rng(left)
    for V in (1003, 20011):
        x = torch.full((4, V), -np.inf, dtype=TYPES[kind], device="cuda")
        for i in range(4):
            at = torch.from_numpy(rng.permutation(V)[:left]).cuda()
            x[i, at] = torch.from_numpy(rng.standard_normal(left)).cuda().to(TYPES[kind])
        check(x, torch.arange(4, device="cuda") * 250, 20)


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_ties_and_orders(top, kind):
    """One value throughout, few values, both orders, all large ones in one thread's or one piece's share."""
    print(f"case logprobs ties {kind} {top}", flush=True)
    V = 40003
    base = torch.arange(V, device="cuda")
    x = torch.zeros((9, V), dtype=torch.float32, device="cuda")
    x[1] = (base * 7919 % 3).float()
    x[2] = base / V * 8
    x[3] = -base / V * 8
    for row, period in ((4, 4 * 1024), (5, 8 * 1024), (6, 4 * 256)):          # of 16-byte pieces over the threads of a workgroup
        x[row] = torch.where(base % period < 4, 5.0 + base / V, base % 17 / 17.0)
    x[7, 100::2] = -0.0
    x[8] = torch.where(base >= V - 70, 3.0, 0.0)
    check(x.to(TYPES[kind]), base[:9].clone(), top)


@pytest.mark.parametrize("period,width", [(8192, 8), (4096, 4), (2048, 8), (1024, 4), (8192, 32), (2048, 64)])
def test_longer_lists_than_there_is_room_for(period, width):
    """Thousands of logits, all different, in the shares of few threads and above all others."""
    V = 262144
    base = torch.arange(V, device="cuda")
    for kind in ("f16", "f32"):
        print(f"case logprobs period {period} {width} {kind}", flush=True)
        x = torch.where(base % period < width, 6.0 + (base * 40503 % 65536) / 65536.0, -2.0 - base % 5)[None].repeat(2, 1)
        x[1] = x[1].flip(0)
        x = x.to(TYPES[kind])
        check(x, base[:2].clone(), 64)
        check(x, base[:2].clone(), 64, out=T.LogProbs(*T.logprobs_buffers(x, given=1, top=64)))


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("M,V,top,given", [(1, 262144, 64, 300), (5, 65537, 20, 1), (64, 70001, 5, 2), (128, 65536, 0, 1), (2, 100003, 64, 0)])
def test_rows_shared_by_workgroups(M, V, top, given, kind):
    """With a workspace and without: the same alternatives, the same numbers but for the order of the sums."""
    print(f"case logprobs shared {M} x {V} {kind} top {top}", flush=True)
    x = rows(M, V, kind, 3, 1, 1)
    x[0, V // 2:] = x[0, 0]                   # ties across the parts
    tokens = torch.randint(-1, V, (M, given), device="cuda") if given else None
    out = T.logprobs_buffers(x, given=given, top=top)
    assert out.workspace.numel() > 256
    out.workspace.fill_(0xff)
    a = check(x, tokens, top, 0.9, out)
    b = check(x, tokens, top, 0.9, T.LogProbs(*T.logprobs_buffers(x, given=given, top=top)))
    assert T.LogProbs(*out).workspace is None and (not top or torch.equal(a.top_ids, b.top_ids))


def test_nan_infinities_and_lowest_values():
    for kind in ("f16", "bf16", "f32"):
        print(f"case logprobs not finite {kind}", flush=True)
        x = rows(9, 5000, kind, 4)
        lowest = torch.finfo(TYPES[kind]).min
        x[0, 4321] = np.nan
        x[1, 17] = np.inf
        x[2, :] = -np.inf
        x[3, :] = lowest                      # uniform
        x[4, 1:] = lowest
        x[5, 2500:] = lowest
        x[6, :] = torch.finfo(TYPES[kind]).max
        x[7, 0], x[7, 4999] = torch.finfo(TYPES[kind]).max, lowest
        x[8, 40:90] = np.nan
        tokens = torch.tensor([[4321, 0], [17, 16], [0, 1], [9, 4999], [0, 1], [3, 4000], [0, 1], [0, 4999], [40, 0]], device="cuda")
        got = check(x, tokens, 30)
        long = torch.cat((x, x, torch.full((9, 70000), -np.inf, dtype=TYPES[kind], device="cuda")), 1)        # in parts
        check(long, tokens, 30)
        assert bool((got.top_ids[8] == torch.arange(40, 70, device="cuda")).all())


def test_large_logits_lose_nothing():
    print("case logprobs far from zero", flush=True)
    x = rows(4, 3000, "f32", 5)
    far = x + 4096.0
    near = far - 4096.0                       # the same differences
    a, b = check(far, None, 5), check(near, None, 5)
    assert torch.equal(a.top_ids, b.top_ids) and torch.equal(a.top, b.top) and torch.equal(a.entropy, b.entropy)
    check(rows(4, 3000, "f16", 5) * 100, None, 5)
    check(x, None, 5, 2.0 ** -20)
    check(x, None, 5, 2.0 ** 20)


def test_tokens_outside_the_vocabulary():
    print("case logprobs tokens outside", flush=True)
    x = rows(5, 1000, "f16", 6)
    edge = np.iinfo(np.int64)
    check(x, torch.tensor([[0, 999, 1000, -1], [edge.max, edge.min, 1 << 32, -(1 << 32)], [1, 2, 3, 4], [-100] * 4, [5, 5, 5, 5]], device="cuda"))


def test_rows_past_32_bits():
    print("case logprobs rows past 32 bits", flush=True)
    V, ld = 32000, (1 << 31) + 8
    buf = torch.empty(2 * ld, dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (2, V), (ld, 1))
    x.copy_(rows(2, V, "f16", 7))
    check(x, torch.tensor([3, 31999], device="cuda"), 5)


def test_outputs_in_place_and_parts_of_them():
    x = rows(6, 700, "bf16", 8)
    out = T.logprobs_buffers(x, given=1, top=3)
    assert check(x, torch.zeros(6, dtype=torch.int64, device="cuda"), 3, out=out) is out
    assert T.logprobs(x, top=2, entropy=False).entropy is None and T.logprobs(x).top is None
    with pytest.raises(B.RosaqError):
        T.logprobs(x, entropy=False)
    for bad in (dict(tokens=torch.zeros(6, dtype=torch.int32, device="cuda")), dict(tokens=torch.zeros(5, dtype=torch.int64, device="cuda")),
                dict(top=3, out=T.logprobs_buffers(x, top=4)), dict(top=1, out=T.logprobs_buffers(x)),
                dict(tokens=torch.zeros(6, dtype=torch.int64))):
        with pytest.raises(ValueError):
            T.logprobs(x, **bad)
    for bad in (x.double(), x.t()):
        with pytest.raises(ValueError):
            T.logprobs(bad)


def test_graph_and_another_stream():
    print("case logprobs in a graph", flush=True)
    x = rows(65, 32000, "f16", 9)
    tokens = torch.randint(0, 32000, (65, 2), device="cuda")
    out = T.logprobs_buffers(x, given=2, top=5)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        T.logprobs(x, tokens, 5, out=out)
    for i in range(4):
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        eager = check(x, tokens, 5)
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        x.copy_(x.roll(1, 1))
    with torch.cuda.stream(side):
        other = T.logprobs(x, tokens, 5)
    side.synchronize()
    assert torch.equal(other.given, T.logprobs(x, tokens, 5).given)
