"""Norm, log probabilities and attention with a window: calls that an ordinary program does not make."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from oracle import rows_oracle as R
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T
from test_gpu_attention import dev
from test_gpu_attention_window import Windowed
from test_gpu_logprobs import TYPES, check, rows
from test_gpu_rmsnorm import close, coded, kept

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,D", [((1 << 20) + 5, 520), ((1 << 22) + 9, 136), ((1 << 24) + 37, 8)])
def test_norm_of_more_rows_than_a_grid_has(M, D):
    """Workgroups take further rows in turn beyond 2^20 of them."""
    print(f"case rmsnorm {M} x {D}", flush=True)
    x = torch.randn((4096, D), device="cuda").half().repeat(M // 4096 + 1, 1)[:M]
    r = x.roll(1, 0)
    y, total = torch.zeros_like(x), torch.empty_like(x)
    T.rmsnorm(x, residual=r, residual_out=total, out=y)
    some = torch.cat((torch.arange(64), torch.arange(M - 300, M), torch.randint(0, M, (200,)))).cuda()
    xs, rs = x[some].cpu().numpy(), r[some].cpu().numpy()
    close(y[some], R.rmsnorm(xs, None, 1e-5, rs)[1])
    kept(total[some], xs, rs)
    assert bool((y.abs().amax(dim=1) > 0).all())


@pytest.mark.parametrize("M,D", [((1 << 20) + 5, 1032), ((1 << 20) + 300, 4096), ((1 << 22) + 9, 136)])
def test_codes_of_more_rows_than_a_grid_has(M, D):
    print(f"case rmsnorm codes {M} x {D}", flush=True)
    x = torch.randn((4096, D), device="cuda").half().repeat(M // 4096 + 1, 1)[:M]
    x[(1 << 20) - 1] = 0                       # its place's next row is not of zeros
    codes, scales = T.rmsnorm_codes(x)
    some = torch.cat((torch.arange(64), torch.arange((1 << 20) - 2, (1 << 20) + 5), torch.arange(M - 300, M), torch.randint(0, M, (200,)))).cuda()
    coded(codes[some], scales[some], R.rmsnorm(x[some].cpu().numpy())[1])
    assert int((codes.view(torch.int32) != 0).any(dim=1).sum()) == M - 1


def test_norm_of_rows_past_32_bits():
    print("case rmsnorm rows past 32 bits", flush=True)
    D, ld = 1000, (1 << 31) + 64
    buf = torch.empty(2 * ld, dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (2, D), (ld, 1))
    x.copy_(torch.randn((2, D), device="cuda"))
    want = x.cpu().numpy()
    y = T.rmsnorm(x, out=x)
    close(y, R.rmsnorm(want)[1])


def test_norm_of_a_negative_zero_and_of_subnormals():
    """Nothing of a row is lost below fp16's and fp32's normal numbers."""
    print("case rmsnorm subnormals", flush=True)
    x = np.full((3, 64), 2.0 ** -24, np.float16)
    x[1] = -0.0
    x[2, ::2] = -2.0 ** -24
    close(T.rmsnorm(dev(x), eps=0.0)[[0, 2]], R.rmsnorm(x[[0, 2]], eps=0.0)[1])
    r = np.full((3, 64), 1e-44, np.float32)
    zero = np.zeros((3, 64), np.float16)
    rd = dev(r)
    close(T.rmsnorm(dev(zero), eps=0.0, residual=rd), R.rmsnorm(zero, None, 0.0, r)[1])
    w = np.full(64, 2.0 ** -24, np.float16)
    codes, scales = T.rmsnorm_codes(dev(x), dev(w), 1.0)          # values of 2^-48 and below
    coded(codes, scales, R.rmsnorm(x, w, 1.0)[1])
    tiny = np.full((2, 64), 1e-38, np.float32)
    tiny[1, 1:] = 3e-39
    codes, scales = T.rmsnorm_codes(dev(zero[:2]), None, 1e4, residual=dev(tiny))        # scales among fp32's subnormals: codes stay in their range
    assert int(codes.min()) >= -127 and bool((scales >= 0).all()) and int(codes[0].min()) == int(codes[0].max())


def test_logprobs_of_more_rows_than_a_grid_has():
    print("case logprobs of many rows", flush=True)
    M = (1 << 20) + 11
    x = torch.randn((M, 6), device="cuda")
    got = T.logprobs(x, torch.arange(M, device="cuda") % 6, top=2)
    some = torch.cat((torch.arange(50), torch.arange(M - 60, M))).cuda()
    log_p, H, ids, bound, bound_h = R.logprobs(x[some].cpu().numpy(), 1.0, 2)
    t = (some % 6).cpu().numpy()[:, None]
    assert np.all(np.abs(got.given[some].cpu().numpy() - np.take_along_axis(log_p, t, 1)) <= np.take_along_axis(bound, t, 1))
    assert np.array_equal(got.top_ids[some].cpu().numpy(), ids) and np.all(np.abs(got.entropy[some].cpu().numpy() - H) <= bound_h)


def test_logprobs_read_nothing_beside_their_rows():
    """Rows at any element, with what would be the largest logits right before and behind them."""
    for kind in ("f16", "bf16", "f32"):
        print(f"case logprobs beside others {kind}", flush=True)
        for V in (5, 63, 64, 65, 4097):
            for shift in range(9):
                x = rows(2, V, kind, shift, pad=3, shift=shift)          # 300 in the gaps
                check(x, torch.zeros((2, 1), dtype=torch.int64, device="cuda"), min(V, 9))


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("top", [2, 31, 32, 33])
def test_alternatives_from_a_count_and_from_a_search(top, kind):
    """Both ways to the bound: few and many values, all large ones in few threads' shares, rows of few pieces."""
    for V in (40, 300, 9000, 40003, 140001):
        print(f"case logprobs {top} of {V} {kind}", flush=True)
        base = torch.arange(V, device="cuda")
        x = torch.zeros((7, V), dtype=torch.float32, device="cuda")
        x[1] = (base * 7919 % 3).float()
        x[2] = (base * 40503 % 65536) / 65536.0
        x[3] = torch.where(base % 4096 < 8, 6.0 + (base * 40503 % 65536) / 65536.0, -2.0 - base % 5)
        x[4] = torch.where(base % 2048 < 4, 6.0 + (base * 40503 % 65536) / 65536.0, -2.0 - base % 5)
        x[5] = torch.where(base < top - 1, 1.0, -np.inf)
        x[6, V // 2] = np.nan
        check(x.to(TYPES[kind]), base[:7].clone(), top)


def test_small_scales_leave_nothing_of_minus_infinity():
    for kind in ("f16", "bf16", "f32"):
        print(f"case logprobs small scales {kind}", flush=True)
        x = rows(3, 5000, kind, masked=0.5)
        for a in (1e-3, 2.0 ** -20, 2.0 ** -60):
            check(x, torch.tensor([1, 2, 3], device="cuda"), 5, a)


def test_two_graphs_of_logprobs_share_a_workspace():
    print("case logprobs in graphs", flush=True)
    xs = [rows(3, 70000, "f16", s) for s in (1, 2)]
    outs = [T.logprobs_buffers(x, top=7) for x in xs]
    outs[1].workspace = outs[0].workspace
    assert outs[0].workspace.numel() > 256
    graphs, side = [torch.cuda.CUDAGraph() for _ in xs], torch.cuda.Stream()
    torch.cuda.synchronize()
    for x, out, g in zip(xs, outs, graphs):
        with torch.cuda.graph(g, stream=side):
            T.logprobs(x, top=7, out=out)
    for i in range(4):
        outs[0].workspace.fill_(0xff)
        for out, g in zip(outs, graphs):
            for t in out[1:]:
                t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for x, out in zip(xs, outs):
            assert all(torch.equal(a, b) for a, b in zip(out[1:], check(x, None, 7)[1:]))
            x.copy_(x.roll(5, 1))


def test_window_offsets_beyond_32_bits_and_strides():
    """Pages past 4 GiB of a cache, queries and answers as columns of wider buffers."""
    print("case window far pages", flush=True)
    cache = T.KvCache(8, 128, 8, 128, 20000)
    assert cache.data.numel() > 5 << 30
    rng = np.random.default_rng(4)
    n, rows, window, sinks = 700, 150, 130, 5
    pages = np.array([[19999, 0, 12345, 19000, 3, 18888]], np.int32)
    t = np.arange(n)
    slots = pages[0][t // 128].astype(np.int64) * 128 + t % 128
    k, v = (rng.standard_normal((n, 1024)).astype(np.float16) for _ in range(2))
    T.cache_append(cache, dev(slots), dev(k), dev(v))
    for m in (1, rows):
        q = rng.standard_normal((m, 1024)).astype(np.float16)
        wide = torch.full((m, 3584), 7.0, dtype=torch.float16, device="cuda")
        wide[:, :1024] = dev(q)
        plan = T.AttentionPlan(cache, 8, 1, max_kv=768, max_rows=m, window=window, sinks=sinks)
        T.attention(plan, wide[:, :1024], dev(np.array([n], np.int32)), dev(pages), row_start=dev(np.array([0, m], np.int32)), out=wide[:, 2560:])
        p, j = np.arange(n - m, n)[:, None], np.arange(n)[None]
        mask = (j <= p) & ((j > p - window) | (j < sinks))
        pick = [0, m // 2, m - 1] if m > 1 else [0]
        want, bound = A.attention(q.reshape(m, 8, 128)[pick], A.held(k, 8, 8), A.held(v, 8, 8), mask[pick], 128 ** -0.5)
        got = wide[:, 2560:].cpu().numpy().reshape(m, 8, 128)[pick].astype(np.float64)
        assert np.all(np.abs(got - want) <= bound) and bool((wide[:, 1024:2560] == 7.0).all())


@pytest.mark.parametrize("rows", [1, 6, 90])
def test_window_at_the_largest_numbers(rows):
    """A window and sinks of 2^30 tokens each, and a window of one, over lengths that move from call to call."""
    print(f"case window bounds, {rows} rows", flush=True)
    b = Windowed(9, [400], [rows], 2, 1, 64, 4, 1 << 30, 1 << 30, 16)
    b.append()
    b.check(b.run())
    q, table, start = dev(b.q), dev(b.table), dev(b.row_start)
    one = b.plan(window=1, sinks=0)
    for n in (rows, rows + 1, 255, 256, 257, 400):
        b.kv_lens, b.window, b.sinks = [n], 1, 0
        y = T.attention(one, q, dev(np.array([n], np.int32)), table, row_start=start)
        # every row sees its own token alone
        want = A.held(b.v, 2, 4)[n - rows:n].reshape(rows, -1)
        assert np.all(np.abs(y.cpu().numpy().astype(np.float64) - want) <= 2.0 ** -10 * np.abs(want) + 2.0 ** -12)


def test_c_calls_take_null_for_what_is_not_wanted():
    """Straight through the C ABI, on the default stream."""
    print("case C calls", flush=True)
    x = torch.randn((5, 256), device="cuda").half()
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    d = B.RmsNormDesc()
    d.M, d.D, d.eps, d.x, d.ldx, d.y, d.ldy = 5, 256, 1e-5, x.data_ptr(), 256, y.data_ptr(), 256
    assert B.lib().rosaq_rmsnorm(C.byref(d), None) == 0
    h = torch.empty(5, device="cuda")
    l = B.LogprobsDesc()
    l.M, l.V, l.type, l.scale, l.logits, l.ld, l.entropy = 5, 256, B.F16, 1.0, x.data_ptr(), 256, h.data_ptr()
    assert B.lib().rosaq_logprobs(C.byref(l), None, 0, None) == 0
    torch.cuda.synchronize()
    close(y, R.rmsnorm(x.cpu().numpy())[1])
    log_p, H, ids, bound, bound_h = R.logprobs(x.float().cpu().numpy())
    assert np.all(np.abs(h.cpu().numpy() - H) <= bound_h)
