"""Attention over the quantised cache with a window and sinks on the GPU, against the fp64 oracle."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from paper_2506_13472_amd import torch_glue as T
from test_gpu_attention import Batch, _spread, dev

pytestmark = pytest.mark.gpu


class Windowed(Batch):
    """A batch whose pages that no row sees are given back: other sequences' (NaN, here) or no pages at all."""

    def __init__(self, seed, kv_lens, rows, kv, group, dim, bits, window, sinks, page=64, **kw):
        super().__init__(seed, kv_lens, rows, kv, group, dim, bits, page, **kw)
        self.window, self.sinks = window, sinks

    def plan(self, **kw):
        return super().plan(**dict(dict(window=self.window, sinks=self.sinks), **kw))

    def seen(self, i):
        """[rows, tokens] of sequence i."""
        n, r = self.kv_lens[i], self.rows[i]
        p, j = np.arange(n - r, n)[:, None], np.arange(n)[None]
        return (j <= p) & ((j > p - self.window) | (j < self.sinks))

    def give_back(self):
        rng = np.random.default_rng(1)
        data = self.cache.data.view(self.cache.num_pages, -1)
        spare = [p for p in range(self.cache.num_pages) if p not in set(self.table.reshape(-1).tolist())]
        given = 0
        for i, n in enumerate(self.kv_lens):
            used = self.seen(i).any(axis=0) if self.rows[i] else np.ones(n, bool)
            for p in range(-(-n // self.page)):
                if not used[p * self.page:(p + 1) * self.page].any():
                    data[int(self.table[i, p])] = 0xff
                    self.table[i, p] = rng.choice([-1, self.cache.num_pages, np.iinfo(np.int32).max, spare[0], int(self.table[i, p])])
                    given += 1
        return given

    def oracle(self, hidden=None):
        k, v = A.held(self.k, self.kv, self.bits), A.held(self.v, self.kv, self.bits)
        y, bound = np.full((self.M, self.kv * self.group, self.dim), 9.0), np.zeros((self.M, self.kv * self.group, self.dim))
        q, at = self.q.reshape(self.M, -1, self.dim), 0
        for i, n in enumerate(self.kv_lens):
            s = slice(self.row_start[i], self.row_start[i + 1])
            mask = self.seen(i)
            used = mask.any(axis=0)                        # the others may be NaN
            y[s], bound[s] = A.attention(q[s], k[at:at + n][used], v[at:at + n][used], mask[:, used], self.scale)
            at += n
        return y, bound


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 4), (15, 0), (16, 17), (31, 4), (33, 33), (64, 0), (100, 5), (257, 64), (700, 4), (5000, 2)])
def test_decode(bits, dim, window, sinks):
    for lens, kv, group, page in (([1, 0, 5, 16, 17, 33, 64, 65], 2, 1, 16), ([300, 7, 1000, 129], 1, 5, 64), ([2049], 1, 8, 32)):
        print(f"case window {window} sinks {sinks} int{bits} dim {dim} lens {lens} heads {kv} x {group} page {page}", flush=True)
        b = Windowed(window + bits, lens, [1] * len(lens), kv, group, dim, bits, window, sinks, page, pad=1)
        b.append()
        given = b.give_back()
        assert given or window + sinks > 100 or max(lens) < 100
        y = b.run(single=True)
        b.check(y)
        assert torch.equal(y, b.run())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,rows,kv,group,page,window,sinks", [
    ([400], [300], 1, 1, 16, 40, 3), ([700], [130], 1, 2, 64, 64, 0), ([500, 90, 3], [77, 90, 3], 2, 1, 32, 1, 0), ([260, 700], [65, 2], 1, 4, 64, 129, 70),
    ([1200], [17], 2, 1, 128, 200, 4), ([330], [5], 1, 7, 16, 31, 16), ([900, 64], [20, 0], 1, 1, 64, 63, 300), ([300], [300], 1, 1, 64, 1000, 4),
    ([20, 0, 9], [40, 2, 9], 2, 2, 16, 4, 1), ([1500], [200], 1, 1, 4096, 333, 1)])
def test_many_rows(bits, dim, lens, rows, kv, group, page, window, sinks):
    print(f"case window {window} sinks {sinks} int{bits} dim {dim} lens {lens} rows {rows} heads {kv} x {group} page {page}", flush=True)
    b = Windowed(sum(rows) + bits, lens, rows, kv, group, dim, bits, window, sinks, page, pad=2)
    b.append()
    b.give_back()
    y = b.run()
    b.check(y)
    assert torch.equal(y, b.run())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("lens,rows,kv,group,window,sinks", [
    ([20000, 100], 1, 1, 2, 9000, 4),            # parts of a sequence, joined by half waves
    ([9000], 1, 2, 1, 3000, 1000),
    ([12000], 60, 1, 1, 5000, 4), ([6000, 6000], 100, 1, 1, 2500, 200)])
def test_parts_of_a_long_window(bits, lens, rows, kv, group, window, sinks):
    print(f"case window {window} sinks {sinks} int{bits} lens {lens} rows {rows} in parts", flush=True)
    b = Windowed(7, lens, [rows] * len(lens), kv, group, 128, bits, window, sinks)
    b.append()
    b.give_back()
    plan = b.plan()
    assert plan.ws_bytes > 256
    plan.ws.fill_(0xff)
    b.check(b.run(plan))


def test_a_launch_of_waves_alone():
    """2048 short tiles and more: a wave each."""
    lens = _spread(70, 300, 3)
    for bits in (4, 8):
        print(f"case window alone int{bits}", flush=True)
        b = Windowed(bits, lens, [1] * 70, 32, 1, 64, bits, 40, 6, 16)
        b.append()
        b.give_back()
        b.check(b.run())


@pytest.mark.parametrize("rows", [1, 3, 40, 150])
def test_a_window_over_everything_is_plain_attention(rows):
    print(f"case window over everything, {rows} rows", flush=True)
    lens = [300, 1500, 150]
    b = Windowed(5, lens, [rows] * 3, 2, 2, 128, 4, 1500, 0)
    b.append()
    want = T.attention(b.plan(window=None, sinks=0), dev(b.q), dev(np.array(lens, np.int32)), dev(b.table), row_start=dev(b.row_start))
    for window, sinks in ((1500, 0), (1 << 30, 0), (1, 1500), (7, 1 << 30)):
        assert torch.equal(b.run(b.plan(window=window, sinks=sinks)), want)


@pytest.mark.parametrize("rows,window,sinks", [(1, 50, 3), (6, 50, 20), (100, 130, 3)])
def test_nan_outside_the_window_reaches_no_row(rows, window, sinks):
    print(f"case window beside NaN, {rows} rows", flush=True)
    for bits in (4, 8):
        b = Windowed(11, [700], [rows], 1, 2, 128, bits, window, sinks)
        used = b.seen(0).any(axis=0)
        b.k[~used], b.v[~used] = np.nan, np.inf
        b.append()
        b.check(b.run())
        # seen by some rows: by those alone
        last = int(np.flatnonzero(b.seen(0)[0])[-1]) - window + 1          # of the first row's window the first token
        b.v[last] = np.nan
        T.cache_append(b.cache, dev(b.slots[last:last + 1]), dev(b.k[last:last + 1]), dev(b.v[last:last + 1]))
        y = b.run().cpu().numpy()
        assert np.isnan(y[0]).all() and np.isfinite(y[1:rows]).all()


def test_lengths_beyond_the_bounds_and_rows_behind():
    """Lengths are cut to max_kv, negative ones are none; rows of no sequence, and beyond max_rows, stay as they are."""
    print("case window bounds", flush=True)
    b = Windowed(2, [200, 90], [3, 2], 1, 1, 64, 8, 20, 2, pad=3)
    b.append()
    want = b.run()
    assert bool((want[5:] == 9.0).all())
    y = torch.full_like(want, 9.0)
    lens = np.array([1 << 30, -5], np.int32)
    T.attention(b.plan(max_kv=200, max_rows=2, rows=8), dev(b.q), dev(lens), dev(b.table[:, :4]), row_start=dev(b.row_start), out=y)
    assert torch.equal(y[:2], want[:2]) and bool((y[2] == 9.0).all()) and not y[3:5].any() and bool((y[5:] == 9.0).all())


def test_two_graphs_share_a_workspace_and_another_stream():
    print("case window in graphs", flush=True)
    b = Windowed(3, [5000, 3000], [1, 1], 2, 2, 128, 4, 2000, 4)
    b.append()
    plan, q = b.plan(), dev(b.q)
    assert plan.ws_bytes > 256
    lens, table, rows = dev(np.array(b.kv_lens, np.int32)), dev(b.table), dev(b.row_start)
    ys, graphs, side = [torch.empty_like(q) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)], torch.cuda.Stream()
    torch.cuda.synchronize()
    for y, g in zip(ys, graphs):
        with torch.cuda.graph(g, stream=side):
            T.attention(plan, q, lens, table, row_start=rows, out=y)
    for i in range(4):
        plan.ws.fill_(0xff)
        for y, g in zip(ys, graphs):
            y.zero_()
            g.replay()
        torch.cuda.synchronize()
        b.q = q.cpu().numpy()
        b.check(ys[0])
        assert torch.equal(ys[0], ys[1])
        q.copy_(q.roll(1, 1))
    with torch.cuda.stream(side):
        y = T.attention(plan, q, lens, table, row_start=rows)
    side.synchronize()
    assert torch.equal(y, T.attention(b.plan(), q, lens, table, row_start=rows))
