"""Norms, projections, cache, attention with a window and log probabilities as one decoder pass, every stage against the oracle on what
the stage before gave."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_oracle as A
from oracle import rosaq_oracle as O
from oracle import rows_oracle as R
from paper_2506_13472_amd import binding as B
from paper_2506_13472_amd import torch_glue as T
from test_gpu_attention import dev, same_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stream", ["f16", "f32"])
def test_prompt_and_decode_steps(stream):
    print(f"case decoder pass, {stream} stream", flush=True)
    from test_gpu_parity import make_case
    D, heads, vocab, window, sinks, page, layers = 512, 4, 1003, 24, 3, 16, 2
    lay, Q, lam = make_case(5, 64, D, D, 300, O.MODE_HEADWISE)
    rng = np.random.default_rng(7)
    pack = lambda N, K, q=None: B.rosaq_pack_weights((rng.standard_normal((N, K)) * 0.05).astype(np.float16), q, lam if K == D else np.ones(K), 128, 4,
                                                     B.Q_NONE if q is None else B.Q_HEADWISE)
    qkv = [[pack(D, D, Q) for _ in range(3)] for _ in range(layers)]
    o = [pack(D, D, Q) for _ in range(layers)]
    ffn = [(pack(768, D), pack(768, D), pack(D, 768)) for _ in range(layers)]
    head = pack(vocab, D)
    weights = [dev((1 + 0.2 * rng.standard_normal(D)).astype(np.float16)) for _ in range(2 * layers + 1)]
    caches = [T.KvCache(heads, 128, 8, page, 8) for _ in range(layers)]
    rope = T.Rope(T.rope_table(256, 128))
    cos, sin = (rope.table[..., i].cpu().numpy() for i in range(2))
    pages = np.array([[4, 1, 5, 0, 7, 2, 6, 3]], np.int32)
    slot_of = lambda t: pages[0][t // page].astype(np.int64) * page + t % page
    seen_k, seen_v = ([np.zeros((0, D), np.float16)] * layers for _ in range(2))
    done = 0
    table = pages.copy()
    for rows in (50, 1, 7, 1, 1):
        r = dev(rng.standard_normal((rows, D)).astype(np.float16 if stream == "f16" else np.float32))
        y = dev(np.zeros((rows, D), np.float16))

        def norm(y, n):
            before, added = r.cpu().numpy(), y.cpu().numpy()
            x = T.rmsnorm(y, weights[n], 1e-5, residual=r)
            assert np.array_equal(r.cpu().numpy(), (added.astype(np.float32) + before.astype(np.float32)).astype(before.dtype))
            want = R.rmsnorm(added, weights[n].cpu().numpy(), 1e-5, before)[1]
            assert np.all(np.abs(x.cpu().numpy().astype(np.float64) - want) <= R.rmsnorm_bound(want, D))
            return x

        at = np.arange(done, done + rows)
        lengths, starts = dev(np.array([done + rows], np.int32)), dev(np.array([0, rows], np.int32))
        # what no row will see any more is given back: its entries say so
        for p in range(pages.shape[1]):
            if p * page >= sinks and (p + 1) * page <= max(0, done - window + 1):
                table[0, p] = -1
        for l in range(layers):
            x = norm(y, 2 * l)
            q, k, v = T.linear_batch(qkv[l], x)
            turned = T.cache_append(caches[l], dev(slot_of(at)), k, v, rope=rope, positions=dev(at.astype(np.int32)), q=q)
            plan = T.AttentionPlan(caches[l], heads, 1, max_kv=128, max_rows=rows, window=window, sinks=sinks)
            att = T.attention(plan, turned, lengths, dev(table), row_start=starts)
            same_bits(turned, A.rope(q.cpu().numpy(), cos[at], sin[at], 128, "half"))
            seen_k[l] = np.concatenate([seen_k[l], A.rope(k.cpu().numpy(), cos[at], sin[at], 128, "half")])
            seen_v[l] = np.concatenate([seen_v[l], v.cpu().numpy()])
            j = np.arange(done + rows)[None]
            mask = (j <= at[:, None]) & ((j > at[:, None] - window) | (j < sinks))
            want, bound = A.attention(turned.cpu().numpy().reshape(rows, heads, 128), A.held(seen_k[l], heads, 8), A.held(seen_v[l], heads, 8), mask,
                                      128 ** -0.5)
            assert np.all(np.abs(att.cpu().numpy().reshape(want.shape).astype(np.float64) - want) <= bound)
            x = norm(T.linear(o[l], att), 2 * l + 1)
            gate, up, down = ffn[l]
            y = torch.empty((rows, D), dtype=torch.float16, device="cuda")
            ws = torch.empty(B.rosaq_workspace_bytes_mlp(gate, up, down, rows), dtype=torch.uint8, device="cuda")
            B.rosaq_mlp_swiglu(gate, up, down, x.data_ptr(), rows, x.stride(0), y.data_ptr(), y.stride(0), ws.data_ptr(), ws.numel(), T.current_stream_ptr())
        logits = T.linear(head, norm(y, 2 * layers))
        tokens = torch.randint(0, vocab, (rows,), device="cuda")
        got = T.logprobs(logits, tokens, top=5)
        log_p, H, ids, bound, bound_h = R.logprobs(logits.float().cpu().numpy(), 1.0, 5)
        t = tokens.cpu().numpy()[:, None]
        assert np.array_equal(got.top_ids.cpu().numpy(), ids) and np.all(np.abs(got.entropy.cpu().numpy() - H) <= bound_h)
        assert np.all(np.abs(got.given.cpu().numpy() - np.take_along_axis(log_p, t, 1)) <= np.take_along_axis(bound, t, 1))
        assert np.all(np.abs(got.top.cpu().numpy() - np.take_along_axis(log_p, ids, 1)) <= np.take_along_axis(bound, ids, 1))
        done += rows
    assert (table == -1).any()
