"""What a decoder's pass needs around its projections, as cases that can be timed and compared: the norm in front of them, attention
that looks back a window, and the log probabilities behind the head projection.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes what a user's program holds
before the call (inputs, page tables, a filled cache, output buffers, workspaces), `run()` makes one pass,
`work()` says what a pass cannot do without, `exact()` computes the same in 64 bits.  With `own` false `run()` computes
the operators from elementary torch operations, with `own` true it calls this library.

Kinds of case:
  norm      rows are added to the residual stream where there is one, and their norm is taken; to fp16, or to 8-bit codes with a scale a row
  window    rows of several sequences attend over their pages of the quantised cache: to the last `window` tokens and the first `sinks`
  logprobs  rows of logits: log probabilities of given tokens, the entropy, the largest alternatives

What the operators compute:
  norm      h = x + residual in fp32, kept rounded to the residual's type; y = h / sqrt(mean(h^2) + eps) * weight from the unrounded h;
            8 bits: scale = fp32(max |y| / 127), code = rne(y / scale), value code * scale, all before the value in 64 bits: a code next
            to a border is as far off as its step when it falls to the other side
  window    row i of a sequence of n rows and l cached tokens is at p = l - n + i and sees token j <= p if j > p - window or j < sinks;
            y = softmax(q k^T / sqrt(dim)) v over them, zero where there are none; keys and values are what the cache's codes stand for:
            lo = min(0, min x), hi = max(0, max x), top = 2^bits - 1, s = fp16(max((hi - lo) / top, 2^-14)), z = rne(-lo / s) in [0, top],
            t = floor(65504 / s), code = clamp(rne(x / s) + z, max(0, z - t), min(top, z + t)), value (code - z) s
  logprobs  log p_v = a x_v - log sum_w exp(a x_w); the entropy -sum p log p, where p = 0 adds nothing; the `top` largest logits, the
            lower index first where they are equal; a given token below zero is padding and gets 0
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One decode step at the benchmark's batch of 64, 7B-shaped, in front of the q/k/v or gate/up projections: latency counts.
        {"name": "norm_decode_m64", "kind": "norm", "m": 64, "dim": 4096, "residual": "f16", "codes": False},
        # A prompt's tokens, 13B-shaped, an odd number of them, behind a stream of 32 bits, for a product in 8 bits.
        {"name": "norm_codes_13b", "kind": "norm", "m": 1003, "dim": 5120, "residual": "f32", "codes": True},
        # Queries' heads, each a row of its own and no residual: many short rows.
        {"name": "norm_heads_2047x32", "kind": "norm", "m": 65504, "dim": 128, "residual": "", "codes": False},
        # Prompts of four users, 7B-shaped: bound by memory.
        {"name": "norm_prompt_7b", "kind": "norm", "m": 8192, "dim": 4096, "residual": "f16", "codes": False},
        # A batch of 64 chats of up to 4096 tokens, 7B-shaped, one token each.
        {"name": "window_decode_7b_m64_int4", "kind": "window", "seqs": 64, "rows": 1, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 4, "page": 64, "low": 1000, "high": 4096, "window": 1024, "sinks": 4},
        # Long chats with grouped heads.
        {"name": "window_decode_gqa_long_int4", "kind": "window", "seqs": 16, "rows": 1, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "bits": 4, "page": 64, "low": 8192, "high": 32768, "window": 4096, "sinks": 4},
        # One user far into one document: all of the card has to share one sequence.
        {"name": "window_decode_one_int8", "kind": "window", "seqs": 1, "rows": 1, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 8, "page": 128, "low": 65537, "high": 65537, "window": 8191, "sinks": 64},
        # Prompts of four users, every token behind a short window: bound by arithmetic.
        {"name": "window_prompt_7b_int8", "kind": "window", "seqs": 4, "rows": 2048, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 8, "page": 64, "low": 2048, "high": 2048, "window": 512, "sinks": 4},
        # A chunk of a long prompt behind what is cached of it, grouped heads, a window that ends inside pages.
        {"name": "window_chunk_gqa_int4", "kind": "window", "seqs": 3, "rows": 509, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "bits": 4, "page": 32, "low": 4096, "high": 8192, "window": 1000, "sinks": 5},
        # One decode step at batch 64: the chosen token's log probability and five alternatives.
        {"name": "logprobs_decode_m64", "kind": "logprobs", "m": 64, "vocab": 32000, "type": "f16", "given": 1, "top": 5, "masked": 0.0,
         "a": 1.0},
        # A text's perplexity: every token's log probability and the entropy.
        {"name": "logprobs_text_4095", "kind": "logprobs", "m": 4095, "vocab": 32000, "type": "f16", "given": 1, "top": 0, "masked": 0.0,
         "a": 1.0},
        # Answers compared under a grammar that forbids half of a large vocabulary, an odd one, with a temperature; an unquantised head.
        {"name": "logprobs_masked_f32", "kind": "logprobs", "m": 257, "vocab": 131071, "type": "f32", "given": 4, "top": 20, "masked": 0.5,
         "a": 1.25},
    ]


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], spread over the logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _fits(case):
    """No dearer than the dearest listed case of its kind."""
    most = [work(c) for c in listed() if c["kind"] == case["kind"]]
    w = work(case)
    return all(w[k] <= max(x[k] for x in most) for k in ("bytes", "flops"))


def draw(rng):
    while True:
        kind = rng.choice(("norm", "window", "window", "logprobs"))
        if kind == "norm":
            case = {"kind": kind, "m": _log_int(rng, 1, 65536), "dim": 8 * _log_int(rng, 8, 2048), "residual": rng.choice(("", "f16", "f16", "f32")),
                    "codes": rng.random() < 0.25}
        elif kind == "window":
            kv = _log_int(rng, 1, 40)
            rows = rng.choice((1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 2048)))
            high = _log_int(rng, rows, 65536)
            low = max(rows, int(high * rng.choice((1.0, 0.5, 0.1, 0.0))))
            case = {"kind": kind, "seqs": _log_int(rng, 1, 128), "rows": rows, "q_heads": kv * rng.choice((1, 1, 2, 4, 5, 7, 8)), "kv_heads": kv,
                    "dim": rng.choice((128, 128, 64)), "bits": rng.choice((4, 8)), "page": rng.choice((16, 32, 64, 128)), "low": low,
                    "high": high, "window": _log_int(rng, 1, 16384), "sinks": rng.choice((0, 1, 4, 4, _log_int(rng, 5, 300)))}
        else:
            case = {"kind": kind, "m": _log_int(rng, 1, 4096), "vocab": _log_int(rng, 1000, 262144), "type": rng.choice(("f16", "f16", "bf16", "f32")),
                    "given": rng.choice((0, 1, 1, 4)), "top": rng.choice((0, 1, 5, 20, 64)), "masked": rng.choice((0.0, 0.0, 0.5, 0.999)),
                    "a": rng.choice((1.0, 1.0, 0.7, 1.25))}
        if _fits(case) and _tokens(case) <= 1 << 21:
            return case


# ---- inputs -------------------------------------------------------------------------------------

def _lengths(case):
    """Cached tokens of every sequence: a matter of the case, not of the seed."""
    rng = random.Random("%d %d %d" % (case["low"], case["high"], case["seqs"]))
    return [rng.randint(case["low"], case["high"]) for _ in range(case["seqs"])]


def _tokens(case):
    """Tokens x heads that a case's cache holds, seen or not."""
    return sum(_lengths(case)) * case["kv_heads"] * case["dim"] // 128 if case["kind"] == "window" else 0


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _heads(g, m, heads, dim, spread=0.0):
    """fp16 [m, heads * dim]: normal, with channel scales of a log-normal spread."""
    sigma = torch.exp(spread * torch.randn(heads * dim, generator=g, device="cuda"))
    return (torch.randn((m, heads * dim), generator=g, device="cuda") * sigma).to(torch.float16)


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "norm":
        m, dim = case["m"], case["dim"]
        # what a projection adds, the stream with some channels of large values, weights around one
        d = {"x": _heads(g, m, 1, dim), "weight": (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(torch.float16), "eps": 1e-5}
        if case["residual"]:
            sigma = torch.exp(torch.randn(dim, generator=g, device="cuda"))
            d["residual"] = (torch.randn((m, dim), generator=g, device="cuda") * sigma).to(TYPES[case["residual"]])
        return d
    if case["kind"] == "logprobs":
        m, vocab = case["m"], case["vocab"]
        # a bias of every token, the row's own part, and a few tokens that stand out
        x = torch.randn((m, vocab), generator=g, device="cuda") * 1.5 + 2.0 * torch.randn(vocab, generator=g, device="cuda")
        ahead = torch.randint(0, vocab, (m, 8), generator=g, device="cuda")
        x.scatter_add_(1, ahead, 4.0 + 4.0 * torch.rand((m, 8), generator=g, device="cuda"))
        if case["masked"]:
            x.masked_fill_(torch.rand(vocab, generator=g, device="cuda") < case["masked"], -math.inf)
            x[:, vocab // 2] = 1.0                   # some token is always allowed
        d = {"x": x.to(TYPES[case["type"]])}
        if case["given"]:
            tokens = torch.randint(0, vocab, (m, case["given"]), generator=g, device="cuda")
            tokens[:, 0] = ahead[:, 0]
            padding = torch.rand(m, generator=g, device="cuda") < 0.05
            tokens[padding] = -100
            d["tokens"] = tokens
        return d
    lens, page = _lengths(case), case["page"]
    own_pages = [(n + page - 1) // page for n in lens]
    total = sum(own_pages)
    shuffled = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((case["seqs"], max(own_pages)), -1, dtype=torch.int32, device="cuda")
    offset = torch.arange(page, device="cuda")
    slots, at = [], 0
    for i, n in enumerate(own_pages):
        table[i, :n] = shuffled[at:at + n]
        at += n
        slots.append((table[i, :n].to(torch.int64)[:, None] * page + offset).reshape(-1)[:lens[i]])
    tokens = sum(lens)
    # the spread of the keys' channels gives scores of a few units
    return {"k": _heads(g, tokens, case["kv_heads"], case["dim"], 0.5), "v": _heads(g, tokens, case["kv_heads"], case["dim"]),
            "q": _heads(g, case["seqs"] * case["rows"], case["q_heads"], case["dim"]), "slots": torch.cat(slots),
            "table": table, "pages": total, "lens": lens, "kv_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
            "row_start": torch.arange(case["seqs"] + 1, dtype=torch.int32, device="cuda") * case["rows"]}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "norm":
        if own:
            s["sum"] = torch.empty_like(s["residual"]) if case["residual"] else None
            if case["codes"]:
                s["codes"] = torch.empty(s["x"].shape, dtype=torch.int8, device="cuda")
                s["scales"] = torch.empty(case["m"], dtype=torch.float32, device="cuda")
            else:
                s["y"] = torch.empty_like(s["x"])
    elif case["kind"] == "logprobs":
        if own:
            from paper_2506_13472_amd import torch_glue as T
            s["out"] = T.logprobs_buffers(s["x"], given=case["given"], top=case["top"])
    elif own:
        from paper_2506_13472_amd import torch_glue as T
        s["cache"] = T.KvCache(case["kv_heads"], case["dim"], case["bits"], case["page"], s["pages"])
        step = 65536
        for i in range(0, s["slots"].numel(), step):
            T.cache_append(s["cache"], s["slots"][i:i + step], s["k"][i:i + step], s["v"][i:i + step])
        s["y"] = torch.empty_like(s["q"])
        s["plan"] = T.AttentionPlan(s["cache"], q_heads=case["q_heads"], sequences=case["seqs"], max_kv=case["high"],
                                    max_rows=case["rows"], window=case["window"], sinks=case["sinks"])
        del s["k"], s["v"]
    else:
        s["kq"] = _quantise(s["k"], case["kv_heads"], case["dim"], case["bits"])
        s["vq"] = _quantise(s["v"], case["kv_heads"], case["dim"], case["bits"])
        del s["k"], s["v"]
    return s


# ---- one pass -----------------------------------------------------------------------------------

def _quantise(x, heads, dim, bits):
    """codes uint8 [m, heads, dim], scales and zeros fp32 [m, heads, 1]."""
    codes, scales, zeros = [], [], []
    top = float(2 ** bits - 1)
    for part in x.split(65536):
        part = part.view(part.shape[0], heads, dim).float()
        lo = part.amin(dim=-1, keepdim=True).clamp(max=0.0)
        hi = part.amax(dim=-1, keepdim=True).clamp(min=0.0)
        s = ((hi - lo) / top).clamp(min=2.0 ** -14).to(torch.float16).float()
        z = torch.round(-lo / s).clamp(0.0, top)
        t = torch.floor(65504.0 / s)
        code = torch.round(part / s) + z
        code = torch.minimum(torch.maximum(code, (z - t).clamp(min=0.0)), (z + t).clamp(max=top))
        codes.append(code.to(torch.uint8))
        scales.append(s)
        zeros.append(z)
    return torch.cat(codes), torch.cat(scales), torch.cat(zeros)


def _plain_norm(s):
    case = s["case"]
    wide = torch.float64 if case["codes"] else torch.float32
    h = s["x"].to(wide)
    out = []
    if case["residual"]:
        h = h + s["residual"].to(wide)
        out.append(h.to(TYPES[case["residual"]]))
    y = h / torch.sqrt((h * h).mean(dim=-1, keepdim=True) + s["eps"]) * s["weight"].to(wide)
    if case["codes"]:
        scale = (y.abs().amax(dim=-1, keepdim=True) / 127.0).float()
        return out + [torch.round(y / scale.double()).float() * scale, scale[:, 0]]
    return out + [y.to(torch.float16)]


def _order(x):
    """int64 keys that are ordered as the logits are, of equal ones the lower index first."""
    bits = (x.float() + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    return bits * (1 << 20) - torch.arange(x.shape[1], device=x.device)


def _plain_logprobs(s):
    case, a = s["case"], s["case"]["a"]
    x = s["x"]
    out = {"given": None, "entropy": torch.empty(x.shape[0], device="cuda"), "top_ids": None, "top": None}
    log_p = torch.empty(x.shape, dtype=torch.float32, device="cuda")
    for i in range(0, x.shape[0], 1024):
        z = x[i:i + 1024].float() * a
        z = z - z.amax(dim=-1, keepdim=True)
        log_p[i:i + 1024] = z - torch.log(torch.exp(z).sum(dim=-1, keepdim=True))
        lp = log_p[i:i + 1024]
        p = torch.exp(lp)
        out["entropy"][i:i + 1024] = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(dim=-1)
    if case["given"]:
        t = s["tokens"]
        out["given"] = torch.where(t >= 0, log_p.gather(1, t.clamp(min=0)), torch.zeros_like(t, dtype=torch.float32))
    if case["top"]:
        keys, ids = _order(x), []
        for _ in range(case["top"]):
            best = keys.amax(dim=-1, keepdim=True)
            ids.append((-best) & ((1 << 20) - 1))
            keys.scatter_(1, ids[-1], -(1 << 62))
        out["top_ids"] = torch.cat(ids, dim=1)
        out["top"] = log_p.gather(1, out["top_ids"])
    return [out[k] for k in ("given", "entropy", "top_ids", "top") if out[k] is not None]


def _plain_window(s):
    case = s["case"]
    kv, group, rows, dim = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["rows"], case["dim"]
    window, sinks = case["window"], case["sinks"]
    q = s["q"].float().view(case["seqs"], rows, kv, group, dim)
    y = torch.empty_like(q)
    at = 0
    for i, n in enumerate(s["lens"]):
        # tokens that some row sees: the first few, and those from the first row's window on
        start = max(0, n - rows - window + 1)
        first = min(sinks, start)
        where = torch.cat((torch.arange(first, device="cuda"), torch.arange(start, n, device="cuda")))
        k, v = (((c[where + at].float() - z[where + at]) * sc[where + at]) for c, sc, z in (s["kq"], s["vq"]))
        kt = k.permute(1, 2, 0).contiguous()                          # [kv, dim, tokens]
        vt = v.permute(1, 0, 2).contiguous()
        step = max(1, (1 << 28) // (kv * group * where.numel()))
        for r0 in range(0, rows, step):
            part = q[i, r0:r0 + step]
            m = part.shape[0]
            score = torch.matmul(part.permute(1, 0, 2, 3).reshape(kv, m * group, dim), kt) * (1.0 / math.sqrt(dim))
            score = score.view(kv, m, group, -1)
            p = torch.arange(n - rows + r0, n - rows + r0 + m, device="cuda")[:, None]
            seen = (where <= p) & ((where > p - window) | (where < sinks))
            score = score.masked_fill(~seen[None, :, None, :], -math.inf)
            w = torch.exp(score - score.amax(dim=-1, keepdim=True))
            w = w / w.sum(dim=-1, keepdim=True)
            y[i, r0:r0 + step] = torch.matmul(w.view(kv, m * group, -1), vt).view(kv, m, group, dim).permute(1, 0, 2, 3)
        at += n
    return y.view(case["seqs"] * rows, -1).to(torch.float16)


def run(s):
    case = s["case"]
    if not own:
        return {"norm": _plain_norm, "logprobs": _plain_logprobs, "window": _plain_window}[case["kind"]](s)
    from paper_2506_13472_amd import torch_glue as T
    if case["kind"] == "norm":
        kept = [s["sum"]] if case["residual"] else []
        if case["codes"]:
            T.rmsnorm_codes(s["x"], s["weight"], s["eps"], residual=s.get("residual"), residual_out=s["sum"], codes=s["codes"], scales=s["scales"])
            return kept + [s["codes"] * s["scales"][:, None], s["scales"]]
        T.rmsnorm(s["x"], s["weight"], s["eps"], residual=s.get("residual"), residual_out=s["sum"], out=s["y"])
        return kept + [s["y"]]
    if case["kind"] == "logprobs":
        out = T.logprobs(s["x"], tokens=s.get("tokens"), top=case["top"], scale=case["a"], out=s["out"])
        return [t for t in out if t is not None]
    return T.attention(s["plan"], s["q"], s["kv_len"], s["table"], row_start=s["row_start"] if case["rows"] > 1 else None, out=s["y"])


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    if case["kind"] == "norm":
        n = case["m"] * case["dim"]
        stream = {"": 0, "f16": 4, "f32": 8}[case["residual"]]               # read and written
        return {"bytes": n * (2 + stream + (1 if case["codes"] else 2)) + 2 * case["dim"] + (4 * case["m"] if case["codes"] else 0),
                "flops": n * (4 + (1 if case["residual"] else 0) + (3 if case["codes"] else 0))}
    if case["kind"] == "logprobs":
        n = case["m"] * case["vocab"]
        return {"bytes": n * (4 if case["type"] == "f32" else 2) + case["m"] * (4 + 12 * case["given"] + 12 * case["top"]), "flops": 6 * n}
    token = 2 * case["kv_heads"] * (case["dim"] * case["bits"] // 8 + 4)      # codes, scale and zero of k and v
    rows, window, sinks = case["rows"], case["window"], case["sinks"]
    held, pairs = 0, 0
    for n in _lengths(case):
        start = max(0, n - rows - window + 1)
        held += n - start + min(sinks, start)
        for p in range(n - rows, n):
            lo = max(0, p - window + 1)
            pairs += p + 1 - lo + min(sinks, lo)
    return {"bytes": held * token + 4 * case["seqs"] * rows * case["q_heads"] * case["dim"], "flops": 4 * case["q_heads"] * case["dim"] * pairs}


# ---- the definition in 64 bits ------------------------------------------------------------------

def _held(x, bits):
    """The values that the codes of fp64 x [m, dim] stand for."""
    top = 2 ** bits - 1
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    lo, hi = torch.minimum(x.min(-1, True).values, zero), torch.maximum(x.max(-1, True).values, zero)
    s = torch.maximum((hi - lo).float().double() / top, zero + 2.0 ** -14).float().half().double()
    z = torch.round(-lo / s)
    z = torch.where(z > top, zero + top, z)
    far = torch.floor(65504 / s)
    low, high = torch.maximum(zero - z, -far), torch.minimum(top - z, far)
    return torch.maximum(low, torch.minimum(high, torch.round(x / s))) * s


def _exact_norm(s, case):
    h = s["x"].double()
    out = []
    if case["residual"]:
        h += s["residual"].double()
        out.append(h.clone())
    h *= torch.rsqrt(h.square().sum(1) / case["dim"] + s["eps"])[:, None]
    h *= s["weight"].double()
    if case["codes"]:
        step = (torch.maximum(h.max(1).values, -h.min(1).values) / 127).float().double()
        return out + [torch.round(h / step[:, None]) * step[:, None], step]
    return out + [h]


def _exact_logprobs(s, case):
    given, entropy, ids, top = [], [], [], []
    for row in range(0, case["m"], 128):
        x = s["x"][row:row + 128].double()
        scaled = x * case["a"]
        total = torch.logsumexp(scaled, 1)
        share = torch.softmax(scaled, 1)
        entropy.append(total - torch.where(share > 0, share * scaled, share).sum(1))
        if case["given"]:
            t = s["tokens"][row:row + 128]
            given.append(torch.where(t < 0, 0.0, torch.take_along_dim(scaled, t.clamp(0), 1) - total[:, None]))
        if case["top"]:
            best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            ids.append(best)
            top.append(torch.take_along_dim(scaled, best, 1) - total[:, None])
    return [torch.cat(t) for t in (given, entropy, ids, top) if t]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s, case)
    if case["kind"] == "logprobs":
        return _exact_logprobs(s, case)
    kv, dim, bits, rows, group = case["kv_heads"], case["dim"], case["bits"], case["rows"], case["q_heads"] // case["kv_heads"]
    q = s["q"].double().view(case["seqs"], rows, kv, group, dim)
    y = torch.zeros_like(q)
    for h in range(kv):
        k, v = (s[name][:, h * dim:(h + 1) * dim].double() for name in ("k", "v"))
        k, v = _held(k, bits), _held(v, bits)
        at = 0
        for i, n in enumerate(s["lens"]):
            behind = torch.arange(rows, device="cuda")[:, None] + (n - rows) - torch.arange(n, device="cuda")      # tokens back
            hidden = (behind < 0) | ((behind >= case["window"]) & (torch.arange(n, device="cuda") >= case["sinks"]))
            for g in range(group):
                e = (q[i, :, h, g] @ k[at:at + n].t()) / dim ** 0.5
                e[hidden] = -math.inf
                w = torch.exp(e - e.max(1).values[:, None])
                y[i, :, h, g] = w @ v[at:at + n] / w.sum(1)[:, None]
            at += n
    return y.view(case["seqs"] * rows, -1)
