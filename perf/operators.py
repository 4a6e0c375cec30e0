"""The attention between the q/k/v projections and the output projection, as cases that can be timed and compared.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes what a user's program holds
before the call (inputs, page tables, a filled cache, a table of angles, workspaces), `run()` makes one pass,
`work()` says what a pass cannot do without, `exact()` computes the same in 64 bits.  With `own` false `run()` computes
the operators from elementary torch operations, with `own` true it calls this library.

Kinds of case:
  rope       rotary positions of one tensor of heads
  cache      new tokens are rotated, quantised and written to the cache, and their values read back
  attention  rows of several sequences over their pages of the cache, behind a prefix that all of them share
             where `prefix` is not zero

What the operators compute:
  rope       of pair (a, b) at position p: a cos - b sin, b cos + a sin, with cos and sin in fp32 from a table, products and
             sums in 64 bits, rounded to fp32 and from there to fp16
  quantiser  of the `dim` channels x of a token's head: lo = min(0, min x), hi = max(0, max x), top = 2^bits - 1,
             s = fp16(max((hi - lo) / top, 2^-14)), z = rne(-lo / s) in [0, top], t = floor(65504 / s),
             code = clamp(rne(x / s) + z, max(0, z - t), min(top, z + t)), value (code - z) s; differences and quotients in fp32
  attention  row i of a sequence of n rows and l cached tokens sees the prefix and the tokens below l - n + i + 1;
             y = softmax(scale q k^T) v over them, zero where there are none
"""
from __future__ import annotations

import math
import random

import torch

own = False


def listed():
    return [
        # One decode step's queries at the benchmark's batch of 64, 7B-shaped: the smallest call, latency counts.
        {"name": "rope_decode_m64", "kind": "rope", "m": 64, "heads": 32, "dim": 128, "rot": 128,
         "layout": "half", "positions": 4096},
        # A long prompt's queries, 13B-shaped, with half of every head rotated in interleaved pairs, far positions.
        {"name": "rope_prompt_13b", "kind": "rope", "m": 8191, "heads": 40, "dim": 128, "rot": 64,
         "layout": "interleaved", "positions": 131072},
        # One decode step at batch 64, 7B-shaped, four-bit codes: one new token of every sequence.
        {"name": "cache_decode_m64_int4", "kind": "cache", "m": 64, "q_heads": 32, "kv_heads": 32, "dim": 128, "bits": 4,
         "page": 64, "rot": 128, "layout": "half", "positions": 4096},
        # Some prompts' tokens with shared heads of 64 channels, kept as they are (no rotation), an odd number of them.
        {"name": "cache_ragged_gqa_int4", "kind": "cache", "m": 1003, "q_heads": 0, "kv_heads": 8, "dim": 64, "bits": 4,
         "page": 16, "rot": 0, "layout": "half", "positions": 4096},
        # A prompt of 4096 tokens, 13B-shaped, eight-bit codes.
        {"name": "cache_prompt_13b_int8", "kind": "cache", "m": 4096, "q_heads": 40, "kv_heads": 40, "dim": 128, "bits": 8,
         "page": 64, "rot": 128, "layout": "half", "positions": 8192},
        # The decode throughput setting of the paper: 64 sequences, 128 tokens of context and up to 128 generated.
        {"name": "decode_7b_m64_int4", "kind": "attention", "seqs": 64, "rows": 1, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 4, "page": 64, "low": 129, "high": 256, "prefix": 0},
        # Long chats with grouped heads: every step reads the whole cache.
        {"name": "decode_gqa_long_int4", "kind": "attention", "seqs": 16, "rows": 1, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "bits": 4, "page": 64, "low": 8192, "high": 32768, "prefix": 0},
        # One user with one long document: all of the card has to share one sequence.
        {"name": "decode_one_long_int8", "kind": "attention", "seqs": 1, "rows": 1, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 8, "page": 128, "low": 65537, "high": 65537, "prefix": 0},
        # Prompts of four users: bound by arithmetic.
        {"name": "prompt_7b_int8", "kind": "attention", "seqs": 4, "rows": 2048, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 8, "page": 64, "low": 2048, "high": 2048, "prefix": 0},
        # A chunk of a long prompt behind what is cached of it, grouped heads.
        {"name": "chunk_gqa_int4", "kind": "attention", "seqs": 3, "rows": 509, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "bits": 4, "page": 32, "low": 4096, "high": 8192, "prefix": 0},
        # A batch of 64 behind one system prompt, 7B-shaped.
        {"name": "prefix_7b_m64_int4", "kind": "attention", "seqs": 64, "rows": 1, "q_heads": 32, "kv_heads": 32, "dim": 128,
         "bits": 4, "page": 64, "low": 1, "high": 256, "prefix": 2051},
        # Many questions about one long document, a few rows each (drafted tokens), grouped heads.
        {"name": "prefix_gqa_long_int8", "kind": "attention", "seqs": 32, "rows": 3, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "bits": 8, "page": 64, "low": 3, "high": 512, "prefix": 16389},
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
        kind = rng.choice(("rope", "cache", "attention", "attention", "attention"))
        dim = rng.choice((128, 128, 64))
        if kind == "rope":
            case = {"kind": kind, "m": _log_int(rng, 1, 16384), "heads": rng.randint(1, 64), "dim": dim,
                    "rot": rng.choice((dim, dim, dim // 2, dim // 4)), "layout": rng.choice(("half", "interleaved")),
                    "positions": _log_int(rng, 16, 131072)}
        elif kind == "cache":
            kv = _log_int(rng, 1, 40)
            rot = rng.choice((0, dim, dim, dim // 2))
            case = {"kind": kind, "m": _log_int(rng, 1, 8192), "q_heads": kv * rng.choice((1, 1, 2, 4, 5)) if rot else 0,
                    "kv_heads": kv, "dim": dim, "bits": rng.choice((4, 8)), "page": rng.choice((16, 32, 64, 128)), "rot": rot,
                    "layout": rng.choice(("half", "interleaved")), "positions": _log_int(rng, 16, 131072)}
        else:
            kv = _log_int(rng, 1, 40)
            group = rng.choice((1, 1, 2, 4, 5, 7, 8))
            rows = rng.choice((1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 2048)))
            high = _log_int(rng, rows, 65536)
            low = max(rows, int(high * rng.choice((1.0, 0.5, 0.1, 0.0))))
            case = {"kind": kind, "seqs": _log_int(rng, 1, 128), "rows": rows, "q_heads": kv * group, "kv_heads": kv, "dim": dim,
                    "bits": rng.choice((4, 8)), "page": rng.choice((16, 32, 64, 128)), "low": low, "high": high,
                    "prefix": rng.choice((0, 0, _log_int(rng, 1, 16384)))}
        if _fits(case):
            return case


# ---- inputs -------------------------------------------------------------------------------------

def _lengths(case):
    """Cached tokens of every sequence: a matter of the case, not of the seed."""
    rng = random.Random("%d %d %d" % (case["low"], case["high"], case["seqs"]))
    return [rng.randint(case["low"], case["high"]) for _ in range(case["seqs"])]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _heads(g, m, heads, dim, spread=0.0):
    """fp16 [m, heads * dim]: normal, with channel scales of a log-normal spread."""
    sigma = torch.exp(spread * torch.randn(heads * dim, generator=g, device="cuda"))
    return (torch.randn((m, heads * dim), generator=g, device="cuda") * sigma).to(torch.float16)


def _table(positions, rot):
    """cos and sin of position * 10000^(-2 i / rot), fp32 [positions, rot / 2, 2]."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack((torch.cos(angle), torch.sin(angle)), dim=-1).to(torch.float32)


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] == "rope":
        return {"x": _heads(g, case["m"], case["heads"], case["dim"]), "table": _table(case["positions"], case["rot"]),
                "at": torch.randint(0, case["positions"], (case["m"],), generator=g, device="cuda", dtype=torch.int32)}
    if case["kind"] == "cache":
        m, kv = case["m"], case["kv_heads"]
        pages = (m + 64 + case["page"] - 1) // case["page"]
        # slots as a serving loop hands them out: anywhere in the pool, every one once
        slots = torch.randperm(pages * case["page"], generator=g, device="cuda")[:m] if m < 512 else \
            (torch.randperm(pages, generator=g, device="cuda")[:, None] * case["page"]
             + torch.arange(case["page"], device="cuda")).reshape(-1)[:m]
        d = {"k": _heads(g, m, kv, case["dim"], 0.5), "v": _heads(g, m, kv, case["dim"]), "slots": slots.to(torch.int64).contiguous(),
             "pages": pages}
        if case["rot"]:
            d["q"] = _heads(g, m, case["q_heads"], case["dim"])
            d["table"] = _table(case["positions"], case["rot"])
            d["at"] = torch.randint(0, case["positions"], (m,), generator=g, device="cuda", dtype=torch.int32)
        return d
    lens, page, prefix = _lengths(case), case["page"], case["prefix"]
    own_pages = [(n + page - 1) // page for n in lens]
    prefix_pages = (prefix + page - 1) // page
    total = sum(own_pages) + prefix_pages
    shuffled = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((case["seqs"], max(own_pages)), -1, dtype=torch.int32, device="cuda")
    starts, at = [], prefix_pages
    for i, n in enumerate(own_pages):
        table[i, :n] = shuffled[at:at + n]
        at += n
    offset = torch.arange(page, device="cuda")

    def slots(of, n):
        return (of.to(torch.int64)[:, None] * page + offset).reshape(-1)[:n]

    parts = [slots(shuffled[:prefix_pages], prefix)] + [slots(table[i, :own_pages[i]], n) for i, n in enumerate(lens)]
    for p in parts:
        starts.append(p.numel())
    tokens = sum(starts)
    # the spread of the keys' channels and a query of 1.5 / sqrt(mean square) give scores of a few units
    return {"k": _heads(g, tokens, case["kv_heads"], case["dim"], 0.5), "v": _heads(g, tokens, case["kv_heads"], case["dim"]),
            "q": _heads(g, case["seqs"] * case["rows"], case["q_heads"], case["dim"]), "slots": torch.cat(parts),
            "table": table, "prefix_table": shuffled[:prefix_pages].contiguous(), "pages": total, "lens": lens,
            "kv_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
            "row_start": torch.arange(case["seqs"] + 1, dtype=torch.int32, device="cuda") * case["rows"]}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "rope":
        if own:
            from paper_2506_13472_amd import torch_glue as T
            s["rope"] = T.Rope(s["table"], case["layout"])
            s["y"] = torch.empty_like(s["x"])
    elif case["kind"] == "cache":
        if own:
            from paper_2506_13472_amd import torch_glue as T
            s["cache"] = T.KvCache(case["kv_heads"], case["dim"], case["bits"], case["page"], s["pages"])
            s["rope"] = T.Rope(s["table"], case["layout"]) if case["rot"] else None
            s["q_out"] = torch.empty_like(s["q"]) if case["rot"] else None
            s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    else:
        if own:
            from paper_2506_13472_amd import torch_glue as T
            s["cache"] = T.KvCache(case["kv_heads"], case["dim"], case["bits"], case["page"], s["pages"])
            T.cache_append(s["cache"], s["slots"], s["k"], s["v"])
            s["y"] = torch.empty_like(s["q"])
            s["plan"] = T.AttentionPlan(
                s["cache"], q_heads=case["q_heads"], sequences=case["seqs"], max_kv=case["high"],
                max_rows=case["rows"], prefix_len=case["prefix"])
        else:
            s["kq"] = _quantise(s["k"], case["kv_heads"], case["dim"], case["bits"])
            s["vq"] = _quantise(s["v"], case["kv_heads"], case["dim"], case["bits"])
        del s["k"], s["v"]
    return s


# ---- one pass -----------------------------------------------------------------------------------

def _rotate(x, dim, rot, layout, table, at):
    x = x.view(x.shape[0], -1, dim)
    cs = table[at.long()].double()[:, None]                       # [m, 1, rot / 2, 2]
    c, s = cs[..., 0], cs[..., 1]
    r = x[..., :rot].double()
    if layout == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    return torch.cat((r.float().to(torch.float16), x[..., rot:]), dim=-1).flatten(1)


def _quantise(x, heads, dim, bits):
    """codes uint8 [m, heads, dim], scales and zeros fp32 [m, heads, 1]."""
    x = x.view(x.shape[0], heads, dim).float()
    top = float(2 ** bits - 1)
    lo = x.amin(dim=-1, keepdim=True).clamp(max=0.0)
    hi = x.amax(dim=-1, keepdim=True).clamp(min=0.0)
    s = ((hi - lo) / top).clamp(min=2.0 ** -14).to(torch.float16).float()
    z = torch.round(-lo / s).clamp(0.0, top)
    t = torch.floor(65504.0 / s)
    code = torch.round(x / s) + z
    code = torch.minimum(torch.maximum(code, (z - t).clamp(min=0.0)), (z + t).clamp(max=top))
    return code.to(torch.uint8), s, z


def _values(q):
    code, s, z = q
    return (code.float() - z) * s


def _attend(q, k, v, rows, group, causal_from):
    """fp32; q [rows, kv, group, dim], k and v [tokens, kv, dim]; row i sees the tokens below causal_from + i + 1."""
    kv, dim, tokens = k.shape[1], k.shape[2], k.shape[0]
    kt = k.permute(1, 2, 0).contiguous()                          # [kv, dim, tokens]
    vt = v.permute(1, 0, 2).contiguous()
    y = torch.empty_like(q)
    step = max(1, (1 << 28) // max(1, kv * group * tokens))
    for r0 in range(0, rows, step):
        part = q[r0:r0 + step]
        n = part.shape[0]
        score = torch.matmul(part.permute(1, 0, 2, 3).reshape(kv, n * group, dim), kt) * (1.0 / math.sqrt(dim))
        score = score.view(kv, n, group, tokens)
        if rows > 1:
            seen = torch.arange(tokens, device=q.device)[None, :] <= torch.arange(r0, r0 + n, device=q.device)[:, None] + causal_from
            score = score.masked_fill(~seen[None, :, None, :], -math.inf)
        p = torch.exp(score - score.amax(dim=-1, keepdim=True))
        p = p / p.sum(dim=-1, keepdim=True)
        y[r0:r0 + step] = torch.matmul(p.view(kv, n * group, tokens), vt).view(kv, n, group, dim).permute(1, 0, 2, 3)
    return y


def _plain(s):
    case = s["case"]
    if case["kind"] == "rope":
        return _rotate(s["x"], case["dim"], case["rot"], case["layout"], s["table"], s["at"])
    if case["kind"] == "cache":
        q, k = None, s["k"]
        if case["rot"]:
            q = _rotate(s["q"], case["dim"], case["rot"], case["layout"], s["table"], s["at"])
            k = _rotate(k, case["dim"], case["rot"], case["layout"], s["table"], s["at"])
        kq = _quantise(k, case["kv_heads"], case["dim"], case["bits"])
        vq = _quantise(s["v"], case["kv_heads"], case["dim"], case["bits"])
        return [q, _values(kq).to(torch.float16).flatten(1), _values(vq).to(torch.float16).flatten(1)]
    kv, group, rows, prefix = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["rows"], case["prefix"]
    k, v = _values(s["kq"]), _values(s["vq"])
    q = s["q"].float().view(case["seqs"], rows, kv, group, case["dim"])
    y = torch.empty_like(q)
    at = prefix
    for i, n in enumerate(s["lens"]):
        ks, vs = k[at:at + n], v[at:at + n]
        if prefix:
            ks, vs = torch.cat((k[:prefix], ks)), torch.cat((v[:prefix], vs))
        y[i] = _attend(q[i], ks, vs, rows, group, prefix + n - rows)
        at += n
    return y.view(case["seqs"] * rows, -1).to(torch.float16)


def run(s):
    if not own:
        return _plain(s)
    from paper_2506_13472_amd import torch_glue as T
    case = s["case"]
    if case["kind"] == "rope":
        return T.rope(s["rope"], s["x"], s["at"], case["dim"], out=s["y"])
    if case["kind"] == "cache":
        if case["rot"]:
            T.cache_append(s["cache"], s["slots"], s["k"], s["v"], rope=s["rope"], positions=s["at"], q=s["q"], q_out=s["q_out"])
        else:
            T.cache_append(s["cache"], s["slots"], s["k"], s["v"])
        T.cache_read(s["cache"], s["slots"], k=s["k_out"], v=s["v_out"])
        return [s["q_out"], s["k_out"], s["v_out"]]
    return T.attention(s["plan"], s["q"], s["kv_len"], s["table"], row_start=s["row_start"] if case["rows"] > 1 else None,
                       prefix_pages=s["prefix_table"] if case["prefix"] else None, out=s["y"])


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    if case["kind"] == "rope":
        n = case["m"] * case["heads"]
        table = min(case["m"], case["positions"]) * case["rot"] * 4
        return {"bytes": 4 * n * case["dim"] + table + 4 * case["m"], "flops": 3 * n * case["rot"]}
    token = 2 * case["kv_heads"] * (case["dim"] * case["bits"] // 8 + 4)      # codes, scale and zero of k and v
    if case["kind"] == "cache":
        m, kv, dim = case["m"], case["kv_heads"], case["dim"]
        rot = min(m, case["positions"]) * case["rot"] * 4 + 4 * m if case["rot"] else 0
        # read k and v, write the cache, read it, write their values; rotate q
        return {"bytes": 8 * m * kv * dim + 2 * m * token + 16 * m + 4 * m * case["q_heads"] * dim + rot,
                "flops": m * (3 * case["rot"] * (case["q_heads"] + kv) + 12 * kv * dim)}
    lens, rows, prefix = _lengths(case), case["rows"], case["prefix"]
    seen = sum(rows * (prefix + n) - rows * (rows - 1) // 2 for n in lens)
    return {"bytes": (sum(lens) + prefix) * token + 4 * case["seqs"] * rows * case["q_heads"] * case["dim"],
            "flops": 4 * case["q_heads"] * case["dim"] * seen}


# ---- the definition in 64 bits ------------------------------------------------------------------

def _turned(x, case, heads, table, at):
    """fp64 [m, heads, dim], unrounded: every pair as a complex number times cos + i sin."""
    rot, dim = case["rot"], case["dim"]
    x = x.double().reshape(-1, heads, dim).clone()
    half = rot // 2
    first = torch.arange(half, device="cuda") if case["layout"] == "half" else 2 * torch.arange(half, device="cuda")
    second = first + (half if case["layout"] == "half" else 1)
    turn = torch.view_as_complex(table.double()[at.long()])[:, None, :]
    pair = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = pair.real, pair.imag
    return x


def _held(x, bits):
    """The values that the codes of fp64 x [m, heads, dim] stand for."""
    top = 2 ** bits - 1
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    lo, hi = torch.minimum(x.min(-1, True).values, zero), torch.maximum(x.max(-1, True).values, zero)
    s = torch.maximum((hi - lo).float().double() / top, zero + 2.0 ** -14).float().half().double()
    z = torch.round(-lo / s)
    z = torch.where(z > top, zero + top, z)
    far = torch.floor(65504 / s)
    low, high = torch.maximum(zero - z, -far), torch.minimum(top - z, far)
    return torch.maximum(low, torch.minimum(high, torch.round(x / s))) * s


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rope":
        return _turned(s["x"], case, case["heads"], s["table"], s["at"]).flatten(1)
    kv, dim, bits = case["kv_heads"], case["dim"], case["bits"]
    if case["kind"] == "cache":
        q, k = None, s["k"].double().view(-1, kv, dim)
        if case["rot"]:
            q = _turned(s["q"], case, case["q_heads"], s["table"], s["at"]).flatten(1)
            k = _turned(s["k"], case, kv, s["table"], s["at"]).float().half().double()      # the cache is given fp16
        return [q, _held(k, bits).flatten(1), _held(s["v"].double().view(-1, kv, dim), bits).flatten(1)]
    rows, prefix, group = case["rows"], case["prefix"], case["q_heads"] // kv
    q = s["q"].double().view(case["seqs"], rows, kv, group, dim)
    y = torch.zeros_like(q)
    for h in range(kv):
        k = _held(s["k"][:, h * dim:(h + 1) * dim].double()[:, None], bits)[:, 0]
        v = _held(s["v"][:, h * dim:(h + 1) * dim].double()[:, None], bits)[:, 0]
        at = prefix
        for i, n in enumerate(s["lens"]):
            shared = [(k[:prefix], v[:prefix], None)] if prefix else []
            parts = shared + [(k[at:at + n], v[at:at + n], n - rows)]
            for g in range(group):
                e = [(q[i, :, h, g] @ a.t()) / dim ** 0.5 for a, _, _ in parts]
                hidden = torch.arange(n, device="cuda") > torch.arange(rows, device="cuda")[:, None] + (n - rows)
                e[-1][hidden] = -math.inf
                most = torch.stack([x.max(-1).values for x in e]).max(0).values[:, None]
                w = [torch.exp(x - most) for x in e]
                y[i, :, h, g] = sum(x @ b for x, (_, b, _) in zip(w, parts)) / sum(x.sum(-1, keepdim=True) for x in w)
            at += n
    return y.view(case["seqs"] * rows, -1)
