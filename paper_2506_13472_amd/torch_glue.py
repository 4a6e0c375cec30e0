"""PyTorch is used for device memory and streams only: allocate y and the
workspace, hand raw pointers and the current stream to the C ABI."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from . import binding as B


# The current stream's pointer alone takes 0.35 us, a Stream object made for it 2.7: a fifth of what issuing a small call
# costs (one of four rows of a 1024 x 1024 layer: some 11 us with it).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def current_stream_ptr() -> int:
    if _raw_stream is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def alloc_workspace(p: B.Packed, M: int) -> torch.Tensor:
    n = B.rosaq_workspace_bytes(p, M)
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def linear(p: B.Packed, x: torch.Tensor, y: torch.Tensor | None = None,
           ws: torch.Tensor | None = None) -> torch.Tensor:
    """y = rosaq_linear*(p, x) on the current stream.  x: fp16 [M, D] on the GPU
    (row stride may exceed D)."""
    if not x.is_cuda or x.dtype != torch.float16 or x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be a 2-D fp16 CUDA tensor with unit column stride")
    M = x.shape[0]
    if y is None:
        y = torch.empty((M, p.N), dtype=torch.float16, device=x.device)
    if ws is None:
        ws = alloc_workspace(p, M)
    fn = B.rosaq_linear_headwise if p.q_mode == B.Q_HEADWISE else B.rosaq_linear
    fn(p, x.data_ptr(), M, x.stride(0), y.data_ptr(), y.stride(0), ws.data_ptr(), ws.numel(),
       current_stream_ptr())
    return y


def linear_batch(layers, x: torch.Tensor, ys=None, ws: torch.Tensor | None = None):
    """[y_i] = rosaq_linear_batch(layers, x): layers share x and the rotation."""
    M = x.shape[0]
    if ys is None:
        ys = [torch.empty((M, p.N), dtype=torch.float16, device=x.device) for p in layers]
    if ws is None:
        ws = alloc_workspace(layers[0], M)
    args = B.BatchArgs(layers, [y.data_ptr() for y in ys], [y.stride(0) for y in ys])
    B.rosaq_linear_batch(args, x.data_ptr(), M, x.stride(0), ws.data_ptr(), ws.numel(),
                         current_stream_ptr())
    return ys


# ---- the attention between the q/k/v projections and the output projection -----------------------------------------
#
# A launch of a few rows runs 3 to 5 us and takes as long to issue, so the checks are kept to what costs little: those of one call
# take about 1.5 us.

_HALF, _INT32, _INT64 = torch.float16, torch.int32, torch.int64
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _ld(name: str, x: torch.Tensor, rows: int, width: int) -> int:
    """The row stride of an fp16 matrix [rows, width]; of a single row, whose stride torch leaves open, its width."""
    stride = x.stride()
    if x.dtype is not _HALF or x.shape != (rows, width) or stride[1] != 1:
        raise ValueError(f"{name} must be an fp16 tensor [{rows}, {width}] with unit column stride")
    return stride[0] if rows > 1 else width


def _integers(name: str, t: torch.Tensor, dtype: torch.dtype, count: int) -> int:
    """The address of a contiguous integer tensor of `count` elements (of any number: -1)."""
    if t.dtype is not dtype or (t.numel() != count and count >= 0) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor" + (f" of {count} elements" if count >= 0 else ""))
    return t.data_ptr()


def _device_of(*tensors) -> int:
    """The GPU that all of a call's tensors (those that are not None) lie on."""
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("the tensors of a call must lie on one GPU")
    if index < 0:
        raise ValueError("the tensors of a call must lie on a GPU")
    return index


def _stream_on(index: int) -> int:
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream


class Rope:
    """A table of angles (fp32 [positions, rot_dim / 2, 2]: cos, sin) and how heads are paired."""

    LAYOUTS = {"half": B.ROPE_HALF, "interleaved": B.ROPE_INTERLEAVED}

    def __init__(self, table: torch.Tensor, layout: str = "half"):
        if not table.is_cuda or table.dtype != torch.float32 or table.dim() != 3 or table.shape[2] != 2 or not table.is_contiguous():
            raise ValueError("table must be a contiguous fp32 CUDA tensor [positions, rot_dim / 2, 2]")
        if layout not in self.LAYOUTS:
            raise ValueError("layout must be 'half' or 'interleaved'")
        self.table = table
        self.args = B.RopeAngles(table.data_ptr(), table.shape[0], 2 * table.shape[1], self.LAYOUTS[layout])


def rope_table(positions: int, rot_dim: int, base: float = 10000.0, scaling: int = B.ROPE_SCALE_NONE, factor: float = 1.0,
               low: float = 0.0, high: float = 0.0, trained_positions: float = 0.0) -> torch.Tensor:
    """The angles of rosaq_rope_table, made on the current stream."""
    table = torch.empty((positions, rot_dim // 2, 2), dtype=torch.float32, device="cuda")
    B.rosaq_rope_table(table.data_ptr(), positions, rot_dim, base, scaling, factor, low, high, trained_positions, current_stream_ptr())
    return table


def rope(r: Rope, x: torch.Tensor, positions: torch.Tensor, head_dim: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """x with its heads turned to their rows' positions (int32 [M]); out may be x.  Rows whose position lies outside the table stay as
    they are in out, and are zero without it."""
    M, width = x.shape
    ldx = _ld("x", x, M, width)
    if width % head_dim:
        raise ValueError("x must hold whole heads")
    at = _integers("positions", positions, _INT32, M)
    device = _device_of(x, positions, r.table, out)
    if device != _current_device():
        with torch.cuda.device(device):
            return rope(r, x, positions, head_dim, out)
    y = torch.zeros((M, width), dtype=_HALF, device=x.device) if out is None else out
    B.rosaq_rope(r.args, at, x.data_ptr(), M, ldx, width // head_dim, head_dim, y.data_ptr(), _ld("out", y, M, width), _stream_on(device))
    return y


class KvCache:
    """Device memory of a quantised cache (rosaq_cache); slot s is token s % page_tokens of page s // page_tokens."""

    def __init__(self, kv_heads: int, head_dim: int, bits: int, page_tokens: int, num_pages: int, device="cuda"):
        self.kv_heads, self.head_dim, self.bits = kv_heads, head_dim, bits
        self.page_tokens, self.num_pages, self.width = page_tokens, num_pages, kv_heads * head_dim
        self.data = torch.empty(B.rosaq_cache_bytes(kv_heads, head_dim, bits, page_tokens, num_pages), dtype=torch.uint8, device=device)
        self.args = B.Cache(kv_heads, head_dim, bits, page_tokens, num_pages, self.data.data_ptr())


def cache_append(cache: KvCache, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rope: Rope | None = None,
                 positions: torch.Tensor | None = None, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None):
    """rosaq_cache_append: keys and values of M tokens to their slots (int64 [M]), keys turned first where `rope` is given, and
    the queries q beside them.  Returns the turned queries (None without q); q_out may be q.  Rows of skipped tokens stay as they are
    in q_out, and are zero without it."""
    M = k.size(0)
    ldk, ldv = _ld("k", k, M, cache.width), _ld("v", v, M, cache.width)
    at_slots = _integers("slots", slots, _INT64, M)
    if rope is None:
        if q is not None:
            raise ValueError("q is only read to be turned: rope is missing")
        device, angles, at = _device_of(k, v, slots, cache.data), None, 0
    else:
        if positions is None:
            raise ValueError("rope needs positions")
        at = _integers("positions", positions, _INT32, M)
        device, angles = _device_of(k, v, slots, cache.data, positions, rope.table, q, q_out), rope.args
    if device != _current_device():
        with torch.cuda.device(device):
            return cache_append(cache, slots, k, v, rope, positions, q, q_out)
    if q is None:
        B.rosaq_cache_append(cache.args, at_slots, M, k.data_ptr(), ldk, v.data_ptr(), ldv, angles, at, stream=_stream_on(device))
        return None
    width = q.size(-1)
    ldq = _ld("q", q, M, width)
    if width % cache.head_dim:
        raise ValueError("q must hold whole heads")
    y = torch.zeros((M, width), dtype=_HALF, device=q.device) if q_out is None else q_out
    B.rosaq_cache_append(cache.args, at_slots, M, k.data_ptr(), ldk, v.data_ptr(), ldv, angles, at, q.data_ptr(), ldq,
                         width // cache.head_dim, y.data_ptr(), _ld("q_out", y, M, width), _stream_on(device))
    return y


def cache_read(cache: KvCache, slots: torch.Tensor, k: torch.Tensor | None = None, v: torch.Tensor | None = None):
    """rosaq_cache_read: (k, v), the values of the slots; both are allocated where neither is given, one alone is read alone.  Rows of
    slots that are none of the cache's stay as they are in what is given, and are zero in what is allocated."""
    M = slots.numel()
    at = _integers("slots", slots, _INT64, M)
    device = _device_of(slots, cache.data, k, v)
    if device != _current_device():
        with torch.cuda.device(device):
            return cache_read(cache, slots, k, v)
    if k is None and v is None:
        k, v = (torch.zeros((M, cache.width), dtype=_HALF, device=slots.device) for _ in range(2))
    pk, ldk = (0, 0) if k is None else (k.data_ptr(), _ld("k", k, M, cache.width))
    pv, ldv = (0, 0) if v is None else (v.data_ptr(), _ld("v", v, M, cache.width))
    B.rosaq_cache_read(cache.args, at, M, pk, ldk, pv, ldv, _stream_on(device))
    return k, v


class AttentionPlan:
    """The bounds of attention calls over one cache and a workspace for them, of the size that these bounds need (fewer sequences may
    need more).  Calls with one plan must not overlap in time."""

    def __init__(self, cache: KvCache, q_heads: int, sequences: int, max_kv: int, max_rows: int = 1, rows: int | None = None,
                 prefix_len: int = 0, causal: bool = True, scale: float | None = None, window: int | None = None, sinks: int = 0):
        """`rows`: rows of q, sequences * max_rows unless given; scale: head_dim^-1/2 unless given.  With `window` a row sees that many
        tokens, its own among them, and the sequence's first `sinks` (rosaq_attention_window)."""
        if window is None and sinks:
            raise ValueError("sinks are those of a window: window is missing")
        self.cache = cache
        self.M, self.width, self.sequences, self.prefix_len = sequences * max_rows if rows is None else rows, q_heads * cache.head_dim, sequences, prefix_len
        self.desc = B.AttentionDesc()
        d = self.desc
        B.int32(q_heads, self.M, sequences, max_kv, max_rows, prefix_len)
        d.cache = C.pointer(cache.args)
        d.q_heads, d.M, d.sequences, d.max_kv, d.max_rows, d.prefix_len = q_heads, self.M, sequences, max_kv, max_rows, prefix_len
        d.causal, d.scale = int(causal), cache.head_dim ** -0.5 if scale is None else scale
        self.window, self.sinks = window, sinks
        need = B.rosaq_workspace_bytes_attention(d) if window is None else B.rosaq_workspace_bytes_attention_window(d, window, sinks)
        self.ws = torch.empty(need, dtype=torch.uint8, device=cache.data.device)
        self.ws_bytes = self.ws.numel()


def attention(plan: AttentionPlan, q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, row_start: torch.Tensor | None = None,
              prefix_pages: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """rosaq_attention, or rosaq_attention_window where the plan has a window: q [rows, q_heads * head_dim], kv_len int32 [sequences], pages int32 [sequences, pages of a sequence],
    row_start int32 [sequences + 1] (without it sequence b has row b), prefix_pages int32.  out must not overlap q; without it,
    rows that belong to no sequence are zero."""
    d, M = plan.desc, plan.M
    ldq = _ld("q", q, M, plan.width)
    if pages.dim() != 2 or pages.size(0) != plan.sequences:
        raise ValueError("pages must be [sequences, pages of a sequence]")
    at_len = _integers("kv_len", kv_len, _INT32, plan.sequences)
    at_pages = _integers("pages", pages, _INT32, -1)
    at_rows = None if row_start is None else _integers("row_start", row_start, _INT32, plan.sequences + 1)
    at_prefix = None
    if plan.prefix_len:
        if prefix_pages is None:
            raise ValueError("the plan has a prefix: prefix_pages is missing")
        at_prefix = _integers("prefix_pages", prefix_pages, _INT32, -1)
        if prefix_pages.numel() * plan.cache.page_tokens < plan.prefix_len:
            raise ValueError("prefix_pages hold fewer tokens than the prefix")
    elif prefix_pages is not None and prefix_pages.numel():
        raise ValueError("prefix_pages given, and the plan has no prefix")
    device = _device_of(q, kv_len, pages, plan.ws, row_start, prefix_pages, out)
    if device != _current_device():
        with torch.cuda.device(device):
            return attention(plan, q, kv_len, pages, row_start, prefix_pages, out)
    y = torch.zeros((M, plan.width), dtype=_HALF, device=q.device) if out is None else out
    d.ldy = _ld("out", y, M, plan.width)
    d.q, d.ldq, d.y = q.data_ptr(), ldq, y.data_ptr()
    d.kv_len, d.pages, d.page_stride, d.row_start, d.prefix_pages = at_len, at_pages, pages.size(1), at_rows, at_prefix
    if plan.window is None:
        B.rosaq_attention(d, plan.ws.data_ptr(), plan.ws_bytes, _stream_on(device))
    else:
        B.rosaq_attention_window(d, plan.window, plan.sinks, plan.ws.data_ptr(), plan.ws_bytes, _stream_on(device))
    return y


# ---- around the projections ------------------------------------------------------------------------------------------

def _row_stride(name: str, x: torch.Tensor, rows: int, width: int, dtype: torch.dtype) -> int:
    """As _ld, of any type."""
    stride = x.stride()
    if x.dtype is not dtype or x.shape != (rows, width) or stride[1] != 1:
        raise ValueError(f"{name} must be a {dtype} tensor [{rows}, {width}] with unit column stride")
    return stride[0] if rows > 1 else width


def _beside(name: str, t: torch.Tensor, shape: torch.Size, dtype: torch.dtype, device: int) -> int:
    """The row stride of a matrix of a call whose first one is of this shape and device (_row_stride and _device_of in one look)."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} tensor {list(shape)} with unit column stride")
    if t.get_device() != device:
        raise ValueError("the tensors of a call must lie on one GPU")
    return shape[1] if t.is_contiguous() else _row_stride(name, t, shape[0], shape[1], dtype)


def _rmsnorm(x, weight, eps, residual, residual_out, y, codes, scales):
    """One rosaq_rmsnorm call on x's device; y, codes and scales: None, or where they go."""
    shape, device = x.shape, x.get_device()
    M, D = shape
    if (M | D) >> 31:
        B.int32(M, D)
    d = B.RmsNormDesc()
    d.M, d.D, d.eps = M, D, eps
    d.ldx, d.x = _beside("x", x, shape, _HALF, device), x.data_ptr()
    if weight is not None:
        if weight.dtype is not _HALF or weight.shape != shape[1:] or not weight.is_contiguous() or weight.get_device() != device:
            raise ValueError(f"weight must be a contiguous fp16 tensor [{D}] on x's GPU")
        d.weight = weight.data_ptr()
    if residual is not None:
        dtype = residual.dtype
        if dtype is torch.float32:
            d.residual_type = B.F32
        elif dtype is not _HALF:
            raise ValueError("residual must be fp16 or fp32")
        d.ld_residual, d.residual = _beside("residual", residual, shape, dtype, device), residual.data_ptr()
        if residual_out is None or residual_out is residual:
            d.ld_residual_out, d.residual_out = d.ld_residual, d.residual
        else:
            d.ld_residual_out, d.residual_out = _beside("residual_out", residual_out, shape, dtype, device), residual_out.data_ptr()
    elif residual_out is not None:
        raise ValueError("residual_out without a residual")
    if y is not None:
        d.ldy, d.y = _beside("out", y, shape, _HALF, device), y.data_ptr()
    if codes is not None:
        d.ld_codes, d.codes = _beside("codes", codes, shape, torch.int8, device), codes.data_ptr()
        if scales.dtype is not torch.float32 or scales.shape != shape[:1] or not scales.is_contiguous() or scales.get_device() != device:
            raise ValueError(f"scales must be a contiguous fp32 tensor [{M}] on x's GPU")
        d.scales = scales.data_ptr()
    if device < 0:
        raise ValueError("the tensors of a call must lie on a GPU")
    if device != _current_device():
        with torch.cuda.device(device):
            B.rosaq_rmsnorm(d, _stream_on(device))
    else:
        B.rosaq_rmsnorm(d, _stream_on(device))


def rmsnorm(x: torch.Tensor, weight: torch.Tensor | None = None, eps: float = 1e-5, residual: torch.Tensor | None = None,
            residual_out: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """rosaq_rmsnorm of x [M, D] + residual (fp16 or fp32): fp16 [M, D].  The sum goes to residual_out, which is residual itself
    unless given; out may be x or residual where the sum does not go there."""
    y = torch.empty(x.shape, dtype=_HALF, device=x.device) if out is None else out
    _rmsnorm(x, weight, eps, residual, residual_out, y, None, None)
    return y


def rmsnorm_codes(x: torch.Tensor, weight: torch.Tensor | None = None, eps: float = 1e-5, residual: torch.Tensor | None = None,
                  residual_out: torch.Tensor | None = None, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None,
                  out: torch.Tensor | None = None):
    """rmsnorm in 8 bits: (codes int8 [M, D], scales fp32 [M]), a value being code * scale; in fp16 too where `out` is given."""
    M, D = x.shape
    if codes is None:
        codes = torch.empty((M, D), dtype=torch.int8, device=x.device)
    if scales is None:
        scales = torch.empty(M, dtype=torch.float32, device=x.device)
    _rmsnorm(x, weight, eps, residual, residual_out, out, codes, scales)
    return codes, scales


class _LogProbs(NamedTuple):
    given: torch.Tensor | None        # fp32 [M, given]
    entropy: torch.Tensor | None      # fp32 [M]
    top_ids: torch.Tensor | None      # int64 [M, top]
    top: torch.Tensor | None          # fp32 [M, top]


class LogProbs(_LogProbs):
    """What logprobs returns: (given, entropy, top_ids, top), None where nothing was asked for.  Made by logprobs_buffers it has a workspace too."""

    workspace: torch.Tensor | None = None


_LOGITS = {torch.float16: B.F16, torch.bfloat16: B.BF16, torch.float32: B.F32}


def logprobs_buffers(logits: torch.Tensor, given: int = 0, top: int = 0, entropy: bool = True) -> LogProbs:
    """Outputs for calls of logprobs over logits of this shape, for loops that keep them, with a workspace.  Calls with one must not overlap
    in time."""
    if logits.dim() != 2 or logits.dtype not in _LOGITS:
        raise ValueError("logits must be [M, V] in fp16, bf16 or fp32")
    if given < 0 or top < 0:
        raise ValueError(f"{given} given tokens and {top} alternatives: neither can be below zero")
    M, V = logits.shape
    B.int32(M, V, given, top)
    device, real = logits.device, torch.float32
    out = LogProbs(torch.empty((M, given), dtype=real, device=device) if given else None,
                   torch.empty(M, dtype=real, device=device) if entropy else None,
                   torch.empty((M, top), dtype=_INT64, device=device) if top else None,
                   torch.empty((M, top), dtype=real, device=device) if top else None)
    d = B.LogprobsDesc()
    d.M, d.V, d.type, d.scale, d.top = M, V, _LOGITS[logits.dtype], 1.0, top
    out.workspace = torch.empty(B.rosaq_workspace_bytes_logprobs(d), dtype=torch.uint8, device=device)
    return out


def logprobs(logits: torch.Tensor, tokens: torch.Tensor | None = None, top: int = 0, entropy: bool = True, scale: float = 1.0,
             out: LogProbs | None = None) -> LogProbs:
    """rosaq_logprobs of logits [M, V] (fp16, bf16 or fp32): of tokens int64 [M, given], or [M] for one of each row (below zero: padding), and
    of the `top` largest, with the entropy.  out (logprobs_buffers) says instead of `entropy` whether that is wanted."""
    shape, device = logits.shape, logits.get_device()
    kind = _LOGITS.get(logits.dtype)
    if len(shape) != 2 or kind is None:
        raise ValueError("logits must be [M, V] in fp16, bf16 or fp32")
    M, V = shape
    given = 0
    if tokens is not None:
        if tokens.dim() not in (1, 2) or tokens.shape[0] != M:
            raise ValueError(f"tokens must be [{M}, given] or [{M}]")
        given = 1 if tokens.dim() == 1 else tokens.shape[1]
    if (M | V | given | top) >> 31:
        B.int32(M, V, given, top)
    d = B.LogprobsDesc()
    d.M, d.V, d.type, d.scale, d.given, d.top = M, V, kind, scale, given, top
    d.ld, d.logits = _beside("logits", logits, shape, logits.dtype, device), logits.data_ptr()
    if tokens is not None:
        d.tokens = _integers("tokens", tokens, _INT64, M * given)
    if out is None:
        out = logprobs_buffers(logits, given, top, entropy)
    for name, t, wanted in (("given", out.given, given), ("entropy", out.entropy, 0), ("top_ids", out.top_ids, top), ("top", out.top, top)):
        if t is None:
            if wanted:
                raise ValueError(f"out.{name} is missing")
        elif t.dtype is not (_INT64 if name == "top_ids" else torch.float32) or t.shape != ((M,) if name == "entropy" else (M, wanted)) or \
                not t.is_contiguous() or (wanted == 0 and name != "entropy"):
            raise ValueError(f"out.{name} must be a contiguous tensor {[M] if name == 'entropy' else [M, wanted]} of its type, and None where nothing is asked for")
    ws = getattr(out, "workspace", None)          # of a plain tuple there is none: no row is shared then
    for t in (tokens, ws, *out):
        if t is not None and t.get_device() != device:
            raise ValueError("the tensors of a call must lie on one GPU")
    if device < 0:
        raise ValueError("the tensors of a call must lie on a GPU")
    d.given_out, d.entropy, d.top_ids, d.top_out = (None if t is None else t.data_ptr() for t in out)
    at_ws, ws_bytes = (0, 0) if ws is None else (ws.data_ptr(), ws.numel())
    if device != _current_device():
        with torch.cuda.device(device):
            B.rosaq_logprobs(d, at_ws, ws_bytes, _stream_on(device))
    else:
        B.rosaq_logprobs(d, at_ws, ws_bytes, _stream_on(device))
    return out
