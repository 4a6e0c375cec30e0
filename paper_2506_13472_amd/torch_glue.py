"""PyTorch is used for device memory and streams only: allocate y and the
workspace, hand raw pointers and the current stream to the C ABI."""
from __future__ import annotations

import ctypes as C

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

def _matrix(name: str, x: torch.Tensor, width: int, rows: int | None = None) -> torch.Tensor:
    if not x.is_cuda or x.dtype != torch.float16 or x.dim() != 2 or x.stride(1) != 1 or x.shape[1] != width:
        raise ValueError(f"{name} must be a 2-D fp16 CUDA tensor of {width} columns with unit column stride")
    if rows is not None and x.shape[0] != rows:
        raise ValueError(f"{name} must have {rows} rows")
    return x


def _integers(name: str, t: torch.Tensor, dtype: torch.dtype, count: int | None = None) -> int:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or (count is not None and t.numel() != count):
        raise ValueError(f"{name} must be a contiguous {dtype} CUDA tensor" + (f" of {count} elements" if count is not None else ""))
    return t.data_ptr()


def _on_device_of(*tensors) -> torch.cuda.device | None:
    """A guard that makes the tensors' device current, or None where it is; raises where they lie on several."""
    index = tensors[0].device.index
    for t in tensors[1:]:
        if t is not None and t.device.index != index:
            raise ValueError("the tensors of a call must lie on one device")
    return None if index == torch.cuda.current_device() else torch.cuda.device(index)


def _ld(x: torch.Tensor) -> int:
    """Row stride; of a single row, whose stride torch leaves open, its width."""
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


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
    """x with its heads turned to their rows' positions (int32 [M]); out may be x."""
    M, width = x.shape
    _matrix("x", x, width)
    if width % head_dim:
        raise ValueError("x must hold whole heads")
    at = _integers("positions", positions, torch.int32, M)
    guard = _on_device_of(x, positions, r.table, out)
    if guard:
        with guard:
            return rope(r, x, positions, head_dim, out)
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else _matrix("out", out, width, M)
    B.rosaq_rope(r.args, at, x.data_ptr(), M, _ld(x), width // head_dim, head_dim, y.data_ptr(), _ld(y), current_stream_ptr())
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
    the queries q beside them.  Returns the turned queries (None without q); q_out may be q."""
    M = k.shape[0]
    _matrix("k", k, cache.width)
    _matrix("v", v, cache.width, M)
    at_slots = _integers("slots", slots, torch.int64, M)
    at = 0
    if rope is not None:
        if positions is None:
            raise ValueError("rope needs positions")
        at = _integers("positions", positions, torch.int32, M)
    elif q is not None:
        raise ValueError("q is only read to be turned: rope is missing")
    guard = _on_device_of(k, v, slots, cache.data, positions, q, q_out, None if rope is None else rope.table)
    if guard:
        with guard:
            return cache_append(cache, slots, k, v, rope, positions, q, q_out)
    if q is None:
        B.rosaq_cache_append(cache.args, at_slots, M, k.data_ptr(), _ld(k), v.data_ptr(), _ld(v),
                             None if rope is None else rope.args, at, stream=current_stream_ptr())
        return None
    _matrix("q", q, q.shape[1], M)
    if q.shape[1] % cache.head_dim:
        raise ValueError("q must hold whole heads")
    y = torch.empty_like(q, memory_format=torch.contiguous_format) if q_out is None else _matrix("q_out", q_out, q.shape[1], M)
    B.rosaq_cache_append(cache.args, at_slots, M, k.data_ptr(), _ld(k), v.data_ptr(), _ld(v), rope.args, at, q.data_ptr(), _ld(q),
                         q.shape[1] // cache.head_dim, y.data_ptr(), _ld(y), current_stream_ptr())
    return y


def cache_read(cache: KvCache, slots: torch.Tensor, k: torch.Tensor | None = None, v: torch.Tensor | None = None):
    """rosaq_cache_read: (k, v), the values of the slots; both are allocated where neither is given, one alone is read alone."""
    M = slots.numel()
    at = _integers("slots", slots, torch.int64)
    guard = _on_device_of(slots, cache.data, k, v)
    if guard:
        with guard:
            return cache_read(cache, slots, k, v)
    if k is None and v is None:
        k, v = (torch.empty((M, cache.width), dtype=torch.float16, device=slots.device) for _ in range(2))
    for name, x in (("k", k), ("v", v)):
        if x is not None:
            _matrix(name, x, cache.width, M)
    B.rosaq_cache_read(cache.args, at, M, 0 if k is None else k.data_ptr(), 0 if k is None else _ld(k),
                       0 if v is None else v.data_ptr(), 0 if v is None else _ld(v), current_stream_ptr())
    return k, v


class AttentionPlan:
    """The bounds of attention calls over one cache and a workspace for them.  Calls with one plan must not overlap in time."""

    def __init__(self, cache: KvCache, q_heads: int, sequences: int, max_kv: int, max_rows: int = 1, rows: int | None = None,
                 prefix_len: int = 0, causal: bool = True, scale: float | None = None):
        """`rows`: rows of q, sequences * max_rows unless given."""
        self.cache = cache
        self.desc = B.AttentionDesc()
        d = self.desc
        d.cache = C.pointer(cache.args)
        d.q_heads, d.sequences, d.max_kv, d.max_rows, d.prefix_len = q_heads, sequences, max_kv, max_rows, prefix_len
        d.M = sequences * max_rows if rows is None else rows
        d.causal, d.scale = int(causal), cache.head_dim ** -0.5 if scale is None else scale
        self.ws = torch.empty(B.rosaq_workspace_bytes_attention(d), dtype=torch.uint8, device=cache.data.device)


def attention(plan: AttentionPlan, q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, row_start: torch.Tensor | None = None,
              prefix_pages: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """rosaq_attention: q [rows, q_heads * head_dim], kv_len int32 [sequences], pages int32 [sequences, pages of a sequence],
    row_start int32 [sequences + 1] (without it sequence b has row b), prefix_pages int32.  out must not overlap q; without it,
    rows that belong to no sequence are zero."""
    d, cache = plan.desc, plan.cache
    width = d.q_heads * cache.head_dim
    _matrix("q", q, width, d.M)
    at_len = _integers("kv_len", kv_len, torch.int32, d.sequences)
    at_pages = _integers("pages", pages, torch.int32)
    if pages.dim() != 2 or pages.shape[0] != d.sequences:
        raise ValueError("pages must be [sequences, pages of a sequence]")
    at_rows = None if row_start is None else _integers("row_start", row_start, torch.int32, d.sequences + 1)
    at_prefix = None
    if d.prefix_len:
        if prefix_pages is None:
            raise ValueError("the plan has a prefix: prefix_pages is missing")
        at_prefix = _integers("prefix_pages", prefix_pages, torch.int32)
        if prefix_pages.numel() * cache.page_tokens < d.prefix_len:
            raise ValueError("prefix_pages hold fewer tokens than the prefix")
    guard = _on_device_of(q, kv_len, pages, cache.data, row_start, prefix_pages, out)
    if guard:
        with guard:
            return attention(plan, q, kv_len, pages, row_start, prefix_pages, out)
    y = torch.zeros((d.M, width), dtype=torch.float16, device=q.device) if out is None else _matrix("out", out, width, d.M)
    d.q, d.ldq, d.y, d.ldy = q.data_ptr(), _ld(q), y.data_ptr(), _ld(y)
    d.kv_len, d.pages, d.page_stride, d.row_start, d.prefix_pages = at_len, at_pages, pages.shape[1], at_rows, at_prefix
    B.rosaq_attention(d, plan.ws.data_ptr(), plan.ws.numel(), current_stream_ptr())
    return y
