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
                 prefix_len: int = 0, causal: bool = True, scale: float | None = None):
        """`rows`: rows of q, sequences * max_rows unless given; scale: head_dim^-1/2 unless given."""
        self.cache = cache
        self.M, self.width, self.sequences, self.prefix_len = sequences * max_rows if rows is None else rows, q_heads * cache.head_dim, sequences, prefix_len
        self.desc = B.AttentionDesc()
        d = self.desc
        d.cache = C.pointer(cache.args)
        d.q_heads, d.M, d.sequences, d.max_kv, d.max_rows, d.prefix_len = q_heads, self.M, sequences, max_kv, max_rows, prefix_len
        d.causal, d.scale = int(causal), cache.head_dim ** -0.5 if scale is None else scale
        self.ws = torch.empty(B.rosaq_workspace_bytes_attention(d), dtype=torch.uint8, device=cache.data.device)
        self.ws_bytes = self.ws.numel()


def attention(plan: AttentionPlan, q: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor, row_start: torch.Tensor | None = None,
              prefix_pages: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """rosaq_attention: q [rows, q_heads * head_dim], kv_len int32 [sequences], pages int32 [sequences, pages of a sequence],
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
    B.rosaq_attention(d, plan.ws.data_ptr(), plan.ws_bytes, _stream_on(device))
    return y
