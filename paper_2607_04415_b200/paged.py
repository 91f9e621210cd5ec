"""Paged key/value cache: page tables from request lengths, the store of new keys and values, and
attention of new tokens over the cached pages.  The rules of the three calls are in include/gorio.h;
this module checks tensors and passes their pointers on.

The calls run on the current stream of the tensors' device (or on their keyword argument `stream`), do
not wait for the GPU and may be captured into a CUDA graph.  A tensor last used on another stream has to be made
ready for this one by the caller, as for any torch operation."""
from __future__ import annotations

import math
import struct
from typing import Optional

import torch

from .binding import GorioError, _invalid, load_library

_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_TABLES = struct.Struct("@12Pq6I")
_STORE = struct.Struct("@5P10q6I")
_ATTENTION = struct.Struct("@10P11q12I2f")
_COUNTER_BYTES = 1 << 16      # the part of an attention workspace that starts as zeros
_WORKSPACES = {}              # (device, stream) -> workspace; calls on one stream do not overlap

_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice
_current_stream_captured = torch._C._cuda_isCurrentStreamCapturing


def _fail(lib, status):
    raise GorioError(status, lib.gorio_last_error(None).decode())


def _vector(name, t, index, length=None, dtype=torch.int32):
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != 1 or not t.is_contiguous():
        raise _invalid(f"{name} must be a contiguous 1-D {dtype} tensor")
    if t.get_device() != index:
        raise _invalid(f"{name} must live on cuda:{index}")
    if length is not None and t.shape[0] != length:
        raise _invalid(f"{name} has {t.shape[0]} elements, expected {length}")


def _tables_2d(tables, rows, index):
    if not isinstance(tables, torch.Tensor) or tables.dtype is not torch.int32 or tables.dim() != 2:
        raise _invalid("tables must be a 2-D int32 tensor [requests, pages]")
    if tables.get_device() != index:
        raise _invalid(f"tables must live on cuda:{index}")
    b, width = tables.shape
    if b != rows:
        raise _invalid(f"tables have {b} rows, expected {rows}")
    row, one = tables.stride()
    if width < 1 or (width > 1 and one != 1):
        raise _invalid("tables need at least one page and contiguous rows")
    return width, row


def _page_pair(key_pages, value_pages, index):
    """Checks the two page tensors [pages, heads, page size, head size]; returns their shape and strides."""
    for name, t in (("key_pages", key_pages), ("value_pages", value_pages)):
        if not isinstance(t, torch.Tensor) or t.dim() != 4 or t.dtype not in _DTYPES:
            raise _invalid(f"{name} must be a 4-D bfloat16 or float16 tensor [pages, heads, page size, head size]")
        if t.get_device() != index:
            raise _invalid(f"{name} must live on cuda:{index}")
    shape = key_pages.shape
    if shape != value_pages.shape or key_pages.dtype is not value_pages.dtype:
        raise _invalid("key_pages and value_pages differ in shape or type")
    ks, vs = key_pages.stride(), value_pages.stride()
    if ks[3] != 1 or vs[3] != 1:
        raise _invalid("the elements of a head must be contiguous in the pages")
    return shape, ks, vs


def _rows_3d(name, t, index, dtype):
    if not isinstance(t, torch.Tensor) or t.dim() != 3 or t.dtype is not dtype:
        raise _invalid(f"{name} must be a 3-D {dtype} tensor [tokens, heads, head size]")
    if t.get_device() != index:
        raise _invalid(f"{name} must live on cuda:{index}")
    strides = t.stride()
    if strides[2] != 1:
        raise _invalid(f"the elements of a head must be contiguous in {name}")
    return strides


def _cuda_index(name, t):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise _invalid(f"{name} must be a CUDA tensor")
    return t.get_device()


def _on(stream, name, t):
    """The context of a `stream` argument, which has to be one of the tensors' device: work would go to that device's current stream."""
    index = _cuda_index(name, t)
    if getattr(stream, "device_index", None) != index:
        raise _invalid(f"stream must be a stream of cuda:{index}, where {name} lives")
    return torch.cuda.stream(stream)


def _call(entry, desc, device_index):
    """The C call on the current stream of the tensors' device, which is made current for it."""
    s = _raw_stream(device_index)
    was = _current_device()
    if was == device_index:
        return entry(desc, s)
    torch._C._cuda_setDevice(device_index)
    try:
        return entry(desc, s)
    finally:
        torch._C._cuda_setDevice(was)


class _NoBackward(torch.autograd.Function):
    """Hands results on, and refuses to go back through them."""

    @staticmethod
    def forward(ctx, call, out, lse, *inputs):
        ctx.call = call
        return out, lse

    @staticmethod
    def backward(ctx, *gradients):
        raise _invalid(f"{ctx.call} has no backward pass: its gradients do not exist (torch.no_grad() or detach() says that none are meant)")


def _without_gradient(out, lse, inputs, call="paged_attention"):
    """The results as they are, or, where an input asks for a gradient, as results whose backward pass raises."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs):
        return _NoBackward.apply(call, out, lse, *inputs)
    return out, lse


def page_tables(lengths: torch.Tensor, new_lens: torch.Tensor, tables: torch.Tensor, free_pages: torch.Tensor,
                free_count: torch.Tensor, page_size: int, n_tokens: int, stream=None) -> dict:
    """Gives the new tokens of a step their pages and slots (gorio_page_tables).

    lengths, new_lens: int32 [requests], cached and new tokens; tables: int32 [requests, pages], updated in
    place; free_pages: int32, a stack of free pages of which free_count (int32 [1]) are left, taken
    from the top; n_tokens: the sum of new_lens.  Returns a dict of tensors: slots (int64) and
    positions, requests of each new token, starts [requests + 1], lengths after the step, served,
    free_count after the step, and tables.  Requests that find no pages are not served: slots -1."""
    if stream is not None:
        with _on(stream, "lengths", lengths):
            return page_tables(lengths, new_lens, tables, free_pages, free_count, page_size, n_tokens)
    lib = load_library()
    index = _cuda_index("lengths", lengths)
    b = lengths.shape[0] if lengths.dim() == 1 else -1
    _vector("lengths", lengths, index)
    _vector("new_lens", new_lens, index, b)
    width, row = _tables_2d(tables, b, index)
    _vector("free_pages", free_pages, index)
    _vector("free_count", free_count, index, 1)
    if n_tokens < 0 or page_size < 1 or n_tokens >= 1 << 31 or page_size >= 1 << 31:
        raise _invalid("n_tokens must not be negative and page_size must be positive")
    slots = lengths.new_empty(n_tokens, dtype=torch.int64)
    # one allocation for the int32 results: their views cost less than an allocation each
    ints = lengths.new_empty(2 * n_tokens + 3 * b + 2)
    positions, requests, starts, out_lengths, served, left = torch.unsafe_split_with_sizes(ints, (n_tokens, n_tokens, b + 1, b, b, 1))
    at = ints.data_ptr()
    to_starts = at + 8 * n_tokens
    desc = _TABLES.pack(lengths.data_ptr(), new_lens.data_ptr(), tables.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(),
                        slots.data_ptr(), at, at + 4 * n_tokens, to_starts, to_starts + 4 * (b + 1), to_starts + 4 * (2 * b + 1),
                        to_starts + 4 * (3 * b + 1), row, b, width, free_pages.shape[0], page_size, n_tokens, 0)
    st = _call(lib.gorio_page_tables, desc, index)
    if st:
        _fail(lib, st)
    return dict(tables=tables, slots=slots, positions=positions, requests=requests, starts=starts, lengths=out_lengths, served=served,
                free_count=left)


def cache_store(keys: torch.Tensor, values: torch.Tensor, key_pages: torch.Tensor, value_pages: torch.Tensor, slots: torch.Tensor,
                stream=None) -> None:
    """Stores new keys and values, [tokens, heads, head size], to their slots of the pages in place
    (gorio_cache_store).  Tokens of a negative slot are skipped.  Numbers are stored, without their autograd history."""
    if stream is not None:
        with _on(stream, "key_pages", key_pages):
            return cache_store(keys, values, key_pages, value_pages, slots)
    lib = load_library()
    index = _cuda_index("key_pages", key_pages)
    (pages, heads, page_size, dim), ks, vs = _page_pair(key_pages, value_pages, index)
    k = _rows_3d("keys", keys, index, key_pages.dtype)
    v = _rows_3d("values", values, index, key_pages.dtype)
    shape = keys.shape
    if shape != values.shape or shape[1] != heads or shape[2] != dim:
        raise _invalid(f"keys and values must be [tokens, {heads}, {dim}], as the pages")
    _vector("slots", slots, index, shape[0], torch.int64)
    desc = _STORE.pack(keys.data_ptr(), values.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), slots.data_ptr(), k[0], k[1], v[0], v[1],
                       ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], shape[0], heads, dim, pages, page_size, 0)
    st = _call(lib.gorio_cache_store, desc, index)
    if st:
        _fail(lib, st)


def _stream_workspace(index):
    """The workspace that this module keeps for the current stream of a device.  While that stream is captured, always a new one, which
    belongs to the graph (its zeroing is captured too): a replay may run beside calls on the stream, or beside other graphs of it."""
    if _current_device() != index:
        with torch.cuda.device(index):
            return _stream_workspace(index)
    if _current_stream_captured():
        return attention_workspace(torch.device("cuda", index))
    key = (index, _raw_stream(index))
    ws = _WORKSPACES.get(key)
    if ws is None:
        ws = _WORKSPACES[key] = attention_workspace(torch.device("cuda", index))
    return ws


def attention_workspace(device=None) -> torch.Tensor:
    """A new workspace for paged_attention on `device` (default: the current one), made on the current stream."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    index = device.index if device.index is not None else torch.cuda.current_device()
    n = load_library().gorio_attention_workspace_bytes(index)
    if n == 0:
        raise GorioError(2, f"no CUDA device {index}")
    ws = torch.empty(n, dtype=torch.uint8, device=torch.device("cuda", index))
    ws[:_COUNTER_BYTES].zero_()
    return ws


def _workspace(lib, t, index):
    if not isinstance(t, torch.Tensor) or t.get_device() != index or t.dtype is not torch.uint8 or not t.is_contiguous() or (
            t.numel() < lib.gorio_attention_workspace_bytes(index)):
        raise _invalid("workspace must come from attention_workspace() for this device")


def attention_check(workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Raises GorioError if a paged_attention call with this workspace (default: the current stream's) ran into the time
    limit of a wait inside its kernel (gorio_attention_check).  Waits for the stream."""
    if stream is not None:
        if workspace is not None:
            with _on(stream, "workspace", workspace):
                return attention_check(workspace)
        with torch.cuda.stream(stream):
            return attention_check()
    lib = load_library()
    if workspace is None:
        workspace = _WORKSPACES.get((torch.cuda.current_device(), _raw_stream(torch.cuda.current_device())))
        if workspace is None:
            return
    index = _cuda_index("workspace", workspace)
    _workspace(lib, workspace, index)
    st = _call(lib.gorio_attention_check, workspace.data_ptr(), index)
    if st:
        _fail(lib, st)


def attention_wait_limit(seconds: float = 0.0) -> None:
    """The limit of a wait inside a paged_attention kernel, for calls from now on (gorio_attention_wait_limit); 0: the 10 s it has
    unless set.  A call whose wait passes it ends, and attention_check raises."""
    if not 0.0 <= seconds < 1e9:
        raise _invalid("the limit of a wait must not be negative, nor longer than 1e9 s")
    load_library().gorio_attention_wait_limit(math.ceil(seconds * 1e9))


def paged_attention(q: torch.Tensor, key_pages: torch.Tensor, value_pages: torch.Tensor, tables: torch.Tensor, lengths: torch.Tensor,
                    starts: torch.Tensor, max_new: int, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                    softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, want_lse: bool = False,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Attention of each request's new tokens over its cached keys and values (gorio_paged_attention).

    q: [tokens, heads, head size] of the pages' type, request r's rows starts[r]:starts[r+1]; pages:
    [pages, key heads, page size, head size], any strides of the outer axes; lengths: int32 [requests],
    keys of each request, the new tokens' own included; max_new: at least the most new tokens of a
    request.  scale defaults to head size ** -0.5.  Returns dict(out, lse), lse None unless wanted.
    `workspace` (attention_workspace()) defaults to one that this module keeps for each stream, or, in a
    captured call, to one of the graph's own, which costs the graph a fill of 64 KB for each call and which attention_check
    cannot see; calls that may overlap need one each.  There is no backward pass: results of inputs that ask for a
    gradient raise when one is taken through them."""
    if stream is not None:
        with _on(stream, "q", q):
            return paged_attention(q, key_pages, value_pages, tables, lengths, starts, max_new, scale, causal, window, softcap, slopes, want_lse,
                                   out, workspace)
    lib = load_library()
    index = _cuda_index("q", q)
    dtype = q.dtype
    (pages, kv_heads, page_size, dim), ks, vs = _page_pair(key_pages, value_pages, index)
    qs = _rows_3d("q", q, index, key_pages.dtype)
    t, heads, qd = q.shape
    if qd != dim:
        raise _invalid(f"q has heads of {qd} elements, the pages of {dim}")
    b = lengths.shape[0] if isinstance(lengths, torch.Tensor) and lengths.dim() == 1 else -1
    _vector("lengths", lengths, index)
    _vector("starts", starts, index, b + 1)
    width, row = _tables_2d(tables, b, index)
    if slopes is not None:
        _vector("slopes", slopes, index, heads, torch.float32)
    if not 0 <= window < 1 << 31 or not 0 <= max_new < 1 << 31:
        raise _invalid("window and max_new must not be negative")
    if out is None:
        out = q.new_empty((t, heads, dim))
        os = (heads * dim, dim)
    else:
        os = _rows_3d("out", out, index, dtype)
        if out.shape != q.shape:
            raise _invalid("out must have the shape of q")
    lse = q.new_empty((t, heads), dtype=torch.float32) if want_lse else None
    if workspace is None:
        workspace = _stream_workspace(index)
    else:
        _workspace(lib, workspace, index)
    desc = _ATTENTION.pack(q.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), out.data_ptr(), lse.data_ptr() if want_lse else 0,
                           tables.data_ptr(), lengths.data_ptr(), starts.data_ptr(), 0 if slopes is None else slopes.data_ptr(),
                           workspace.data_ptr(), qs[0], qs[1], os[0], os[1], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], row,
                           b, t, heads, kv_heads, dim, pages, page_size, width, _DTYPES[dtype], 1 if causal else 0, window, max_new,
                           1.0 / math.sqrt(dim) if scale is None else scale, softcap)
    st = _call(lib.gorio_paged_attention, desc, index)
    if st:
        _fail(lib, st)
    if q.requires_grad or key_pages.requires_grad or value_pages.requires_grad or slopes is not None:      # most calls need no more
        out, lse = _without_gradient(out, lse, (q, key_pages, value_pages, slopes))
    return dict(out=out, lse=lse)
