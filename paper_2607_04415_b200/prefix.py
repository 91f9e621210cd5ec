"""Attention of a batch whose requests share prefixes (system prompts, retrieved passages): what a group of requests shares is
read once for all of them.  The rules are in include/gorio.h; streams, workspaces and graphs as for paged_attention."""
from __future__ import annotations

import math
import struct
from typing import Optional

import torch

from .binding import _invalid, load_library
from .paged import _ATTENTION, _DTYPES, _call, _cuda_index, _fail, _on, _page_pair, _rows_3d, _stream_workspace, _tables_2d, _vector, _without_gradient, _workspace

_PREFIX = struct.Struct("@4Pq2I")


def attention_fields(lib, index, q, pages, key_pages, value_pages, tables, lengths, starts, max_new, scale, causal, window, softcap, slopes, want_lse,
                     out, workspace):
    """Checks what the attention calls have in common beside their pages, whose (shape, key strides, value strides) are `pages`.
    Returns the packed descriptor, out, lse and the workspace, which a captured call has to hold until its last allocation: the graph's
    memory is given out again as soon as nobody does.  (paged_attention does the same in line: on small calls the host's time is
    what counts.)"""
    (n_pages, kv_heads, page_size, dim), ks, vs = pages
    dtype = q.dtype
    if dtype not in _DTYPES:
        raise _invalid("q must be a 3-D bfloat16 or float16 tensor [tokens, heads, head size]")
    qs = _rows_3d("q", q, index, dtype)
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
                           b, t, heads, kv_heads, dim, n_pages, page_size, width, _DTYPES[dtype], 1 if causal else 0, window, max_new,
                           1.0 / math.sqrt(dim) if scale is None else scale, softcap)
    return desc, out, lse, workspace


def prefix_attention(q: torch.Tensor, key_pages: torch.Tensor, value_pages: torch.Tensor, prefix_tables: torch.Tensor,
                     prefix_lengths: torch.Tensor, group_starts: torch.Tensor, tables: torch.Tensor, lengths: torch.Tensor,
                     starts: torch.Tensor, max_new: int, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                     softcap: float = 0.0, slopes: Optional[torch.Tensor] = None, want_lse: bool = False,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Attention of each request's new tokens over the prefix that its group shares and its own cached keys behind it
    (gorio_prefix_attention).

    Requests group_starts[g]:group_starts[g + 1] (int32 [groups + 1]) share the prefix_lengths[g] (int32 [groups]) tokens in the
    pages of prefix_tables[g] (int32 [groups, pages]); the rest is as for paged_attention, where tables and lengths are those of
    each request's own tokens alone.  The result is that of paged_attention over both, the prefix first, read once for
    the whole group.  Besides the workspace a call takes some 40 MB, and 4 bytes for each number of q, until its kernels have run.
    There is no backward pass."""
    if stream is not None:
        with _on(stream, "q", q):
            return prefix_attention(q, key_pages, value_pages, prefix_tables, prefix_lengths, group_starts, tables, lengths, starts, max_new, scale,
                                    causal, window, softcap, slopes, want_lse, out, workspace)
    lib = load_library()
    index = _cuda_index("q", q)
    pages = _page_pair(key_pages, value_pages, index)
    if q.dtype is not key_pages.dtype:
        raise _invalid(f"q must be of the pages' type, {key_pages.dtype}")
    groups = prefix_lengths.shape[0] if isinstance(prefix_lengths, torch.Tensor) and prefix_lengths.dim() == 1 else -1
    _vector("prefix_lengths", prefix_lengths, index)
    _vector("group_starts", group_starts, index, groups + 1)
    prefix_width, prefix_row = _tables_2d(prefix_tables, groups, index)
    if groups < 1:
        raise _invalid("prefix_lengths must name at least one group")
    desc, out, lse, workspace = attention_fields(lib, index, q, pages, key_pages, value_pages, tables, lengths, starts, max_new, scale, causal, window,
                                                 softcap, slopes, want_lse, out, workspace)
    t, heads, dim = q.shape
    # kept by the allocator until the stream has passed the call, as for any tensor of its stream
    scratch = torch.empty(max(1, lib.gorio_prefix_scratch_bytes(index, t, heads, dim)), dtype=torch.uint8, device=q.device)
    desc += _PREFIX.pack(prefix_tables.data_ptr(), prefix_lengths.data_ptr(), group_starts.data_ptr(), scratch.data_ptr(), prefix_row, groups, prefix_width)
    st = _call(lib.gorio_prefix_attention, desc, index)
    if st:
        _fail(lib, st)
    if q.requires_grad or key_pages.requires_grad or value_pages.requires_grad or slopes is not None:
        out, lse = _without_gradient(out, lse, (q, key_pages, value_pages, slopes), "prefix_attention")
    return dict(out=out, lse=lse)
