"""The paged key/value cache in 8 bits: keys and values are quantised as they are stored, read back, and attended over as they
lie.  The rules are in include/gorio.h; streams, workspaces and graphs as for the 16-bit cache's calls.

Pages are torch.float8_e4m3fn or torch.int8 tensors [pages, heads, page size, head size], with any strides of the outer axes; each row
of a token and a head has a scale, float32 [pages, heads, page size].  page_tables serves such a cache as it does any."""
from __future__ import annotations

import struct
from typing import Optional, Tuple

import torch

from .binding import _invalid, load_library
from .paged import _DTYPES, _call, _cuda_index, _fail, _on, _rows_3d, _vector, _without_gradient
from .prefix import attention_fields

_FORMATS = {torch.float8_e4m3fn: 0, torch.int8: 1}
_ROWS = struct.Struct("@7P16q8I")
_SCALES = struct.Struct("@2P6q2I")


def _coded_pages(key_pages, value_pages, key_scales, value_scales, index):
    """Checks pages and scales; returns the pages' shape and all four's strides.  On small calls the host's time is what counts: what is right is found
    so in one look, and only what is not goes through the checks one by one."""
    try:
        shape, dtype = key_pages.shape, key_pages.dtype
        n, h, p, _ = shape
        ks, vs = key_pages.stride(), value_pages.stride()
        if (dtype in _FORMATS and value_pages.dtype is dtype and value_pages.shape == shape and ks[3] == 1 and vs[3] == 1
                and key_scales.dtype is torch.float32 and value_scales.dtype is torch.float32 and key_scales.shape == (n, h, p)
                and value_scales.shape == (n, h, p) and key_pages.get_device() == index and value_pages.get_device() == index
                and key_scales.get_device() == index and value_scales.get_device() == index):
            return shape, ks, vs, key_scales.stride(), value_scales.stride()
    except (AttributeError, TypeError, ValueError):
        pass
    for name, t in (("key_pages", key_pages), ("value_pages", value_pages)):
        if not isinstance(t, torch.Tensor) or t.dim() != 4 or t.dtype not in _FORMATS:
            raise _invalid(f"{name} must be a 4-D float8_e4m3fn or int8 tensor [pages, heads, page size, head size]")
        if t.get_device() != index:
            raise _invalid(f"{name} must live on cuda:{index}")
    shape = key_pages.shape
    if shape != value_pages.shape or key_pages.dtype is not value_pages.dtype:
        raise _invalid("key_pages and value_pages differ in shape or type")
    ks, vs = key_pages.stride(), value_pages.stride()
    if ks[3] != 1 or vs[3] != 1:
        raise _invalid("the elements of a head must be contiguous in the pages")
    for name, t in (("key_scales", key_scales), ("value_scales", value_scales)):
        if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != shape[:3]:
            raise _invalid(f"{name} must be a float32 tensor [pages, heads, page size], as the pages")
        if t.get_device() != index:
            raise _invalid(f"{name} must live on cuda:{index}")
    return shape, ks, vs, key_scales.stride(), value_scales.stride()


def _move(store, keys, values, key_pages, value_pages, key_scales, value_scales, slots, index, dtype):
    lib = load_library()
    (pages, heads, page_size, dim), ks, vs, kss, vss = _coded_pages(key_pages, value_pages, key_scales, value_scales, index)
    if dtype not in _DTYPES:
        raise _invalid("keys and values must be bfloat16 or float16")
    k = _rows_3d("keys", keys, index, dtype)
    v = _rows_3d("values", values, index, dtype)
    shape = keys.shape
    if shape != values.shape or shape[1] != heads or shape[2] != dim:
        raise _invalid(f"keys and values must be [tokens, {heads}, {dim}], as the pages")
    _vector("slots", slots, index, shape[0], torch.int64)
    desc = _ROWS.pack(keys.data_ptr(), values.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), key_scales.data_ptr(), value_scales.data_ptr(),
                      slots.data_ptr(), k[0], k[1], v[0], v[1], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], *kss, *vss,
                      shape[0], heads, dim, pages, page_size, _DTYPES[dtype], _FORMATS[key_pages.dtype], 0)
    st = _call(lib.gorio_cache_store_quantized if store else lib.gorio_cache_load_quantized, desc, index)
    if st:
        _fail(lib, st)


def cache_store_quantized(keys: torch.Tensor, values: torch.Tensor, key_pages: torch.Tensor, value_pages: torch.Tensor, key_scales: torch.Tensor,
                          value_scales: torch.Tensor, slots: torch.Tensor, stream=None) -> None:
    """Quantises new keys and values, [tokens, heads, head size] in 16 bits, and stores codes and scales to their slots in place
    (gorio_cache_store_quantized).  Tokens of a negative slot are skipped.  Numbers are stored, without their autograd history."""
    if stream is not None:
        with _on(stream, "key_pages", key_pages):
            return cache_store_quantized(keys, values, key_pages, value_pages, key_scales, value_scales, slots)
    index = _cuda_index("key_pages", key_pages)
    _move(True, keys, values, key_pages, value_pages, key_scales, value_scales, slots, index,
          keys.dtype if isinstance(keys, torch.Tensor) else None)


def cache_load_quantized(key_pages: torch.Tensor, value_pages: torch.Tensor, key_scales: torch.Tensor, value_scales: torch.Tensor, slots: torch.Tensor,
                         dtype: torch.dtype = torch.bfloat16, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                         stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values of the slots, [tokens, heads, head size] of `dtype` (gorio_cache_load_quantized), new or in the two tensors of `out`, which have to
    be of that type; zeros for a negative slot.  There is no backward pass."""
    if stream is not None:
        with _on(stream, "key_pages", key_pages):
            return cache_load_quantized(key_pages, value_pages, key_scales, value_scales, slots, dtype, out)
    index = _cuda_index("key_pages", key_pages)
    if out is None:
        if dtype not in _DTYPES:
            raise _invalid("dtype must be bfloat16 or float16")
        if key_pages.dim() != 4 or not isinstance(slots, torch.Tensor) or slots.dim() != 1:
            raise _invalid("key_pages must be 4-D and slots a 1-D tensor")
        shape = (slots.shape[0], key_pages.shape[1], key_pages.shape[3])
        out = key_pages.new_empty(shape, dtype=dtype), key_pages.new_empty(shape, dtype=dtype)
    keys, values = out
    _move(False, keys, values, key_pages, value_pages, key_scales, value_scales, slots, index, dtype)
    if key_scales.requires_grad or value_scales.requires_grad or key_pages.requires_grad or value_pages.requires_grad:
        return _without_gradient(keys, values, (key_pages, value_pages, key_scales, value_scales), "cache_load_quantized")
    return keys, values


def paged_attention_quantized(q: torch.Tensor, key_pages: torch.Tensor, value_pages: torch.Tensor, key_scales: torch.Tensor, value_scales: torch.Tensor,
                              tables: torch.Tensor, lengths: torch.Tensor, starts: torch.Tensor, max_new: int, scale: Optional[float] = None,
                              causal: bool = True, window: int = 0, softcap: float = 0.0, slopes: Optional[torch.Tensor] = None,
                              want_lse: bool = False, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Attention of each request's new tokens over its keys and values in a quantised cache (gorio_paged_attention_quantized).

    q and the result are bfloat16 or float16, key_pages, value_pages, key_scales and value_scales as cache_store_quantized leaves them;
    all else, the workspaces included, is as for paged_attention.  Prompts are several times faster where scales are contiguous along
    a page.  There is no backward pass."""
    if stream is not None:
        with _on(stream, "q", q):
            return paged_attention_quantized(q, key_pages, value_pages, key_scales, value_scales, tables, lengths, starts, max_new, scale, causal, window,
                                             softcap, slopes, want_lse, out, workspace)
    lib = load_library()
    index = _cuda_index("q", q)
    shape, ks, vs, kss, vss = _coded_pages(key_pages, value_pages, key_scales, value_scales, index)
    desc, out, lse, workspace = attention_fields(lib, index, q, (shape, ks, vs), key_pages, value_pages, tables, lengths, starts, max_new, scale, causal,
                                                 window, softcap, slopes, want_lse, out, workspace)
    desc += _SCALES.pack(key_scales.data_ptr(), value_scales.data_ptr(), *kss, *vss, _FORMATS[key_pages.dtype], 0)
    st = _call(lib.gorio_paged_attention_quantized, desc, index)
    if st:
        _fail(lib, st)
    if (q.requires_grad or key_scales.requires_grad or value_scales.requires_grad or key_pages.requires_grad or value_pages.requires_grad
            or slopes is not None):
        out, lse = _without_gradient(out, lse, (q, key_pages, value_pages, key_scales, value_scales, slopes), "paged_attention_quantized")
    return dict(out=out, lse=lse)
