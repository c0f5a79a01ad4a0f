"""A key/value cache held in 4 bits and attention over it: binding of the squant_cache_* entry points (argument marshalling only; all work runs in the
CUDA library).

A cache is a uint8 tensor [pages, kv heads, page size / 16, 18 * head dim] (alloc_cache): 4.5 bits a value, since 32 neighbouring channels of a key or value share
a scale.  What it stands for is exact in bfloat16, and every call sees the same values.

The calls share three int32 tensors next to the cache, which are read on the device, so that a captured graph may be replayed with other contents:
  lens    [batch]: positions of each sequence
  pages   [batch, width]: position p of sequence b lies in page pages[b, p // page size]; columns behind a sequence's last page are not read
  starts  [batch + 1], or None: rows starts[b] .. starts[b + 1] of k, v, q and the outputs are the LAST positions of sequence b, which are counted in lens[b];
          None: row b is the last position of sequence b
Rows behind the last sequence (a batch padded to a fixed size) are left as they are.  Nothing that the tensors hold leads outside the cache: lengths are cut to what
pages covers, starts to the rows there are, and a page that the cache does not have counts as not there.

None of the calls is recorded by autograd: inputs that require a gradient are refused where one would be recorded (grad mode on), and inputs that carry a forward-mode tangent.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple, Union

import torch
from torch.autograd import forward_ad

from . import binding, linear
from .binding import _check, load_library
from .linear import _TYPES, _On, _ptr, _result

GRANULE = 16   # positions that are stored together


class CacheRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_count", ctypes.c_int64), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("batch", ctypes.c_int32), ("width", ctypes.c_int32), ("lens", ctypes.c_void_p), ("pages", ctypes.c_void_p),
                ("pages_stride", ctypes.c_int64), ("starts", ctypes.c_void_p), ("rows", ctypes.c_int64)]


class CacheMoveArgs(ctypes.Structure):
    _fields_ = [("rows", CacheRows), ("dtype", ctypes.c_uint32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64),
                ("k_head_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("v_head_stride", ctypes.c_int64)]


class CacheAttentionArgs(ctypes.Structure):
    _fields_ = [("rows", CacheRows), ("dtype", ctypes.c_uint32), ("group", ctypes.c_int32), ("most", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64), ("out", ctypes.c_void_p),
                ("out_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64), ("lse", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_int64)]


_device = linear._device
_ready = None
_checked = (None, None, None)   # extension, library, and the extension if it was built with the library's argument structs


def _native():
    """The extension that makes whole calls for plain tensors (None: not built, or built with other argument structs)."""
    global _checked
    if _checked[0] is binding._marshal and _checked[1] is binding._lib and _checked[1] is not None:
        return _checked[2]
    if not torch.cuda.is_initialized():
        return None
    m, lib = binding._marshal, _lib()
    fits = (getattr(m, "cache_move_bytes", None) == ctypes.sizeof(CacheMoveArgs) and getattr(m, "cache_attention_bytes", None) == ctypes.sizeof(CacheAttentionArgs)
            and binding._raw_stream is not None)
    if fits:
        m.use_cache(*(ctypes.cast(getattr(lib, f), ctypes.c_void_p).value for f in ("squant_cache_write", "squant_cache_read", "squant_cache_attention",
                                                                                   "squant_cache_attention_workspace")))
    _checked = (m, lib, m if fits else None)
    return _checked[2]


def _lib() -> ctypes.CDLL:
    global _ready
    lib = load_library()
    if _ready is not lib:
        vp, move, attention = ctypes.c_void_p, ctypes.POINTER(CacheMoveArgs), ctypes.POINTER(CacheAttentionArgs)
        lib.squant_cache_write.argtypes = lib.squant_cache_read.argtypes = [move, vp]
        lib.squant_cache_attention.argtypes = [attention, vp]
        lib.squant_cache_attention_workspace.argtypes = lib.squant_cache_attention_plan.argtypes = [attention]
        for f in ("squant_cache_write", "squant_cache_read", "squant_cache_attention", "squant_cache_attention_plan"):
            getattr(lib, f).restype = ctypes.c_int
        lib.squant_cache_attention_workspace.restype = ctypes.c_int64
        _ready = lib
    return lib


def alloc_cache(pages: int, kv_heads: int, head_dim: int, *, page_size: int = 64, device: Union[torch.device, str, None] = "cuda") -> torch.Tensor:
    """A cache of `pages` pages, all zeros.  head_dim: 64, 128 or 256; page_size: a multiple of 16."""
    if pages < 0 or kv_heads < 1:
        raise ValueError("a cache needs at least one kv head and no fewer than zero pages")
    if head_dim not in (64, 128, 256):
        raise ValueError("head_dim must be 64, 128 or 256")
    if page_size < GRANULE or page_size % GRANULE:
        raise ValueError(f"page_size must be a multiple of {GRANULE}")
    return torch.zeros((pages, kv_heads, page_size // GRANULE, 18 * head_dim), dtype=torch.uint8, device=device)


def _index(t: torch.Tensor, shape: Tuple[int, ...], what: str, device: torch.device) -> None:
    if t.dtype != torch.int32 or t.shape != shape or t.device != device:
        raise ValueError(f"{what} must be an int32 tensor {list(shape)} next to the cache")
    if t.numel() and t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the elements of {what} must lie next to each other")


def _cache_rows(cache: torch.Tensor, lens: torch.Tensor, pages: torch.Tensor, starts: Optional[torch.Tensor], rows: int) -> CacheRows:
    if cache.dtype != torch.uint8 or cache.dim() != 4 or cache.shape[3] not in (18 * 64, 18 * 128, 18 * 256) or not cache.is_contiguous():
        raise ValueError("a cache is a contiguous uint8 tensor [pages, kv heads, page size / 16, 18 * head dim], as of alloc_cache")
    if cache.shape[1] < 1 or cache.shape[2] < 1:
        raise ValueError("a cache has at least one kv head and one granule of 16 positions a page")
    device = cache.device
    if lens.dim() != 1 or pages.dim() != 2:
        raise ValueError("lens must be an int32 tensor [batch], pages an int32 tensor [batch, width]")
    batch = lens.shape[0]
    _index(lens, (batch,), "lens", device)
    _index(pages, (batch, pages.shape[1]), "pages", device)
    if starts is not None:
        _index(starts, (batch + 1,), "starts", device)
    if max(cache.shape[1], cache.shape[2] * GRANULE, batch, pages.shape[1]) >= 1 << 31:
        raise ValueError("kv heads, a page's positions, sequences and columns of pages are counted in 32 bits")
    if starts is None and rows != batch:
        raise ValueError(f"without starts there is one row a sequence: {rows} rows, {batch} sequences")
    return CacheRows(_ptr(cache), cache.shape[0], cache.shape[1], cache.shape[3] // 18, cache.shape[2] * GRANULE, batch, pages.shape[1], _ptr(lens),
                     _ptr(pages), pages.stride(0), _ptr(starts), rows)


def _heads(t: torch.Tensor, rows: Optional[int], heads: int, dim: int, what: str, device: torch.device, dtype: Optional[torch.dtype]) -> None:
    if t.dim() != 3 or t.shape[1:] != (heads, dim) or (rows is not None and t.shape[0] != rows) or t.device != device:
        raise ValueError(f"{what} must be a tensor [{'rows' if rows is None else rows}, {heads}, {dim}] next to the cache")
    if t.dtype not in _TYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{what} must be {'bfloat16 or float16' if dtype is None else dtype}")
    if t.stride(2) != 1 and t.numel():
        raise ValueError(f"the channels of {what} must lie next to each other")


def _no_graph(what: str, *inputs: Optional[torch.Tensor]) -> None:
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs):
        raise ValueError(f"{what} is not recorded by autograd: call it under torch.no_grad()")
    if any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in inputs):
        raise ValueError(f"{what} has no forward-mode derivative: its inputs must not carry a tangent")


def _written(*tensors: Optional[torch.Tensor]) -> None:
    for t in tensors:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


def squant_cache_write(cache: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, pages: torch.Tensor,
                       starts: Optional[torch.Tensor] = None, *, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantizes keys and values [rows, kv heads, head dim] (bfloat16 or float16; slices of wider buffers are taken as they are) into the cache.

    32 neighbouring channels share a scale, the largest magnitude over 7 rounded to four significant bits; a value is at most half a scale off.  Groups with an
    infinity, a NaN or a magnitude from 2^120 on stand for NaN.  No two rows of a call may have the same place."""
    native = None if stream is not None else _native()
    if native is not None:
        device = _device()
        if _result(native.cache_write(binding._raw_stream(device), device, cache, lens, pages, starts, k, v)) is not None:
            return
    _no_graph("squant_cache_write", k, v)
    device = cache.device
    with _On(device, stream) as handle:
        if k.dim() != 3:
            raise ValueError("k must be a tensor [rows, kv heads, head dim]")
        r = _cache_rows(cache, lens, pages, starts, k.shape[0])
        _heads(k, None, r.kv_heads, r.head_dim, "k", device, None)
        _heads(v, r.rows, r.kv_heads, r.head_dim, "v", device, k.dtype)
        a = CacheMoveArgs(r, _TYPES[k.dtype], _ptr(k), _ptr(v), k.stride(0), k.stride(1), v.stride(0), v.stride(1))
        _check(_lib().squant_cache_write(ctypes.byref(a), handle))
    _written(cache)


def squant_cache_read(cache: torch.Tensor, lens: torch.Tensor, pages: torch.Tensor, starts: Optional[torch.Tensor], rows: int, *,
                      dtype: torch.dtype = torch.bfloat16, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values [rows, kv heads, head dim] that the cache holds for these rows: exact in bfloat16, rounded in float16.

    Rows before a sequence's first position or in a page that is not there are zeros.  k, v: tensors to write, both or none; in new ones, rows behind the
    last sequence hold anything."""
    native = None if stream is not None or k is not None or v is not None or dtype not in _TYPES else _native()
    if native is not None:
        device = _device()
        got = native.cache_read(binding._raw_stream(device), device, cache, lens, pages, starts, rows, _TYPES[dtype])
        if got is not None:
            return _result(got)
    device = cache.device
    with _On(device, stream) as handle:
        if rows < 0:
            raise ValueError("there are no fewer than zero rows")
        if (k is None) != (v is None):
            raise ValueError("k and v are given both or not at all")
        if k is None and dtype not in _TYPES:
            raise ValueError("keys and values are read as bfloat16 or float16")
        r = _cache_rows(cache, lens, pages, starts, rows)
        given = k is not None
        if given:
            _no_graph("squant_cache_read", k, v)
            _heads(k, rows, r.kv_heads, r.head_dim, "k", device, None)
            _heads(v, rows, r.kv_heads, r.head_dim, "v", device, k.dtype)
        else:
            k, v = torch.empty((2, rows, r.kv_heads, r.head_dim), dtype=dtype, device=device).unbind(0)
        a = CacheMoveArgs(r, _TYPES[k.dtype], _ptr(k), _ptr(v), k.stride(0), k.stride(1), v.stride(0), v.stride(1))
        _check(_lib().squant_cache_read(ctypes.byref(a), handle))
    if given:
        _written(k, v)
    return k, v


def squant_cache_attention(q: torch.Tensor, cache: torch.Tensor, lens: torch.Tensor, pages: torch.Tensor, starts: Optional[torch.Tensor] = None, *,
                           scale: Optional[float] = None, most: int = 0, lse: bool = False, out: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None):
    """Softmax attention of queries [rows, heads, head dim] over the cache, which holds their own positions already: a row sees its sequence's positions up to its own.

    heads is a multiple of the cache's kv heads; query head h reads kv head h // (heads / kv heads).  scale: of the products, 1 / sqrt(head dim) by default.
    most: the number of rows that no sequence has more of, where the caller knows it: it chooses the kernel, and with it the results' last places; without it, a step of
    many sequences takes the slower one, for prompts.  With `lse` returns
    (out, logarithms of the sums of exponentials, fp32 [rows, heads]).  out: the tensor to write, like q, which it must not overlap; in a new one, rows behind the last sequence hold
    anything.  A row that sees nothing is zeros, its lse -infinity.

    Weights are rounded to q's type for their product with the values in sequences of more than 128 rows times query heads of a kv head, and keep twice its bits elsewhere.
    fp16 wants a cache of what fp16 holds: groups of 32 channels up to 65,504.  From 2^-18 on their values are those that squant_cache_read returns, below they are 2^-22 off at
    most."""
    native = None if stream is not None or q.dim() != 3 else _native()
    if native is not None:
        device = _device()
        got = native.cache_attention(binding._raw_stream(device), device, cache, lens, pages, starts, q, out, 1.0 / math.sqrt(q.shape[2] or 1) if scale is None else scale, most, lse)
        if got is not None:
            return _result(got)
    _no_graph("squant_cache_attention", q, out)
    device = cache.device
    with _On(device, stream) as handle:
        if q.dim() != 3:
            raise ValueError("q must be a tensor [rows, heads, head dim]")
        r = _cache_rows(cache, lens, pages, starts, q.shape[0])
        heads = q.shape[1]
        if heads < 1 or heads % r.kv_heads:
            raise ValueError(f"{heads} query heads are no multiple of {r.kv_heads} kv heads")
        _heads(q, None, heads, r.head_dim, "q", device, None)
        if most < 0:
            raise ValueError("most must not be negative")
        written = out
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=device)
        _heads(out, r.rows, heads, r.head_dim, "out", device, q.dtype)
        sums = torch.empty((r.rows, heads), dtype=torch.float32, device=device) if lse else None
        if scale is None:
            scale = 1.0 / math.sqrt(r.head_dim)
        a = CacheAttentionArgs(r, _TYPES[q.dtype], heads // r.kv_heads, min(most, (1 << 31) - 1), scale, _ptr(q), q.stride(0), q.stride(1), _ptr(out), out.stride(0), out.stride(1),
                               _ptr(sums), None, 0)
        lib = _lib()
        linear._run(lib.squant_cache_attention, lib.squant_cache_attention_workspace, a, handle, device)
    _written(written)
    return (out, sums) if lse else out
