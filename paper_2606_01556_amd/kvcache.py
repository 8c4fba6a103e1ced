"""The operators between a decoder block's linear layers, for inference: norm and
position rotation of queries and keys, the paged key-value cache in 16, 8 or 4
bits, and the attention of one new token over it.

Binding of the ``tq_kv_*``, ``tq_qk_*`` and ``tq_paged_attention`` entry points of
``libtq.so``; the arithmetic runs in the library's HIP kernels.  As in the rest of
the package, every tensor is checked before the call (the library sees pointers; the
checks are native, in ``csrc/tq_torch.cpp``, since an eager decode step waits for its
host work), nothing is synchronized, and ``stream`` (a torch stream or a hipStream_t;
default: the current one) has to have the inputs ready.

A decode step of one block:

    cache = tq.empty_kv_cache(pages, 16, kv_heads, 128, bits=4)
    ...
    q = tq.qk_norm_rope_append(cache, q, k, v, positions, table, slots, q_weight, k_weight)
    y = tq.paged_attention(cache, q, page_table, lengths)
"""
from __future__ import annotations

import ctypes
import importlib.util
import os

from . import TQError, _HERE, _other_stream, _stream, lib

__all__ = ["KVCache", "empty_kv_cache", "rope_table", "kv_append", "kv_read", "qk_norm_rope",
           "qk_norm_rope_append", "paged_attention"]


class _CacheDesc(ctypes.Structure):     # tq_kv_cache
    _fields_ = [("pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("bits", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scales", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p)]


class _HeadRows(ctypes.Structure):      # tq_head_rows
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _NormRope(ctypes.Structure):      # tq_norm_rope
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("table", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("max_positions", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("eps", ctypes.c_float)]


def declare(L):
    """Argument types of this module's entry points (called as the library loads)."""
    P, I = ctypes.c_void_p, ctypes.c_int
    C, H, N = (ctypes.POINTER(s) for s in (_CacheDesc, _HeadRows, _NormRope))
    L.tq_qk_norm_rope.argtypes = [N, H, H, I, I, I, I, I, P, P, P]
    L.tq_kv_append.argtypes = [C, H, H, P, I, I, P]
    L.tq_qk_norm_rope_append.argtypes = [N, C, H, H, H, P, I, I, I, P, P, P]
    L.tq_kv_read.argtypes = [C, P, I, P, P, I, P]
    L.tq_paged_attention_scratch_bytes.argtypes = [C, I, I, I, I]
    L.tq_paged_attention_scratch_bytes.restype = ctypes.c_size_t
    L.tq_paged_attention.argtypes = [C, H, I, I, I, P, ctypes.c_int64, I, P, ctypes.c_float, I, P, P, P, P]


# ------------------------------------------------------------------ the native half
_native = None


def _load():
    """csrc/tq_torch.cpp, built next to libtq.so and bound to its entry points."""
    global _native, _torch, _get_device, _get_raw
    import torch                        # (its libraries, which the module is linked to)
    path = os.path.join(_HERE, "_tqtorch.so")
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2606_01556_amd.build` "
                           "(there is no fallback)")
    spec = importlib.util.spec_from_file_location("_tqtorch", path)
    native = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(native)
    L = lib()
    native.bind(TQError, torch.OutOfMemoryError, *(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.tq_qk_norm_rope, L.tq_kv_append, L.tq_qk_norm_rope_append, L.tq_kv_read,
        L.tq_paged_attention_scratch_bytes, L.tq_paged_attention)))
    _torch, _get_device, _get_raw = torch, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _native = native
    return native


def _here():
    """The current device and its current stream's hipStream_t."""
    try:
        dev = _get_device()
    except RuntimeError:                 # no GPU: the tensors are refused by name
        return -1, 0
    return dev, _get_raw(dev)


def _elsewhere(stream, inputs, call):
    """call(device, hipStream_t) on a given stream.  Where that is not the current one,
    outputs and scratch come from its memory (a block of the current stream's may
    still be in use by the work it was freed behind); outputs may then be used, and
    dropped, on the current stream, and inputs stay until that stream is done."""
    torch = _torch
    torch.cuda.current_stream()          # initialises CUDA
    dev, st = _get_device(), _stream(stream)
    device = torch.device("cuda", dev)
    other = _other_stream(stream, st, device)
    if other is None:
        return call(dev, st)
    with torch.cuda.stream(other):
        out = call(dev, st)
    for t in inputs:
        if t is not None:
            t.record_stream(other)
    for t in out if type(out) is tuple else () if out is None else (out,):
        t.record_stream(torch.cuda.current_stream(device))
    return out


# ------------------------------------------------------------------ the cache
class KVCache:
    """A paged key-value cache: rows of head_dim values in [pages, kv_heads,
    page_size, row] tensors k and v.

      16 bits  float16 or bfloat16 rows of head_dim values
      8 bits   float8_e4m3fn rows of head_dim codes
      4 bits   int32 rows of head_dim / 8 TQ4 words (the package's 4-bit quantizer)

    The last two with one float16 scale per row, [pages, kv_heads, page_size], in
    k_scales and v_scales.  head_dim 64, 128 or 256; page_size a power of two of at
    least 16.  Slot number = page * page_size + place in the page.  The object holds
    the tensors and no state: which slots are in use is the program's to know."""

    __slots__ = ("_t", "_c", "_sizes")

    def __init__(self, k, v, k_scales=None, v_scales=None):
        self._c, *self._sizes = (_native or _load()).make_cache(k, v, k_scales, v_scales)
        self._t = (k, v, k_scales, v_scales)

    k = property(lambda self: self._t[0])
    v = property(lambda self: self._t[1])
    k_scales = property(lambda self: self._t[2])
    v_scales = property(lambda self: self._t[3])
    pages = property(lambda self: self._sizes[0])
    page_size = property(lambda self: self._sizes[1])
    kv_heads = property(lambda self: self._sizes[2])
    head_dim = property(lambda self: self._sizes[3])
    bits = property(lambda self: self._sizes[4])
    device = property(lambda self: self._t[0].device)


def _handle(cache):
    if not isinstance(cache, KVCache):
        raise TypeError(f"cache: expected a KVCache, got {type(cache).__name__}")
    return cache._c


def empty_kv_cache(pages: int, page_size: int, kv_heads: int, head_dim: int, bits: int = 16,
                   dtype=None, device="cuda") -> KVCache:
    """A cache of uninitialised rows; dtype (16 bits): float16 (default) or bfloat16."""
    import torch
    if bits not in (16, 8, 4):
        raise ValueError(f"bits {bits}: 16, 8 or 4 are supported")
    if head_dim not in (64, 128, 256):
        raise ValueError(f"head_dim {head_dim}: 64, 128 or 256 are supported")
    if bits != 16 and dtype is not None:
        raise ValueError("dtype: only rows of 16 bits have one")
    if dtype not in (None, torch.float16, torch.bfloat16):
        raise TypeError(f"dtype {dtype}: torch.float16 or torch.bfloat16")
    kind = {16: dtype or torch.float16, 8: torch.float8_e4m3fn, 4: torch.int32}[bits]
    shape = (pages, kv_heads, page_size)
    new = lambda s, t: torch.empty(s, dtype=t, device=device)
    k, v = (new((*shape, head_dim // 8 if bits == 4 else head_dim), kind) for _ in range(2))
    return KVCache(k, v, *((None, None) if bits == 16 else (new(shape, torch.float16) for _ in range(2))))


def rope_table(max_positions: int, rotary_dim: int, base: float = 10000.0, device="cuda"):
    """The table [max_positions, rotary_dim] float32 of the plain rotation: cosines,
    then sines, of position * base^(-2 i / rotary_dim).  A model with scaled
    frequencies brings a table of its own."""
    import torch
    freq = base ** (-torch.arange(0, rotary_dim, 2, dtype=torch.float64) / rotary_dim)
    angle = torch.arange(max_positions, dtype=torch.float64)[:, None] * freq
    return torch.cat((angle.cos(), angle.sin()), 1).float().to(device)


# ------------------------------------------------------------------ the operators
def kv_append(cache: KVCache, k, v, slots, stream=None) -> None:
    """k and v [tokens, kv_heads, head_dim] into the cache at slots [tokens] int64,
    quantized where it has 8 or 4 bits (tq_kv_append).  A token whose slot is
    negative or past the cache is not written; slots of one call are distinct (rows
    written twice are a mixture of both)."""
    c = _handle(cache)
    call = lambda dev, st: _native.append(c, k, v, slots, dev, st)
    if stream is not None:
        return _elsewhere(stream, (k, v, slots, *cache._t), call)
    call(*_here())


def kv_read(cache: KVCache, slots, bf16: bool | None = None, stream=None):
    """(k, v) [tokens, kv_heads, head_dim] of slots [tokens] int64 (tq_kv_read); zeros
    for a slot outside the cache.  bf16: bfloat16 instead of float16 values from a
    cache of 8 or 4 bits (a 16-bit cache gives its own type)."""
    c = _handle(cache)
    if stream is not None:
        return _elsewhere(stream, (slots, *cache._t), lambda dev, st: _native.read(c, slots, bf16, dev, st))
    return _native.read(c, slots, bf16, *_here())


def qk_norm_rope(q, k, positions, table, q_weight=None, k_weight=None, eps: float = 1e-6,
                 interleaved: bool = False, stream=None):
    """(q, k) [tokens, heads, head_dim] with each head normed (RMS, weight [head_dim]
    of q's type; None: no norm) and rotated by its token's position (positions
    [tokens] int32, table [max_positions, rotary_dim] float32 as ``rope_table`` makes;
    None: no rotation), in fp32, rounded once (tq_qk_norm_rope).  q and k may be
    views of a fused projection's output."""
    native = _native or _load()
    if stream is not None:
        return _elsewhere(stream, (q, k, positions, table, q_weight, k_weight), lambda dev, st: native.norm_rope(
            q, k, positions, table, q_weight, k_weight, eps, interleaved, dev, st))
    return native.norm_rope(q, k, positions, table, q_weight, k_weight, eps, interleaved, *_here())


def qk_norm_rope_append(cache: KVCache, q, k, v, positions, table, slots, q_weight=None, k_weight=None,
                        eps: float = 1e-6, interleaved: bool = False, return_k: bool = False, stream=None):
    """``qk_norm_rope`` and ``kv_append`` in one launch (tq_qk_norm_rope_append): the
    rotated q back, the rotated k and v into the cache at slots [tokens] int64.  With
    return_k (q, k), the k as it was before the cache's quantizer."""
    c = _handle(cache)
    if stream is not None:
        return _elsewhere(stream, (q, k, v, slots, positions, table, q_weight, k_weight, *cache._t),
                          lambda dev, st: _native.norm_rope_append(
                              c, q, k, v, slots, positions, table, q_weight, k_weight, eps, interleaved, return_k,
                              dev, st))
    return _native.norm_rope_append(c, q, k, v, slots, positions, table, q_weight, k_weight, eps, interleaved,
                                    return_k, *_here())


def paged_attention(cache: KVCache, q, page_table, lengths, scale: float | None = None, window: int = 0,
                    return_lse: bool = False, stream=None):
    """Attention of one new token of every stream over the cache (tq_paged_attention):
    q [batch, q_heads, head_dim], page_table [batch, max_pages] int32 (rows may be
    strided), lengths [batch] int32 the tokens of each stream, its newest one among
    them.  window > 0: only the last so many.  scale: head_dim^-1/2 by default.
    Returns out [batch, q_heads, head_dim] of q's type, zeros for a stream of length
    0; with return_lse (out, lse [batch, q_heads] float32)."""
    c = _handle(cache)
    if stream is not None:
        return _elsewhere(stream, (q, page_table, lengths, *cache._t), lambda dev, st: _native.attend(
            c, q, page_table, lengths, scale, window, return_lse, dev, st))
    return _native.attend(c, q, page_table, lengths, scale, window, return_lse, *_here())
