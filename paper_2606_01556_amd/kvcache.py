"""The operators between a decoder block's linear layers, for inference: norm and
position rotation of queries and keys, the paged key-value cache in 16, 8 or 4
bits, and the attention of one new token over it.

Binding of the ``tq_kv_*``, ``tq_qk_*`` and ``tq_paged_attention`` entry points of
``libtq.so``; the arithmetic runs in the library's HIP kernels.  As in the rest of
the package, every tensor is checked before the call (the library sees pointers),
nothing is synchronized, and ``stream`` (a torch stream or a hipStream_t; default:
the current one) has to have the inputs ready.

A decode step of one block:

    cache = tq.empty_kv_cache(pages, 16, kv_heads, 128, bits=4)
    ...
    q = tq.qk_norm_rope_append(cache, q, k, v, positions, table, slots, q_weight, k_weight)
    y = tq.paged_attention(cache, q, page_table, lengths)
"""
from __future__ import annotations

import contextlib
import ctypes
import functools

from . import TQ_BF16, TQ_F16, _check, _other_stream, _stream, lib

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


# ------------------------------------------------------------------ argument checks
# The usual tensor passes a chain of tests (about 0.3 us); where one fails, a second
# look says which.  get_device() is -1 for a host tensor.
def _refuse(t, name, dtypes, device):
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{name}: must be a GPU tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if t.get_device() != device:
        raise ValueError(f"{name}: on device {t.get_device()}, the others are on {device}")


def _plain(t, name, dtype, shape, device):
    """The address of a contiguous tensor of one type and shape."""
    if not (isinstance(t, _torch().Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == device
            and t.is_contiguous()):
        _refuse(t, name, (dtype,), device)
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
        raise ValueError(f"{name}: must be contiguous")
    return t.data_ptr()


def _rows(t, name, dtypes, device, tokens, heads, head_dim):
    """The tq_head_rows of t [tokens, heads, head_dim] (None: any number)."""
    if not (isinstance(t, _torch().Tensor) and t.dtype in dtypes and t.get_device() == device):
        _refuse(t, name, dtypes, device)
    shape = t.shape
    if len(shape) != 3 or not (tokens is None or shape[0] == tokens) or not (
            heads is None or shape[1] == heads) or shape[2] != head_dim:
        want = ", ".join(n if v is None else str(v) for n, v in (("tokens", tokens), ("heads", heads),
                                                                 ("head_dim", head_dim)))
        raise ValueError(f"{name}: shape {tuple(shape)}, expected [{want}]")
    ts, hs, ds = t.stride()
    if shape[0] <= 1:
        ts = 0
    if shape[1] <= 1:
        hs = 0
    p = t.data_ptr()
    if ds != 1 or (ts | hs) & 7 or p & 15:
        raise ValueError(f"{name}: rows must be contiguous and start on 16 bytes (strides {tuple(t.stride())}, "
                         f"address {p:#x}); pass {name}.contiguous()")
    return _HeadRows(p, ts, hs)


def _on_device(device, name):
    here = _torch()._C._cuda_getDevice()
    if device != here:
        raise ValueError(f"{name}: on device {device}, but the current device is {here}")


def _other(stream, st, device, inputs):
    """`stream` as a torch stream where it is not the current one, else None; the
    inputs then stay until that stream is done with them."""
    torch = _torch()
    other = _other_stream(stream, st, torch.device("cuda", device))
    if other is not None:
        for t in inputs:
            if t is not None:
                t.record_stream(other)
    return other


def _new(stream, st, device, inputs, like, *shapes):
    """Tensors like `like` of the given shapes (a number: so many float32), from the
    memory of the stream that the work runs on; on a stream other than the current
    one they may be used and dropped on the current one."""
    torch = _torch()
    new = (like if type(like) is torch.Tensor else like.as_subclass(torch.Tensor)).new_empty
    if stream is not None and (other := _other(stream, st, device, inputs)) is not None:
        with torch.cuda.stream(other):
            out = [new(s) if type(s) is tuple else new(s, dtype=torch.float32) for s in shapes]
        here = torch.cuda.current_stream(device)
        for t in out:
            t.record_stream(here)
        return out
    return [new(s) if type(s) is tuple else new(s, dtype=torch.float32) for s in shapes]


@functools.lru_cache(maxsize=None)
def _torch():
    import torch
    return torch


@functools.lru_cache(maxsize=None)
def _types():
    import torch
    return torch.float16, torch.bfloat16


def _at(stream, device):
    """The hipStream_t of `stream`, by default the current one."""
    return _torch()._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)


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

    __slots__ = ("_t", "_c", "_dtypes", "pages", "page_size", "kv_heads", "head_dim", "bits", "device")

    def __init__(self, k, v, k_scales=None, v_scales=None):
        torch = _torch()
        f16, bf16 = _types()
        kinds = (f16, bf16, torch.float8_e4m3fn, torch.int32)
        if not (isinstance(k, torch.Tensor) and k.is_cuda and k.dtype in kinds):
            _refuse(k, "k", kinds, None)
        if k.dim() != 4:
            raise ValueError(f"k: shape {tuple(k.shape)}, expected [pages, kv_heads, page_size, row]")
        shape, dev = k.shape, k.get_device()
        bits = 8 if k.dtype is torch.float8_e4m3fn else 4 if k.dtype is torch.int32 else 16
        kp, vp = _plain(k, "k", k.dtype, shape, dev), _plain(v, "v", k.dtype, shape, dev)
        ks = vs = None
        if bits < 16:
            if k_scales is None or v_scales is None:
                raise ValueError(f"k_scales, v_scales: a {bits}-bit cache needs both")
            ks = _plain(k_scales, "k_scales", f16, shape[:3], dev)
            vs = _plain(v_scales, "v_scales", f16, shape[:3], dev)
        elif k_scales is not None or v_scales is not None:
            raise ValueError("k_scales, v_scales: a 16-bit cache has none")
        pages, heads, size, row = shape
        d = row * 8 if bits == 4 else row
        if d not in (64, 128, 256):
            raise ValueError(f"k: rows of {d} values; 64, 128 or 256 are supported")
        if not 16 <= size <= 32768 or size & (size - 1):
            raise ValueError(f"k: page size {size}; a power of two from 16 to 32768 is supported")
        if not 1 <= heads <= 1024 or pages < 1:
            raise ValueError(f"k: {pages} pages of {heads} heads")
        self._t = (k, v, k_scales, v_scales)
        self._c = _CacheDesc(pages, size, heads, d, bits, TQ_BF16 if k.dtype is bf16 else TQ_F16, kp, vp, ks, vs)
        self.pages, self.page_size, self.kv_heads, self.head_dim = pages, size, heads, d
        self.bits, self.device = bits, dev
        self._dtypes = (k.dtype,) if bits == 16 else _types()    # of rows written, read or asked with

    k = property(lambda self: self._t[0])
    v = property(lambda self: self._t[1])
    k_scales = property(lambda self: self._t[2])
    v_scales = property(lambda self: self._t[3])


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
    if dtype not in (None, *_types()):
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


def _is_cache(cache):
    if not isinstance(cache, KVCache):
        raise TypeError(f"cache: expected a KVCache, got {type(cache).__name__}")
    _on_device(cache.device, "cache")
    return cache._c


def _slots(slots, device, tokens=None):
    torch = _torch()
    if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
        raise ValueError("slots: expected an int64 tensor [tokens]")
    return _plain(slots, "slots", torch.int64, slots.shape if tokens is None else (tokens,), device)


def kv_append(cache: KVCache, k, v, slots, stream=None) -> None:
    """k and v [tokens, kv_heads, head_dim] into the cache at slots [tokens] int64,
    quantized where it has 8 or 4 bits (tq_kv_append).  A token whose slot is
    negative is not written; slots of one call are distinct."""
    c = _is_cache(cache)
    dev, heads, d = cache.device, cache.kv_heads, cache.head_dim
    kr = _rows(k, "k", cache._dtypes, dev, None, heads, d)
    tokens, dtype = k.shape[0], k.dtype
    vr = _rows(v, "v", (dtype,), dev, tokens, heads, d)
    sp = _slots(slots, dev, tokens)
    if tokens == 0:
        return
    st = _at(stream, dev)
    if stream is not None:
        _other(stream, st, dev, (k, v, slots))
    _check(lib().tq_kv_append(c, kr, vr, sp, tokens, TQ_F16 if dtype is _types()[0] else TQ_BF16, st),
           "tq_kv_append")


def kv_read(cache: KVCache, slots, bf16: bool | None = None, stream=None):
    """(k, v) [tokens, kv_heads, head_dim] of slots [tokens] int64 (tq_kv_read); zeros
    for a slot outside the cache.  bf16: bfloat16 instead of float16 values from a
    cache of 8 or 4 bits (a 16-bit cache gives its own type)."""
    c = _is_cache(cache)
    dev = cache.device
    sp = _slots(slots, dev)
    tokens = slots.shape[0]
    if cache.bits == 16:
        dtype = cache.k.dtype
        if bf16 is not None and bool(bf16) != (dtype is _types()[1]):
            raise TypeError(f"bf16: the cache holds {dtype}")
    else:
        dtype = _types()[bool(bf16)]
    st = _at(stream, dev)
    torch = _torch()
    other = None if stream is None else _other(stream, st, dev, (slots,))
    with torch.cuda.stream(other) if other is not None else _NO_STREAM:
        k, v = torch.empty((2, tokens, cache.kv_heads, cache.head_dim), dtype=dtype, device=dev).unbind()
    if other is not None:
        k.record_stream(torch.cuda.current_stream(dev))      # (v is in the same memory)
    if tokens:
        _check(lib().tq_kv_read(c, sp, tokens, k.data_ptr(), v.data_ptr(),
                                TQ_F16 if dtype is _types()[0] else TQ_BF16, st), "tq_kv_read")
    return k, v


_NO_STREAM = contextlib.nullcontext()


def _norm_rope(positions, table, q_weight, k_weight, eps, interleaved, tokens, head_dim, dtype, dev):
    torch = _torch()
    shape = (head_dim,)
    qw = None if q_weight is None else _plain(q_weight, "q_weight", dtype, shape, dev)
    kw = None if k_weight is None else _plain(k_weight, "k_weight", dtype, shape, dev)
    if table is None:
        return _NormRope(qw, kw, None, None, 0, 0, 0, eps)
    if not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("table: expected a float32 tensor [max_positions, rotary_dim]")
    shape = table.shape
    tp = _plain(table, "table", torch.float32, shape, dev)
    n, rot = shape
    if not 0 < rot <= head_dim or rot % 16 or n < 1:
        raise ValueError(f"table: {n} positions of {rot} values; a multiple of 16 up to head_dim {head_dim}")
    if positions is None:
        raise ValueError("positions: a rotation needs them")
    pp = _plain(positions, "positions", torch.int32, (tokens,), dev)
    return _NormRope(qw, kw, pp, tp, rot, n, bool(interleaved), eps)


def qk_norm_rope(q, k, positions, table, q_weight=None, k_weight=None, eps: float = 1e-6,
                 interleaved: bool = False, stream=None):
    """(q, k) [tokens, heads, head_dim] with each head normed (RMS, weight [head_dim]
    of q's type; None: no norm) and rotated by its token's position (positions
    [tokens] int32, table [max_positions, rotary_dim] float32 as ``rope_table`` makes;
    None: no rotation), in fp32, rounded once (tq_qk_norm_rope).  q and k may be
    views of a fused projection's output."""
    types = _types()
    if not (isinstance(q, _torch().Tensor) and q.is_cuda and q.dtype in types):
        _refuse(q, "q", types, None)
    dev, dtype, shape = q.get_device(), q.dtype, q.shape
    _on_device(dev, "q")
    if len(shape) != 3 or shape[2] not in (64, 128, 256):
        raise ValueError(f"q: shape {tuple(shape)}; [tokens, heads, head_dim] with head_dim 64, 128 or 256")
    tokens, hq, d = shape
    qr = _rows(q, "q", types, dev, tokens, hq, d)
    kr = _rows(k, "k", (dtype,), dev, tokens, None, d)
    hkv = k.shape[1]
    p = _norm_rope(positions, table, q_weight, k_weight, eps, interleaved, tokens, d, dtype, dev)
    st = _at(stream, dev)
    qo, ko = _new(stream, st, dev, (q, k, positions, table, q_weight, k_weight), q, (tokens, hq, d), (tokens, hkv, d))
    if tokens:
        _check(lib().tq_qk_norm_rope(p, qr, kr, tokens, hq, hkv, d, TQ_F16 if dtype is types[0] else TQ_BF16,
                                     qo.data_ptr(), ko.data_ptr(), st), "tq_qk_norm_rope")
    return qo, ko


def qk_norm_rope_append(cache: KVCache, q, k, v, positions, table, slots, q_weight=None, k_weight=None,
                        eps: float = 1e-6, interleaved: bool = False, return_k: bool = False, stream=None):
    """``qk_norm_rope`` and ``kv_append`` in one launch (tq_qk_norm_rope_append): the
    rotated q back, the rotated k and v into the cache at slots [tokens] int64.  With
    return_k (q, k), the k as it was before the cache's quantizer."""
    c = _is_cache(cache)
    dev, d, hkv = cache.device, cache.head_dim, cache.kv_heads
    qr = _rows(q, "q", cache._dtypes, dev, None, None, d)
    tokens, hq, _ = q.shape
    dtype = q.dtype
    kr = _rows(k, "k", (dtype,), dev, tokens, hkv, d)
    vr = _rows(v, "v", (dtype,), dev, tokens, hkv, d)
    sp = _slots(slots, dev, tokens)
    p = _norm_rope(positions, table, q_weight, k_weight, eps, interleaved, tokens, d, dtype, dev)
    st = _at(stream, dev)
    inputs = (q, k, v, positions, table, slots, q_weight, k_weight)
    if return_k:
        qo, ko = _new(stream, st, dev, inputs, q, (tokens, hq, d), (tokens, hkv, d))
    else:
        (qo,), ko = _new(stream, st, dev, inputs, q, (tokens, hq, d)), None
    if tokens:
        _check(lib().tq_qk_norm_rope_append(p, c, qr, kr, vr, sp, tokens, hq,
                                            TQ_F16 if dtype is _types()[0] else TQ_BF16, qo.data_ptr(),
                                            None if ko is None else ko.data_ptr(), st),
               "tq_qk_norm_rope_append")
    return (qo, ko) if return_k else qo


def paged_attention(cache: KVCache, q, page_table, lengths, scale: float | None = None, window: int = 0,
                    return_lse: bool = False, stream=None):
    """Attention of one new token of every stream over the cache (tq_paged_attention):
    q [batch, q_heads, head_dim], page_table [batch, max_pages] int32 (rows may be
    strided), lengths [batch] int32 the tokens of each stream, its newest one among
    them.  window > 0: only the last so many.  scale: head_dim^-1/2 by default.
    Returns out [batch, q_heads, head_dim] of q's type, zeros for a stream of length
    0; with return_lse (out, lse [batch, q_heads] float32)."""
    c = _is_cache(cache)
    torch = _torch()
    dev, d = cache.device, cache.head_dim
    qr = _rows(q, "q", cache._dtypes, dev, None, None, d)
    batch, hq, _ = q.shape
    if hq == 0 or hq % cache.kv_heads:
        raise ValueError(f"q: {hq} heads are no multiple of the cache's {cache.kv_heads}")
    if not (isinstance(page_table, torch.Tensor) and page_table.dtype is torch.int32 and page_table.get_device() == dev):
        _refuse(page_table, "page_table", (torch.int32,), dev)
    shape = page_table.shape
    if len(shape) != 2 or shape[0] != batch or shape[1] == 0:
        raise ValueError(f"page_table: shape {tuple(shape)}, expected [{batch}, max_pages]")
    pages = shape[1]
    stride, step = page_table.stride()
    if (step != 1 and pages > 1) or (stride < pages and batch > 1):
        raise ValueError("page_table: rows must be contiguous")
    lp = _plain(lengths, "lengths", torch.int32, (batch,), dev)
    if window < 0:
        raise ValueError(f"window {window}: must not be negative")
    if scale is None:
        scale = d ** -0.5
    st = _at(stream, dev)
    L = lib()
    nscratch = L.tq_paged_attention_scratch_bytes(c, batch, hq, pages, window)
    shapes = [(batch, hq, d)]
    if nscratch:
        shapes.append(nscratch // 4)
    if return_lse:
        shapes.append(batch * hq)
    out = _new(stream, st, dev, (q, page_table, lengths), q, *shapes)
    y = out[0]
    lse = out[-1].view(batch, hq) if return_lse else None
    if batch:
        _check(L.tq_paged_attention(c, qr, TQ_F16 if q.dtype is _types()[0] else TQ_BF16, batch, hq,
                                    page_table.data_ptr(), stride, pages, lp, scale, window, y.data_ptr(),
                                    None if lse is None else lse.data_ptr(),
                                    out[1].data_ptr() if nscratch else None, st), "tq_paged_attention")
    return (y, lse) if return_lse else y
