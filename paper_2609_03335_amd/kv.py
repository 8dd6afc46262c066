"""The paged 4-bit key/value cache of a replica: binding of include/wf_kv.h
(same names) and helpers that allocate the outputs.  Only marshalling: every
step runs in the gfx950 kernels.

The helpers take sound tensors through _kvbind (csrc/kv_bind.cpp), which checks, allocates and calls
in one step: a step of 64 rows takes 8.4 us, 14 through ctypes.  What it
does not take at once (addresses, other strides, wrong arguments) goes through
KVContext's methods, which accept it or say what is wrong.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

from ._lib import WF_OK, WFError, _buf, _stream, load, wf_kv_desc, wf_kv_norm_rope

WF_KV_BF16, WF_KV_F16 = 0, 1
_TYPES = {"bf16": WF_KV_BF16, "f16": WF_KV_F16}


def _desc(q_heads, kv_heads, head_dim, block_tokens, n_blocks, max_blocks, dtype) -> wf_kv_desc:
    return wf_kv_desc(q_heads, kv_heads, head_dim, block_tokens, n_blocks, max_blocks, _TYPES.get(dtype, dtype))


def wf_kv_cache_bytes(q_heads: int, kv_heads: int, head_dim: int, block_tokens: int, n_blocks: int,
                      max_blocks: int = 1, dtype="bf16") -> int:
    """Bytes of one layer's cache (host only)."""
    lib, out = load(), ctypes.c_int64()
    d = _desc(q_heads, kv_heads, head_dim, block_tokens, n_blocks, max_blocks, dtype)
    st = lib.wf_kv_cache_bytes(ctypes.byref(d), ctypes.byref(out))
    if st != WF_OK:
        raise WFError(st, lib.wf_kv_last_error(None).decode())
    return out.value


class KVContext:
    """A wf_kv_ctx on one HIP device: the geometry of a cache.  Tensor
    arguments are checked before any call reaches the library (GPU tensor, the
    context's device, enough bytes, type or size of the elements, length of the rows
    of block tables and rotations).

    Calls on several streams may overlap, on tensors of their own: kv_attend has a work area for each of the
    first 8 streams it is called on, and does without on others (long rows of few queries then take
    longer).  A captured call keeps the area of the stream of its capture, so replays of graphs captured on one
    stream must not overlap.  One thread at a time may use a context."""

    def __init__(self, device: int = 0, *, q_heads: int, kv_heads: int, head_dim: int, block_tokens: int,
                 n_blocks: int, max_blocks: int, dtype="bf16"):
        self.lib = load()
        self.handle = None
        d = _desc(q_heads, kv_heads, head_dim, block_tokens, n_blocks, max_blocks, dtype)
        h = ctypes.c_void_p()
        st = self.lib.wf_kv_ctx_create(device, ctypes.byref(d), ctypes.byref(h))
        if st != WF_OK:
            raise WFError(st, self.lib.wf_kv_last_error(None).decode())
        self.handle = h
        self.device = device
        self.q_heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.block_tokens, self.n_blocks, self.max_blocks = block_tokens, n_blocks, max_blocks
        self.dtype, self.torch_dtype = d.dtype, torch_type(d.dtype)
        self._current = _current_stream()
        self._bind = _bind() if self._current is not None else None
        self.cache_bytes = n_blocks * kv_heads * block_tokens * (head_dim + 4)
        if self._bind is not None:
            self._geometry = self._bind.geometry(h.value, device, q_heads, kv_heads, head_dim, n_blocks, max_blocks,
                                                 self.cache_bytes, d.dtype == WF_KV_F16)

    def _check(self, st):
        if st != WF_OK:
            raise WFError(st, self.lib.wf_kv_last_error(self.handle).decode())

    def _b(self, x, need: int, name: str, size: int = 4, floating: bool = False) -> Optional[int]:
        """Address of a buffer of `size`-byte whole numbers (or floating ones); an int is an address
        the caller vouches for.  (A sound tensor passes in 0.4 us; an exception
        on the way to an int would cost twice that.)"""
        if x is None or x.__class__ is int:
            return x
        try:
            if (x.get_device() == self.device and x.nbytes >= need and x.element_size() == size and
                    x.is_contiguous() and x.is_floating_point() == floating):
                return x.data_ptr()
        except AttributeError:
            pass
        if hasattr(x, "element_size") and x.element_size() != size:
            raise TypeError(f"{name}: elements of {x.element_size()} bytes, {size} needed")
        address = _buf(x, max(int(need), 0), self.device, name)
        if hasattr(x, "is_floating_point") and x.is_floating_point() != floating:
            raise TypeError(f"{name}: elements of type {x.dtype}")
        return address

    def _rows(self, x, pitch: int, need: int, name: str, floating: bool = False) -> Optional[int]:
        """A buffer of 4-byte elements whose rows, where it has several axes, are `pitch` elements apart."""
        address = self._b(x, need, name, 4, floating)
        if getattr(x, "ndim", 0) > 1 and x.numel() != x.shape[0] * pitch:
            raise ValueError(f"{name}: shape {tuple(x.shape)}, rows of {pitch} elements needed")
        return address

    def _wide(self, x, need: int, name: str) -> Optional[int]:
        """A buffer of the context's 16-bit type."""
        if x is None or x.__class__ is int:
            return x
        self._type(x, name)
        return self._b(x, need, name, 2, True)

    def _type(self, x, name: str) -> None:
        if getattr(x, "dtype", None) is not self.torch_dtype:
            raise TypeError(f"{name}: {getattr(x, 'dtype', type(x))}, the context takes {self.torch_dtype}")

    def _tokens(self, x, n: int, heads: int, name: str, stride: Optional[int] = None):
        """(address, token stride) of n tokens of heads: a tensor [n, heads, D]
        or [n, heads * D] whose heads are contiguous, or a raw address with
        its stride (default: dense)."""
        width = heads * self.head_dim
        if x is None or x.__class__ is int:
            return x, width if stride is None else int(stride)
        self._type(x, name)
        if x.get_device() != self.device:
            raise ValueError(f"{name}: tensor on {x.device}, context on cuda:{self.device}"
                             if x.is_cuda else f"{name}: a host tensor cannot be passed to the GPU library")
        shape, st = x.shape, x.stride()
        if shape == (n, heads, self.head_dim) and st[1:] == (self.head_dim, 1):
            return x.data_ptr(), st[0] if n > 1 else width
        if len(shape) == 3:
            dense = (shape[1] == heads and shape[2] == self.head_dim and st[2] == 1 and
                     (st[1] == self.head_dim or heads == 1))
        else:
            dense = len(shape) == 2 and shape[1] == width and st[1] == 1
        if not dense or shape[0] < n:
            raise ValueError(f"{name}: shape {tuple(shape)} and strides {st}; [{n}, {heads}, {self.head_dim}] with "
                             "contiguous heads needed")
        return x.data_ptr(), st[0] if n > 1 else width

    def _s(self, stream) -> Optional[int]:
        """The stream's handle; by default the current stream of the context's device."""
        if stream is None and self._current is not None:
            return self._current(self.device) or None
        return _stream(stream)

    def wf_kv_step(self, new_tokens, n_rows: int, n_tokens: int, len_in, len_out, pool_in, pool_out, ring, table,
                   q_off, slot, pos, granted, stream=None) -> None:
        b, r, t = self._b, max(int(n_rows), 0), max(int(n_tokens), 0)
        self._check(self.lib.wf_kv_step(
            self.handle, b(new_tokens, 4 * r, "new_tokens"), int(n_rows), int(n_tokens), b(len_in, 4 * r, "len_in"),
            b(len_out, 4 * r, "len_out"), b(pool_in, 8, "pool_in"), b(pool_out, 8, "pool_out"),
            b(ring, 4 * self.n_blocks, "ring"), self._rows(table, self.max_blocks, 4 * r * self.max_blocks, "table"),
            b(q_off, 4 * r + 4, "q_off"), b(slot, 8 * t, "slot", 8), b(pos, 4 * t, "pos"), b(granted, r, "granted", 1),
            self._s(stream)))

    def wf_kv_store(self, q, k, v, n_tokens: int, pos, slot, q_out, cache, *, cos_sin=None, n_pos: int = 0,
                    rot_dim: int = 0, interleaved: bool = False, q_weight=None, k_weight=None, eps: float = 1e-6,
                    strides=(None, None, None), stream=None) -> None:
        n, d = max(int(n_tokens), 0), self.head_dim
        (qp, qs), (kp, ks), (vp, vs) = (self._tokens(q, n, self.q_heads, "q", strides[0]),
                                        self._tokens(k, n, self.kv_heads, "k", strides[1]),
                                        self._tokens(v, n, self.kv_heads, "v", strides[2]))
        need = 4 * n_pos * rot_dim
        if 0 < rot_dim <= d and rot_dim % 16 == 0 and n_pos > 0 and pos is not None:
            angles = self._rows(cos_sin, rot_dim, need, "cos_sin", True)
        else:                                   # not read, or the library says what is wrong
            angles = self._b(cos_sin, need, "cos_sin", 4, True)
        how = wf_kv_norm_rope(self._wide(q_weight, 2 * d, "q_weight"), self._wide(k_weight, 2 * d, "k_weight"), eps,
                              rot_dim, int(interleaved), n_pos, angles)
        self._check(self.lib.wf_kv_store(
            self.handle, qp, kp, vp, qs, ks, vs, int(n_tokens), ctypes.byref(how), self._b(pos, 4 * n, "pos"),
            self._b(slot, 8 * n, "slot", 8), self._wide(q_out, 2 * n * self.q_heads * d, "q_out"),
            self._b(cache, self.cache_bytes, "cache", 1), self._s(stream)))

    def wf_kv_load(self, cache, slot, n_tokens: int, k_out, v_out, stream=None) -> None:
        n = max(int(n_tokens), 0)
        need = 2 * n * self.kv_heads * self.head_dim
        self._check(self.lib.wf_kv_load(
            self.handle, self._b(cache, self.cache_bytes, "cache", 1), self._b(slot, 8 * n, "slot", 8), int(n_tokens),
            self._wide(k_out, need, "k_out"), self._wide(v_out, need, "v_out"), self._s(stream)))

    def wf_kv_attend(self, q, n_tokens: int, cache, table, kv_len, q_off, pos, n_rows: int, scale: float, out, *,
                     window: int = 0, max_q: int = 0, max_kv: int = 0, q_stride=None, stream=None) -> None:
        n, r, b = max(int(n_tokens), 0), max(int(n_rows), 0), self._b
        qp, qs = self._tokens(q, n, self.q_heads, "q", q_stride)
        self._check(self.lib.wf_kv_attend(
            self.handle, qp, qs, int(n_tokens), b(cache, self.cache_bytes, "cache", 1),
            self._rows(table, self.max_blocks, 4 * r * self.max_blocks, "table"), b(kv_len, 4 * r, "kv_len"), b(q_off, 4 * r + 4, "q_off"),
            b(pos, 4 * n, "pos"), int(n_rows), float(scale), int(window), int(max_q), int(max_kv),
            self._wide(out, 2 * n * self.q_heads * self.head_dim, "out"), self._s(stream)))

    def close(self):
        self._bind = None
        if getattr(self, "handle", None):
            self.lib.wf_kv_ctx_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


@functools.lru_cache(maxsize=None)
def _bind():
    """The module _kvbind with the library's calls, None where it was not built."""
    import torch  # noqa: F401  (its libraries are _kvbind's)
    try:
        from . import _kvbind
    except ImportError:
        return None
    lib = load()
    _kvbind.calls(*(ctypes.cast(f, ctypes.c_void_p).value
                    for f in (lib.wf_kv_step, lib.wf_kv_store, lib.wf_kv_load, lib.wf_kv_attend)))
    return _kvbind


def _current_stream():
    """Device index -> handle of torch's current stream there, without building
    a Stream object (2.9 us a call); None where this torch has no such call."""
    import torch
    return getattr(torch._C, "_cuda_getCurrentRawStream", None)


@functools.lru_cache(maxsize=None)
def torch_type(dtype: int):
    import torch
    return torch.bfloat16 if dtype == WF_KV_BF16 else torch.float16


def _made_current(ctx: KVContext, stream):
    """Makes a stream (torch's, or a handle) torch's current one, so that outputs are
    allocated for it: their memory is not given to another stream's work while this one's runs."""
    import torch
    if isinstance(stream, int):
        at = torch.device("cuda", ctx.device)
        stream = torch.cuda.ExternalStream(stream, device=at) if stream else torch.cuda.default_stream(at)
    return torch.cuda.stream(stream)


def kv_step(ctx: KVContext, new_tokens, n_tokens: int, lens, pool, ring, table, stream=None):
    """Allocate the outputs of wf_kv_step and enqueue it.  table and ring are
    updated in place; returns (lens, pool, q_off, slot, pos, granted).  Here and below,
    `stream` (a torch stream or a handle; default: the current one) takes the work and
    owns the outputs."""
    if stream is not None:
        with _made_current(ctx, stream):
            return kv_step(ctx, new_tokens, n_tokens, lens, pool, ring, table)
    if ctx._bind is not None:
        out = ctx._bind.step(ctx._geometry, ctx._current(ctx.device), new_tokens, n_tokens, lens, pool, ring, table)
        if out is not None:
            if out.__class__ is int:
                ctx._check(out)
            return out
    import torch
    r, empty = new_tokens.shape[0], new_tokens.new_empty
    # one allocation for the int32 outputs: lens, pool, q_off, pos
    flat = empty(2 * r + 3 + n_tokens, dtype=torch.int32)
    slot = empty(n_tokens, dtype=torch.int64)
    granted = empty(r, dtype=torch.uint8)
    at = flat.data_ptr()
    ctx.wf_kv_step(new_tokens, r, n_tokens, lens, at, pool, at + 4 * r, ring, table, at + 4 * r + 8, slot.data_ptr(),
                   at + 8 * r + 12, granted.data_ptr())
    lens_out, pool_out, q_off, pos = flat.split((r, 2, r + 1, n_tokens))
    return lens_out, pool_out, q_off, slot, pos, granted


def kv_store(ctx: KVContext, q, k, v, pos, slot, cache, cos_sin=None, *, rot_dim: int = 0, interleaved: bool = False,
             q_weight=None, k_weight=None, eps: float = 1e-6, stream=None):
    """Norm, rotate and store the tokens of q [T, q_heads, D], k and v [T,
    kv_heads, D]; returns the queries [T, q_heads, D]."""
    if stream is not None:
        with _made_current(ctx, stream):
            return kv_store(ctx, q, k, v, pos, slot, cache, cos_sin, rot_dim=rot_dim, interleaved=interleaved,
                            q_weight=q_weight, k_weight=k_weight, eps=eps)
    if ctx._bind is not None:
        out = ctx._bind.store(ctx._geometry, ctx._current(ctx.device), q, k, v, pos, slot, cache, cos_sin, rot_dim,
                              interleaved, q_weight, k_weight, eps)
        if out is not None:
            if out.__class__ is int:
                ctx._check(out)
            return out
    n = q.shape[0]
    out = q.new_empty((n, ctx.q_heads, ctx.head_dim))
    ctx.wf_kv_store(q, k, v, n, pos, slot, out.data_ptr(), cache, cos_sin=cos_sin,
                    n_pos=0 if cos_sin is None else cos_sin.shape[0], rot_dim=rot_dim, interleaved=interleaved,
                    q_weight=q_weight, k_weight=k_weight, eps=eps)
    return out


def kv_load(ctx: KVContext, cache, slot, stream=None):
    """The cached keys and values [T, kv_heads, D] at the given slots."""
    if stream is not None:
        with _made_current(ctx, stream):
            return kv_load(ctx, cache, slot)
    if ctx._bind is not None:
        out = ctx._bind.load(ctx._geometry, ctx._current(ctx.device), cache, slot)
        if out is not None:
            if out.__class__ is int:
                ctx._check(out)
            return out
    n, shape = slot.shape[0], (slot.shape[0], ctx.kv_heads, ctx.head_dim)
    k, v = slot.new_empty(shape, dtype=ctx.torch_dtype), slot.new_empty(shape, dtype=ctx.torch_dtype)
    ctx.wf_kv_load(cache, slot, n, k.data_ptr(), v.data_ptr())
    return k, v


def kv_attend(ctx: KVContext, q, cache, table, kv_len, q_off, pos, *, scale: float, window: int = 0, max_q: int = 0,
              max_kv: int = 0, stream=None):
    """Attention of the packed queries q [T, q_heads, D] over the cache:
    [T, q_heads, D].  Rows of tokens past q_off[-1] are not written.  max_q and max_kv, the most
    queries and cached tokens of a row, choose the kernel for the whole call; 0 (not known) costs time."""
    if stream is not None:
        with _made_current(ctx, stream):
            return kv_attend(ctx, q, cache, table, kv_len, q_off, pos, scale=scale, window=window, max_q=max_q, max_kv=max_kv)
    if ctx._bind is not None:
        out = ctx._bind.attend(ctx._geometry, ctx._current(ctx.device), q, cache, table, kv_len, q_off, pos, scale, window,
                               max_q, max_kv)
        if out is not None:
            if out.__class__ is int:
                ctx._check(out)
            return out
    n = q.shape[0]
    out = q.new_empty((n, ctx.q_heads, ctx.head_dim))
    ctx.wf_kv_attend(q, n, cache, table, kv_len, q_off, pos, kv_len.shape[0], scale, out.data_ptr(), window=window,
                     max_q=max_q, max_kv=max_kv)
    return out
