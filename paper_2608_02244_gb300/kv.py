"""Python binding of the decode step over a paged KV cache, of prompts and of a cache in 4 bits (argument
marshalling only).

``Decoder`` checks tensors, allocates outputs and calls the entry points of
``include/isjl_kv.h``, whose structures it packs as bytes (the ctypes ones have the
same layout, for callers of the library itself).  All work runs in the library's
CUDA kernels: there is no CPU fallback.

    d = kv.Decoder(n_blocks, block_size, n_q_heads, n_kv_heads, head_dim, max_rows=B)
    plan = d.assign(lens, new_tokens, table, free, n_free, max_tokens)
    q = d.append(qkv, plan.positions, plan.slots, k_cache, v_cache, rope, q_weight, k_weight)
    out = d.attend(q, k_cache, v_cache, table, plan.visible, rows=plan.rows, window=4096, sinks=4)

Prompts, whose tokens `assign` and `append` take all at once:

    out = d.prompt(q, k_cache, v_cache, table, plan.starts, plan.lens)

A cache in 4 bits, in append's and attend's place:

    cache = d.cache4()
    q = d.append4(qkv, plan.positions, plan.slots, cache, rope, q_weight, k_weight)
    out = d.attend4(q, cache, table, plan.visible, rows=plan.rows)
"""
from __future__ import annotations

import collections
import ctypes
import struct

from . import sim
from .sim import ISJL_ERR_INVALID_ARG, ISJL_OK, IsjlError

BF16, FP16 = 0, 1
MAX_ROWS = 4096
EXPORTS = ["isjl_kv_create", "isjl_kv_destroy", "isjl_kv_assign", "isjl_kv_append", "isjl_kv_attend",
           "isjl_kv_status", "isjl_kv_prompt", "isjl_kv_append4", "isjl_kv_attend4", "isjl_kv_read4"]
GROUP4 = 32      # values of a group of a cache in 4 bits

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class isjl_kv_config(ctypes.Structure):
    _fields_ = [(f, _i32) for f in ("n_blocks", "block_size", "n_q_heads", "n_kv_heads", "head_dim", "type", "max_rows")]


class isjl_kv_cache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_stride", _i64 * 3), ("v_stride", _i64 * 3)]


class isjl_kv_assign_args(ctypes.Structure):
    _fields_ = [(f, _i32) for f in ("n_rows", "table_width", "max_tokens", "prefix_len")] + [
        (f, _vp) for f in ("lens", "new_tokens", "table", "free_list", "n_free", "lens_out", "n_free_out", "granted",
                           "starts", "slots", "positions", "rows", "visible")]


class isjl_kv_append_args(ctypes.Structure):
    _fields_ = [("n_tokens", _i32), ("n_positions", _i32), ("rot", _i32), ("interleaved", _i32), ("eps", _f32),
                ("qkv", _vp), ("qkv_stride", _i64), ("q_out", _vp), ("q_out_stride", _i64), ("q_weight", _vp),
                ("k_weight", _vp), ("rope", _vp), ("positions", _vp), ("slots", _vp)]


class isjl_kv_attend_args(ctypes.Structure):
    _fields_ = [(f, _i32) for f in ("n", "n_table_rows", "table_width", "n_prefix_blocks", "window", "sinks")] + [
        ("scale", _f32), ("q", _vp), ("q_stride", _i64 * 2), ("out", _vp), ("out_stride", _i64 * 2), ("lse", _vp),
        ("lens", _vp), ("rows", _vp), ("table", _vp), ("prefix", _vp)]


class isjl_kv_prompt_args(ctypes.Structure):
    _fields_ = [(f, _i32) for f in ("n_rows", "n_tokens", "table_width", "n_prefix_blocks", "window", "sinks")] + [
        ("scale", _f32), ("q", _vp), ("q_stride", _i64 * 2), ("out", _vp), ("out_stride", _i64 * 2), ("lse", _vp),
        ("starts", _vp), ("lens", _vp), ("table", _vp), ("prefix", _vp)]


class isjl_kv_cache4(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("k", "v", "k_scale", "v_scale")] + [
        (f, _i64 * 3) for f in ("k_stride", "v_stride", "k_scale_stride", "v_scale_stride")]


class isjl_kv_read4_args(ctypes.Structure):
    _fields_ = [("n_tokens", _i32), ("slots", _vp), ("k_out", _vp), ("k_stride", _i64 * 2), ("v_out", _vp),
                ("v_stride", _i64 * 2)]


# The same layouts as bytes: filling a structure field by field costs a call 3 us of host time, packing 0.3
_CACHE = struct.Struct("=2Q6q")
_ASSIGN = struct.Struct("=4i13Q")
_APPEND = struct.Struct("=4if4xQqQq5Q")
_ATTEND = struct.Struct("=6if4xQ2qQ2q5Q")
_PROMPT = struct.Struct("=6if4xQ2qQ2q5Q")
_CACHE4 = struct.Struct("=4Q12q")
_READ4 = struct.Struct("=i4x2Q2qQ2q")

_lib = None


def lib():
    """The shared library with the argument types of the entry points set (raises if it was not built)."""
    global _lib
    if _lib is None:
        L = sim.lib()
        L.isjl_kv_create.argtypes = [ctypes.POINTER(isjl_kv_config), ctypes.POINTER(_vp)]
        L.isjl_kv_destroy.argtypes = [_vp]
        L.isjl_kv_destroy.restype = None
        L.isjl_kv_assign.argtypes = [_vp, _vp, _vp]            # structures by address, or their bytes
        L.isjl_kv_append.argtypes = [_vp, _vp, _vp, _vp]
        L.isjl_kv_attend.argtypes = [_vp, _vp, _vp, _vp]
        L.isjl_kv_prompt.argtypes = [_vp, _vp, _vp, _vp]
        L.isjl_kv_append4.argtypes = [_vp, _vp, _vp, _vp]
        L.isjl_kv_attend4.argtypes = [_vp, _vp, _vp, _vp]
        L.isjl_kv_read4.argtypes = [_vp, _vp, _vp, _vp]
        L.isjl_kv_status.argtypes = [_vp]
        for f in ("create", "assign", "append", "attend", "prompt", "append4", "attend4", "read4", "status"):
            getattr(L, "isjl_kv_" + f).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(st, where):
    if st != ISJL_OK:
        raise IsjlError(st, where)


def isjl_kv_create(n_blocks, block_size, n_q_heads, n_kv_heads, head_dim, type, max_rows):
    cfg = isjl_kv_config(int(n_blocks), int(block_size), int(n_q_heads), int(n_kv_heads), int(head_dim), int(type),
                         int(max_rows))
    h = _vp()
    _check(lib().isjl_kv_create(ctypes.byref(cfg), ctypes.byref(h)), "isjl_kv_create")
    return h


def isjl_kv_destroy(handle):
    if handle:
        lib().isjl_kv_destroy(handle)


# A step's results: maps of its tokens (slots, positions, rows, visible), the first
# entry of each row in them and their total (starts), tokens granted to each row,
# lengths and free blocks after the step.
Plan = collections.namedtuple("Plan", "slots positions rows visible starts granted lens n_free")

# A cache in 4 bits: codes of keys and values, uint8 [n_blocks, block_size, n_kv_heads, head_dim / 2], and the scales and
# offsets of their groups, [n_blocks, block_size, n_kv_heads, head_dim / 32, 2] of the decoder's type.
Cache4 = collections.namedtuple("Cache4", "k v k_scale v_scale")


class Decoder:
    """Owns a library handle for one cache and head shape.  Caches, tables and
    lengths are the caller's.  Calls go to `stream` (default: the current one) and
    must not overlap on the GPU; the device that was current when the decoder was made
    has to be current (else IsjlError).  A call's inputs have to be ready for its stream, and
    its results are ready when that stream is done with it.  Caches are
    [n_blocks, block_size, n_kv_heads, head_dim] with any order of the first three axes
    in memory.  Serving only: results carry no gradient, whatever the inputs require,
    and torch's version counters do not see what is written to caches, tables and
    lengths."""

    def __init__(self, n_blocks, block_size, n_q_heads, n_kv_heads, head_dim, dtype=None, max_rows=512):
        import torch
        self.torch = torch
        self.dtype = torch.bfloat16 if dtype is None else dtype
        self.handle = None
        if self.dtype not in (torch.bfloat16, torch.float16):
            raise IsjlError(ISJL_ERR_INVALID_ARG, "Decoder: dtype must be bfloat16 or float16")
        self.n_blocks, self.block_size = int(n_blocks), int(block_size)
        self.n_q_heads, self.n_kv_heads, self.head_dim = int(n_q_heads), int(n_kv_heads), int(head_dim)
        self.max_rows = int(max_rows)
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.handle = isjl_kv_create(n_blocks, block_size, n_q_heads, n_kv_heads, head_dim,
                                     BF16 if self.dtype == torch.bfloat16 else FP16, max_rows)
        self._lib = lib()
        self._index = self.device.index
        self._raw_stream = torch._C._cuda_getCurrentRawStream      # 0.1 us; torch.cuda.current_stream 1.9
        self._cache_shape = (self.n_blocks, self.block_size, self.n_kv_heads, self.head_dim)
        self._qkv = (self.n_q_heads + 2 * self.n_kv_heads) * self.head_dim
        self._codes_shape = self._cache_shape[:3] + (self.head_dim // 2,)
        self._scales_shape = self._cache_shape[:3] + (self.head_dim // GROUP4, 2)

    def close(self):
        if self.handle:
            isjl_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    # ---- checks ----------------------------------------------------------
    def _bad(self, what):
        raise IsjlError(ISJL_ERR_INVALID_ARG, f"Decoder: {what}")

    def _ints(self, name, t, shape, dtype):
        if t.dtype is not dtype or t.get_device() != self._index or t.shape != shape or not t.is_contiguous():
            self._bad(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}")
        return t.data_ptr()

    def _cache(self, k, v):
        shape, dtype, index = self._cache_shape, self.dtype, self._index
        ks, vs = k.stride(), v.stride()
        if k.shape != shape or v.shape != shape or k.dtype is not dtype or v.dtype is not dtype or \
                k.get_device() != index or v.get_device() != index or ks[3] != 1 or vs[3] != 1:
            self._bad(f"caches must be {dtype} of shape {shape} on {self.device} with stride 1 last")
        if shape[0] == 1 or shape[2] == 1:
            # the stride of an axis of one element says nothing: any valid one
            ks, vs = ([x if n > 1 else 8 for x, n in zip(y, shape)] for y in (ks, vs))
        return _CACHE.pack(k.data_ptr(), v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2])

    def _cache4(self, cache):
        if len(cache) != 4:
            self._bad("a cache in 4 bits is codes of keys and of values, scales of keys and of values")
        k, v, ks, vs = cache
        codes, scales, index, dtype, u8 = self._codes_shape, self._scales_shape, self._index, self.dtype, self.torch.uint8
        a, b, c, d = k.stride(), v.stride(), ks.stride(), vs.stride()
        if k.shape != codes or v.shape != codes or ks.shape != scales or vs.shape != scales or \
                k.dtype is not u8 or v.dtype is not u8 or ks.dtype is not dtype or vs.dtype is not dtype or \
                k.get_device() != index or v.get_device() != index or ks.get_device() != index or vs.get_device() != index or \
                a[3] != 1 or b[3] != 1 or c[4] != 1 or d[4] != 1 or (scales[3] > 1 and (c[3] != 2 or d[3] != 2)):
            self._bad(f"a cache in 4 bits has codes of torch.uint8 {codes} and scales of {dtype} {scales} on {self.device}, "
                      "a head's next to one another")
        if codes[0] == 1 or codes[2] == 1:
            # the stride of an axis of one element says nothing: any valid one
            a, b, c, d = ([x if n > 1 else 16 for x, n in zip(y, codes)] for y in (a, b, c, d))
        return _CACHE4.pack(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), a[0], a[1], a[2], b[0], b[1], b[2],
                            c[0], c[1], c[2], d[0], d[1], d[2])

    def _empty(self, stream, shape, dtype):
        """Memory for a result.  The allocator hands out what is free in the order of one stream's
        work, so it is asked on the stream that the call goes to; the current stream may use the
        result until it is dropped."""
        torch = self.torch
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        current = torch.cuda.current_stream(self.device)
        with torch.cuda.stream(stream):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(current)
        return t

    def _stream(self, stream, tensors):
        """The stream's number; the caller's memory in a call on another stream than the current one
        stays until that stream is done with it."""
        if stream is None:
            return self._raw_stream(self._index)
        if stream != self.torch.cuda.current_stream(self.device):
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
        return stream.cuda_stream

    # ---- the step's parts --------------------------------------------------
    def assign(self, lens, new_tokens, table, free, n_free, max_tokens, prefix_len=0, in_place=False, stream=None):
        """Block tables and slot maps of a step: see isjl_kv_assign.  `table` and `free`
        are updated, `lens` and `n_free` too with `in_place` (else the plan holds new ones)."""
        torch = self.torch
        i32 = torch.int32
        n, m = lens.shape[0], int(max_tokens)
        if not 1 <= m < 2**31 or n > self.max_rows or table.dim() != 2 or table.shape[0] != n:
            self._bad("assign needs max_tokens >= 1, at most max_rows lengths and a table row for each")
        prefix_len = int(prefix_len)
        if not 0 <= prefix_len < 2**31:
            self._bad("prefix_len out of range")
        ptrs = (self._ints("lens", lens, (n,), i32), self._ints("new_tokens", new_tokens, (n,), i32),
                self._ints("table", table, table.shape, i32), self._ints("free", free, (self.n_blocks,), i32),
                self._ints("n_free", n_free, (1,), i32))
        # one allocation for the 32-bit results, whose maps begin at multiples of 16 bytes
        w = (m + 3) & ~3
        sizes = [w, w, w, n + 1, n] if in_place else [w, w, w, n + 1, n, n, 1]
        slots = self._empty(stream, m, torch.int64)
        block = self._empty(stream, 3 * w + (2 * n + 1 if in_place else 3 * n + 2), i32)
        parts = block.unsafe_split_with_sizes(sizes)       # integers: no view to keep track of, 2 us less
        positions, rows, visible, starts, granted = parts[:5]
        if w != m:
            positions, rows, visible = positions[:m], rows[:m], visible[:m]
        lens_out, n_free_out = (lens, n_free) if in_place else parts[5:]
        base = block.data_ptr()
        at = base + 12 * w + 4 * (n + 1)
        out = (ptrs[0], ptrs[4]) if in_place else (at + 4 * n, at + 8 * n)
        args = _ASSIGN.pack(n, table.shape[1], m, prefix_len, *ptrs, *out, at, base + 12 * w, slots.data_ptr(), base,
                            base + 4 * w, base + 8 * w)
        st = self._stream(stream, (lens, new_tokens, table, free, n_free))
        _check(self._lib.isjl_kv_assign(self.handle, args, st), "isjl_kv_assign")
        return Plan(slots, positions, rows, visible, starts, granted, lens_out, n_free_out)

    def append(self, qkv, positions, slots, k, v, rope=None, q_weight=None, k_weight=None, eps=1e-6, pairs=False,
               out=None, stream=None):
        """Norms, rotation and cache write of new tokens: see isjl_kv_append.  qkv is
        [tokens, (n_q_heads + 2 n_kv_heads) * head_dim]; returns the queries,
        [tokens, n_q_heads, head_dim].  rope None: no rotation; `pairs`: neighbours."""
        return self._append(self._lib.isjl_kv_append, "isjl_kv_append", (k, v), self._cache(k, v), qkv, positions, slots, rope,
                            q_weight, k_weight, eps, pairs, out, stream)

    def append4(self, qkv, positions, slots, cache, rope=None, q_weight=None, k_weight=None, eps=1e-6, pairs=False,
                out=None, stream=None):
        """append with a cache in 4 bits (`cache4`): see isjl_kv_append4."""
        return self._append(self._lib.isjl_kv_append4, "isjl_kv_append4", cache, self._cache4(cache), qkv, positions, slots,
                            rope, q_weight, k_weight, eps, pairs, out, stream)

    def _append(self, call, name, tensors, cache, qkv, positions, slots, rope, q_weight, k_weight, eps, pairs, out, stream):
        torch = self.torch
        hq, d, dtype, index = self.n_q_heads, self.head_dim, self.dtype, self._index
        n = qkv.shape[0]
        if qkv.shape != (n, self._qkv) or qkv.dtype is not dtype or qkv.get_device() != index or (n > 0 and qkv.stride(1) != 1):
            self._bad(f"qkv must be {dtype} [tokens, {self._qkv}] with stride 1 last")
        if out is None:
            out = self._empty(stream, (n, hq, d), dtype)
        elif out.shape != (n, hq, d) or out.dtype is not dtype or out.get_device() != index or \
                out.stride(2) != 1 or (hq > 1 and out.stride(1) != d):
            self._bad("out must be [tokens, n_q_heads, head_dim] of the cache's type, heads side by side")
        angles = places = n_positions = rot = 0
        if rope is not None:
            if rope.dim() != 2 or rope.dtype is not torch.float32 or rope.get_device() != index or not rope.is_contiguous():
                self._bad("rope must be contiguous float32 [positions, rot]")
            n_positions, rot = rope.shape
            angles, places = rope.data_ptr(), self._ints("positions", positions, (n,), torch.int32)
        weights = [0 if w is None else self._ints(name, w, (d,), dtype) for name, w in (("q_weight", q_weight), ("k_weight", k_weight))]
        x, y = qkv.data_ptr(), out.data_ptr()
        # the stride of a single row says nothing
        step, out_step = (qkv.stride(0), out.stride(0)) if n > 1 else (self._qkv, self._qkv if x == y else hq * d)
        args = _APPEND.pack(n, n_positions, rot, bool(pairs), eps, x, step, y, out_step, *weights, angles, places,
                            self._ints("slots", slots, (n,), torch.int64))
        st = self._stream(stream, (qkv, out, *tensors, rope, positions, slots, q_weight, k_weight))
        _check(call(self.handle, args, cache, st), name)
        return out

    def attend(self, q, k, v, table, lens, rows=None, prefix=None, window=0, sinks=0, scale=None, out=None, lse=False,
               stream=None):
        """Attention of single queries [n, n_q_heads, head_dim] over their requests'
        tokens: see isjl_kv_attend.  scale defaults to head_dim ** -0.5.  With `lse`
        returns (out, lse)."""
        return self._attend(self._lib.isjl_kv_attend, "isjl_kv_attend", (k, v), self._cache(k, v), q, table, lens, rows, prefix,
                            window, sinks, scale, out, lse, stream)

    def attend4(self, q, cache, table, lens, rows=None, prefix=None, window=0, sinks=0, scale=None, out=None, lse=False,
                stream=None):
        """attend over a cache in 4 bits (`cache4`): see isjl_kv_attend4."""
        return self._attend(self._lib.isjl_kv_attend4, "isjl_kv_attend4", cache, self._cache4(cache), q, table, lens, rows,
                            prefix, window, sinks, scale, out, lse, stream)

    def _queries(self, q, out, stream, most):
        """Checks of queries and results; the results and both's strides, any valid one for an axis of one element
        (it says nothing)."""
        hq, d, dtype, index = self.n_q_heads, self.head_dim, self.dtype, self._index
        n = q.shape[0]
        shape = (n, hq, d)
        if q.shape != shape or q.dtype is not dtype or q.get_device() != index or q.stride(2) != 1 or n > most:
            self._bad(f"q must be {dtype} [at most {most}, {hq}, {d}] with stride 1 last")
        if out is None:
            out = self._empty(stream, shape, dtype)
        elif out.shape != shape or out.dtype is not dtype or out.get_device() != index or out.stride(2) != 1:
            self._bad("out must have q's shape and type with stride 1 last")
        qs, os = q.stride(), out.stride()
        if n <= 1 or hq == 1:
            qs, os = ([x if m > 1 else 8 for x, m in zip(y, shape)] for y in (qs, os))
        return out, qs, os

    def _sight(self, table, window, sinks):
        if table.dim() != 2:
            self._bad("table must be [rows, width]")
        window, sinks = int(window), int(sinks)
        if not (0 <= window < 2**31 and 0 <= sinks < 2**31):
            self._bad("window and sinks must be in 0..2^31 - 1")
        return window, sinks

    def _attend(self, call, name, tensors, cache, q, table, lens, rows, prefix, window, sinks, scale, out, lse, stream):
        n, i32 = q.shape[0], self.torch.int32
        out, qs, os = self._queries(q, out, stream, self.max_rows)
        window, sinks = self._sight(table, window, sinks)
        weights = self._empty(stream, (n, self.n_q_heads), self.torch.float32) if lse else None
        args = _ATTEND.pack(n, table.shape[0], table.shape[1], 0 if prefix is None else prefix.numel(), window, sinks,
                            self.head_dim ** -0.5 if scale is None else scale, q.data_ptr(), qs[0], qs[1], out.data_ptr(),
                            os[0], os[1], weights.data_ptr() if lse else 0, self._ints("lens", lens, (n,), i32),
                            0 if rows is None else self._ints("rows", rows, (n,), i32),
                            self._ints("table", table, table.shape, i32),
                            0 if prefix is None else self._ints("prefix", prefix, (prefix.numel(),), i32))
        st = self._stream(stream, (q, *tensors, table, lens, rows, prefix, out, weights))
        _check(call(self.handle, args, cache, st), name)
        return (out, weights) if lse else out

    def prompt(self, q, k, v, table, starts, lens, prefix=None, window=0, sinks=0, scale=None, out=None, lse=False,
               stream=None):
        """Causal attention of the rows' newest tokens, packed: see isjl_kv_prompt.  q is [tokens, n_q_heads,
        head_dim], row i's queries at starts[i]..starts[i + 1] - 1, the last of its lens[i] own tokens.  scale
        defaults to head_dim ** -0.5.  With `lse` returns (out, lse).  Of tokens beyond starts[-1] a given `out`
        keeps what it holds; in new results they are not defined."""
        torch, i32, n = self.torch, self.torch.int32, lens.shape[0]
        cache = self._cache(k, v)
        out, qs, os = self._queries(q, out, stream, (2**31 - 1) // self.n_q_heads)
        window, sinks = self._sight(table, window, sinks)
        if n > self.max_rows or table.shape[0] != n:
            self._bad("prompt needs at most max_rows lengths and a table row for each")
        weights = self._empty(stream, (q.shape[0], self.n_q_heads), torch.float32) if lse else None
        args = _PROMPT.pack(n, q.shape[0], table.shape[1], 0 if prefix is None else prefix.numel(), window, sinks,
                            self.head_dim ** -0.5 if scale is None else scale, q.data_ptr(), qs[0], qs[1], out.data_ptr(),
                            os[0], os[1], weights.data_ptr() if lse else 0, self._ints("starts", starts, (n + 1,), i32),
                            self._ints("lens", lens, (n,), i32), self._ints("table", table, table.shape, i32),
                            0 if prefix is None else self._ints("prefix", prefix, (prefix.numel(),), i32))
        st = self._stream(stream, (q, k, v, table, starts, lens, prefix, out, weights))
        _check(self._lib.isjl_kv_prompt(self.handle, args, cache, st), "isjl_kv_prompt")
        return (out, weights) if lse else out

    # ---- a cache in 4 bits ---------------------------------------------------
    def cache4(self):
        """A new cache in 4 bits whose tokens stand for zeros, each block's heads outermost in memory: a head's
        codes and scales of a block then lie next to one another, in whole lines of memory for attend4."""
        n, bs, heads, _ = self._cache_shape

        def zeros(dtype, *inner):
            return self.torch.zeros((n, heads, bs) + inner, dtype=dtype, device=self.device).transpose(1, 2)

        codes, scales = (self.torch.uint8, self.head_dim // 2), (self.dtype, self.head_dim // GROUP4, 2)
        return Cache4(zeros(*codes), zeros(*codes), zeros(*scales), zeros(*scales))

    def read4(self, slots, cache, k=None, v=None, stream=None):
        """Keys and values of slots in 16 bits, [tokens, n_kv_heads, head_dim] each: see isjl_kv_read4.  `k` and `v`
        take them if given: any strides but 1 last, such as a cache's own slots."""
        n, dtype, index = slots.shape[0], self.dtype, self._index
        shape = (n, self.n_kv_heads, self.head_dim)
        places, packed = self._ints("slots", slots, (n,), self.torch.int64), self._cache4(cache)
        if k is None:
            k = self._empty(stream, shape, dtype)
        if v is None:
            v = self._empty(stream, shape, dtype)
        ks, vs = k.stride(), v.stride()
        if k.shape != shape or v.shape != shape or k.dtype is not dtype or v.dtype is not dtype or \
                k.get_device() != index or v.get_device() != index or ks[2] != 1 or vs[2] != 1:
            self._bad(f"k and v must be {dtype} {shape} on {self.device} with stride 1 last")
        if n <= 1 or shape[1] == 1:
            # the stride of an axis of one element says nothing: any valid one
            ks, vs = ([x if m > 1 else 8 for x, m in zip(y, shape)] for y in (ks, vs))
        args = _READ4.pack(n, places, k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1])
        st = self._stream(stream, (slots, *cache, k, v))
        _check(self._lib.isjl_kv_read4(self.handle, args, packed, st), "isjl_kv_read4")
        return k, v

    def status(self):
        """Wait for the device; the status code of all calls since the last report."""
        return self._lib.isjl_kv_status(self.handle)
