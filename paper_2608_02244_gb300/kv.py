"""Python binding of the decode step over a paged KV cache (argument marshalling only).

The functions with C names forward to the entry points of ``include/isjl_kv.h``;
``Decoder`` checks tensors, allocates outputs and calls them.  All work runs in
the library's CUDA kernels: there is no CPU fallback.

    d = kv.Decoder(n_blocks, block_size, n_q_heads, n_kv_heads, head_dim, max_rows=B)
    plan = d.assign(lens, new_tokens, table, free, n_free, max_tokens)
    q = d.append(qkv, plan.positions, plan.slots, k_cache, v_cache, rope, q_weight, k_weight)
    out = d.attend(q, k_cache, v_cache, table, plan.visible, rows=plan.rows, window=4096, sinks=4)
"""
from __future__ import annotations

import collections
import ctypes

from . import sim
from .sim import ISJL_ERR_INVALID_ARG, ISJL_OK, IsjlError

BF16, FP16 = 0, 1
MAX_ROWS = 4096
EXPORTS = ["isjl_kv_create", "isjl_kv_destroy", "isjl_kv_assign", "isjl_kv_append", "isjl_kv_attend",
           "isjl_kv_status"]

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


_lib = None


def lib():
    """The shared library with the argument types of the entry points set (raises if it was not built)."""
    global _lib
    if _lib is None:
        L = sim.lib()
        L.isjl_kv_create.argtypes = [ctypes.POINTER(isjl_kv_config), ctypes.POINTER(_vp)]
        L.isjl_kv_destroy.argtypes = [_vp]
        L.isjl_kv_destroy.restype = None
        L.isjl_kv_assign.argtypes = [_vp, ctypes.POINTER(isjl_kv_assign_args), _vp]
        L.isjl_kv_append.argtypes = [_vp, ctypes.POINTER(isjl_kv_append_args), ctypes.POINTER(isjl_kv_cache), _vp]
        L.isjl_kv_attend.argtypes = [_vp, ctypes.POINTER(isjl_kv_attend_args), ctypes.POINTER(isjl_kv_cache), _vp]
        L.isjl_kv_status.argtypes = [_vp]
        for f in ("create", "assign", "append", "attend", "status"):
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


class Decoder:
    """Owns a library handle for one cache and head shape.  Caches, tables and
    lengths are the caller's.  Calls go to `stream` (default: the current one) and
    must not overlap on the GPU.  Caches are [n_blocks, block_size, n_kv_heads,
    head_dim] with any order of the first three axes in memory."""

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
        self._cache_shape = (self.n_blocks, self.block_size, self.n_kv_heads, self.head_dim)

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
        if t.dtype != dtype or t.device != self.device or t.shape != shape or not t.is_contiguous():
            self._bad(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}")
        return t.data_ptr()

    def _cache(self, k, v):
        for name, t in (("k", k), ("v", v)):
            if t.shape != self._cache_shape or t.dtype != self.dtype or t.device != self.device or t.stride(3) != 1:
                self._bad(f"{name} cache must be {self.dtype} of shape {self._cache_shape} on {self.device} with stride 1 last")
        ks, vs = k.stride(), v.stride()
        return isjl_kv_cache(k.data_ptr(), v.data_ptr(), (_i64 * 3)(*self._steps(ks, k.shape)), (_i64 * 3)(*self._steps(vs, v.shape)))

    @staticmethod
    def _steps(strides, shape):
        # the stride of an axis of one element says nothing: any valid one
        return [s if n > 1 else 8 for s, n in zip(strides[:3], shape)]

    def _stream(self, stream, tensors):
        """The stream's number; memory of a call on another stream than the current one stays
        until that stream is done with it."""
        current = self.torch.cuda.current_stream(self.device)
        if stream is None or stream == current:
            return current.cuda_stream
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
        if m < 1 or n > self.max_rows or table.dim() != 2 or table.shape[0] != n:
            self._bad("assign needs max_tokens >= 1, at most max_rows lengths and a table row for each")
        a = isjl_kv_assign_args(n, table.shape[1], m, int(prefix_len))
        a.lens = self._ints("lens", lens, (n,), i32)
        a.new_tokens = self._ints("new_tokens", new_tokens, (n,), i32)
        a.table = self._ints("table", table, table.shape, i32)
        a.free_list = self._ints("free", free, (self.n_blocks,), i32)
        a.n_free = self._ints("n_free", n_free, (1,), i32)
        # one allocation for the 32-bit results
        sizes = [m, m, m, n + 1, n] + ([] if in_place else [n, 1])
        slots = torch.empty(m, dtype=torch.int64, device=self.device)
        block = torch.empty(sum(sizes), dtype=i32, device=self.device)
        parts = block.split(sizes)
        positions, rows, visible, starts, granted = parts[:5]
        lens_out, n_free_out = (lens, n_free) if in_place else parts[5:]
        a.slots, base = slots.data_ptr(), block.data_ptr()
        a.positions, a.rows, a.visible, a.starts = base, base + 4 * m, base + 8 * m, base + 12 * m
        a.granted = a.starts + 4 * (n + 1)
        a.lens_out, a.n_free_out = (a.lens, a.n_free) if in_place else (a.granted + 4 * n, a.granted + 8 * n)
        st = self._stream(stream, (lens, new_tokens, table, free, n_free, slots, block))
        _check(self._lib.isjl_kv_assign(self.handle, ctypes.byref(a), st), "isjl_kv_assign")
        return Plan(slots, positions, rows, visible, starts, granted, lens_out, n_free_out)

    def append(self, qkv, positions, slots, k, v, rope=None, q_weight=None, k_weight=None, eps=1e-6, pairs=False,
               out=None, stream=None):
        """Norms, rotation and cache write of new tokens: see isjl_kv_append.  qkv is
        [tokens, (n_q_heads + 2 n_kv_heads) * head_dim]; returns the queries,
        [tokens, n_q_heads, head_dim].  rope None: no rotation; `pairs`: neighbours."""
        torch = self.torch
        n, hq, d = qkv.shape[0], self.n_q_heads, self.head_dim
        if qkv.dim() != 2 or qkv.shape[1] != (hq + 2 * self.n_kv_heads) * d or qkv.dtype != self.dtype or \
                qkv.device != self.device or (n > 0 and qkv.stride(1) != 1):
            self._bad(f"qkv must be {self.dtype} [tokens, {(hq + 2 * self.n_kv_heads) * d}] with stride 1 last")
        cache = self._cache(k, v)
        if out is None:
            out = torch.empty(n, hq, d, dtype=self.dtype, device=self.device)
        elif out.shape != (n, hq, d) or out.dtype != self.dtype or out.device != self.device or \
                out.stride(2) != 1 or (hq > 1 and out.stride(1) != d):
            self._bad("out must be [tokens, n_q_heads, head_dim] of the cache's type, heads side by side")
        a = isjl_kv_append_args(n, 0, 0, bool(pairs), float(eps), qkv.data_ptr(), qkv.stride(0) if n > 1 else qkv.shape[1],
                                out.data_ptr(), out.stride(0) if n > 1 else hq * d)
        if n == 1 and a.q_out == a.qkv:
            a.q_out_stride = a.qkv_stride
        if rope is not None:
            if rope.dim() != 2 or rope.dtype != torch.float32 or rope.device != self.device or not rope.is_contiguous():
                self._bad("rope must be contiguous float32 [positions, rot]")
            a.n_positions, a.rot = rope.shape
            a.rope = rope.data_ptr()
            a.positions = self._ints("positions", positions, (n,), torch.int32)
        a.slots = self._ints("slots", slots, (n,), torch.int64)
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is not None:
                setattr(a, name, self._ints(name, w, (d,), self.dtype))
        st = self._stream(stream, (qkv, out, k, v, rope, positions, slots, q_weight, k_weight))
        _check(self._lib.isjl_kv_append(self.handle, ctypes.byref(a), ctypes.byref(cache), st), "isjl_kv_append")
        return out

    def attend(self, q, k, v, table, lens, rows=None, prefix=None, window=0, sinks=0, scale=None, out=None, lse=False,
               stream=None):
        """Attention of single queries [n, n_q_heads, head_dim] over their requests'
        tokens: see isjl_kv_attend.  scale defaults to head_dim ** -0.5.  With `lse`
        returns (out, lse)."""
        torch = self.torch
        n, hq, d = q.shape[0], self.n_q_heads, self.head_dim
        shape = (n, hq, d)
        if q.shape != shape or q.dtype != self.dtype or q.device != self.device or q.stride(2) != 1 or n > self.max_rows:
            self._bad(f"q must be {self.dtype} [at most {self.max_rows}, {hq}, {d}] with stride 1 last")
        cache = self._cache(k, v)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=self.device)
        elif out.shape != shape or out.dtype != self.dtype or out.device != self.device or out.stride(2) != 1:
            self._bad("out must have q's shape and type with stride 1 last")
        if table.dim() != 2:
            self._bad("table must be [rows, width]")
        a = isjl_kv_attend_args(n, table.shape[0], table.shape[1], 0, int(window), int(sinks),
                                d ** -0.5 if scale is None else float(scale), q.data_ptr())
        a.q_stride[0], a.q_stride[1] = q.stride(0) if n > 1 else 8, q.stride(1) if hq > 1 else 8
        a.out_stride[0], a.out_stride[1] = out.stride(0) if n > 1 else 8, out.stride(1) if hq > 1 else 8
        a.out = out.data_ptr()
        weights = None
        if lse:
            weights = torch.empty((n, hq), dtype=torch.float32, device=self.device)
            a.lse = weights.data_ptr()
        a.table = self._ints("table", table, table.shape, torch.int32)
        a.lens = self._ints("lens", lens, (n,), torch.int32)
        if rows is not None:
            a.rows = self._ints("rows", rows, (n,), torch.int32)
        if prefix is not None:
            a.n_prefix_blocks = prefix.numel()
            a.prefix = self._ints("prefix", prefix, (prefix.numel(),), torch.int32)
        st = self._stream(stream, (q, k, v, table, lens, rows, prefix, out, weights))
        _check(self._lib.isjl_kv_attend(self.handle, ctypes.byref(a), ctypes.byref(cache), st), "isjl_kv_attend")
        return (out, weights) if lse else out

    def status(self):
        """Wait for the last call; the status code of everything since the last report."""
        return self._lib.isjl_kv_status(self.handle)
