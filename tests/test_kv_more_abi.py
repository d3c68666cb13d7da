"""Prompts and the cache in 4 bits: header and binding agree, and what their entry points and the binding refuse, seen
without a GPU."""
import ctypes
import os
import subprocess

import pytest

from conftest import ROOT
from test_kv_abi import HEADER, kv  # noqa: F401

STRUCTS = ["isjl_kv_prompt_args", "isjl_kv_cache4", "isjl_kv_read4_args"]
CSRC = os.path.join(ROOT, "paper_2608_02244_gb300", "csrc")


def test_layout(kv, tmp_path):  # noqa: F811
    lines = []
    for s in STRUCTS:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (s, s))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (s, f[0], s, f[0]) for f in getattr(kv, s)._fields_]
    src, exe = tmp_path / "a.c", tmp_path / "a"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "isjl_kv.h"\nint main(void) { %s return 0; }' % "\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    out = dict(x.split() for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for s in STRUCTS:
        cls = getattr(kv, s)
        assert int(out[s]) == ctypes.sizeof(cls)
        for f in cls._fields_:
            assert int(out["%s.%s" % (s, f[0])]) == getattr(cls, f[0]).offset, (s, f[0])


@pytest.mark.parametrize("name,packed", [("isjl_kv_prompt_args", "_PROMPT"), ("isjl_kv_cache4", "_CACHE4"),
                                         ("isjl_kv_read4_args", "_READ4")])
def test_packed_layout(kv, name, packed):  # noqa: F811
    """The bytes that Decoder packs are the structure's: each value at its field."""
    cls, s = getattr(kv, name), getattr(kv, packed)
    assert s.size == ctypes.sizeof(cls)
    flat = []
    for f, t in cls._fields_:
        flat += [(f, i) for i in range(t._length_)] if hasattr(t, "_length_") else [(f, None)]
    a = cls.from_buffer_copy(s.pack(*range(1, len(flat) + 1)))
    for k, (f, i) in enumerate(flat):
        assert (getattr(a, f) if i is None else getattr(a, f)[i]) == k + 1, f


def test_null_handles(kv):  # noqa: F811
    L = kv.lib()
    for f in (L.isjl_kv_prompt, L.isjl_kv_append4, L.isjl_kv_attend4, L.isjl_kv_read4):
        assert f(None, None, None, None) == kv.ISJL_ERR_INVALID_ARG


# A handle without memory, for calls that are refused, or have nothing to do, before anything is launched.
PROG = r"""
#include <cstdio>
#include "kv.cu"
static int failures = 0;
#define SAME(call, what) do { const int got = (call); if (got != (what)) { ++failures; printf("%d: %d\n", __LINE__, got); } } while (0)
int main() {
    isjl_kv h;
    h.cfg = {10, 16, 8, 2, 64, ISJL_KV_BF16, 4};
    h.shift = 4;
    if (cudaGetDevice(&h.device) != cudaSuccess) h.device = -1;
    alignas(16) static char mem[64];
    char *p = mem;
    const int bad = ISJL_ERR_INVALID_ARG;

    const isjl_kv_cache4 c4 = {p, p, p, p, {1024, 64, 32}, {1024, 64, 32}, {128, 8, 4}, {128, 8, 4}};
    const isjl_kv_cache c16 = {p, p, {2048, 128, 64}, {2048, 128, 64}};
    {
        isjl_kv_read4_args a = {0, nullptr, nullptr, {0, 0}, nullptr, {0, 0}};
        SAME(isjl_kv_read4(&h, &a, &c4, nullptr), ISJL_OK);
        SAME(isjl_kv_read4(&h, &a, nullptr, nullptr), bad);
        for (int i = 0; i < 4; ++i)
            for (char *x : {(char *)nullptr, p + 8}) {
                isjl_kv_cache4 c = c4;
                (i == 0 ? c.k : i == 1 ? c.v : i == 2 ? c.k_scale : c.v_scale) = x;
                SAME(isjl_kv_read4(&h, &a, &c, nullptr), bad);
            }
        for (int i = 0; i < 12; ++i)
            for (const int64_t x : {(int64_t)0, (int64_t)-64, (int64_t)2, (int64_t)1 << 40}) {
                isjl_kv_cache4 c = c4;
                (i < 3 ? c.k_stride : i < 6 ? c.v_stride : i < 9 ? c.k_scale_stride : c.v_scale_stride)[i % 3] = x;
                SAME(isjl_kv_read4(&h, &a, &c, nullptr), bad);
            }
        isjl_kv_cache4 c = c4;
        c.k_stride[0] = 1032;                      // codes: multiples of 16 bytes
        SAME(isjl_kv_read4(&h, &a, &c, nullptr), bad);
        h.cfg.head_dim = 128;                      // scales: multiples of 8 numbers
        SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        h.cfg.head_dim = 64;
        const isjl_kv_read4_args good = {1, (int64_t *)p, p, {128, 64}, p, {128, 64}};
        a = good; a.n_tokens = -1; SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        a = good; a.slots = nullptr; SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        a = good; a.slots = (int64_t *)(p + 4); SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        a = good; a.k_out = p + 8; SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        a = good; a.v_out = nullptr; SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        a = good; a.k_stride[0] = 12; SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
        a = good; a.v_stride[1] = -8; SAME(isjl_kv_read4(&h, &a, &c4, nullptr), bad);
    }
    {
        isjl_kv_append_args a = {};
        SAME(isjl_kv_append4(&h, &a, &c4, nullptr), ISJL_OK);
        SAME(isjl_kv_append4(&h, &a, nullptr, nullptr), bad);
        SAME(isjl_kv_append(&h, &a, nullptr, nullptr), bad);
        a.rot = 24; SAME(isjl_kv_append4(&h, &a, &c4, nullptr), bad);
        a.rot = 0; a.eps = -1.f; SAME(isjl_kv_append4(&h, &a, &c4, nullptr), bad);
        a.eps = 0.f; a.n_tokens = 1; SAME(isjl_kv_append4(&h, &a, &c4, nullptr), bad);
    }
    {
        const isjl_kv_attend_args good = {1, 2, 3, 0, 0, 0, 1.f, p, {512, 64}, p, {512, 64}, nullptr, (int32_t *)p, nullptr, (int32_t *)p, nullptr};
        isjl_kv_attend_args a = good;
        a.n = 0; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), ISJL_OK);
        SAME(isjl_kv_attend4(&h, &a, nullptr, nullptr), bad);
        a = good; a.n = 5; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        a = good; a.n_table_rows = 0; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        h.cfg.max_rows = 4096;                     // slices, and a place for each query, are counted in 32 bits
        a = good; a.n = a.n_table_rows = 4096; a.table_width = 1048570; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        h.cfg.max_rows = 4;
        a = good; a.table_width = 1 << 27; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        a = good; a.n_prefix_blocks = 1; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        a = good; a.scale = -1.f; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        a = good; a.q = p + 8; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        a = good; a.out_stride[1] = 4; SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
        a = good; a.lens = (int32_t *)(p + 2); SAME(isjl_kv_attend4(&h, &a, &c4, nullptr), bad);
    }
    {
        const isjl_kv_prompt_args good = {2, 7, 3, 0, 0, 0, 1.f, p, {512, 64}, p, {512, 64}, nullptr, (int32_t *)p, (int32_t *)p, (int32_t *)p, nullptr};
        isjl_kv_prompt_args a = good;
        a.n_rows = 0; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), ISJL_OK);
        a = good; a.n_tokens = 0; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), ISJL_OK);
        SAME(isjl_kv_prompt(&h, &a, nullptr, nullptr), bad);
        a = good; a.n_rows = 5; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.n_rows = -1; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.n_tokens = -1; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.n_tokens = 1 << 28; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.table_width = 0; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.table_width = 1 << 27; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.n_prefix_blocks = 1; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.n_prefix_blocks = -1; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.window = -1; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.sinks = -1; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.scale = 0.f; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.scale = INFINITY; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.q = nullptr; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.out = p + 4; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.q_stride[0] = 4; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.out_stride[1] = 0; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.lse = (float *)(p + 2); SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.starts = nullptr; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.lens = nullptr; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        a = good; a.table = nullptr; SAME(isjl_kv_prompt(&h, &a, &c16, nullptr), bad);
        isjl_kv_cache c = c16;
        c.k_stride[1] = 4; SAME(isjl_kv_prompt(&h, &good, &c, nullptr), bad);
        h.device += 1;                             // another device's handle
        SAME(isjl_kv_prompt(&h, &good, &c16, nullptr), bad);
    }
    printf("failures %d\n", failures);
    return 0;
}
"""


def test_refusals_of_the_library(kv, tmp_path):  # noqa: F811
    from paper_2608_02244_gb300 import build
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    src, exe = tmp_path / "refusals.cu", tmp_path / "refusals"
    src.write_text(PROG)
    objs = [os.path.join(build.OUT, f) for f in sorted(os.listdir(build.OUT)) if f.endswith(".o") and f != "kv.cu.o"]
    subprocess.run([nvcc, str(src), "-o", str(exe)] + objs + build._flags(False), check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == "failures 0\n"


def test_refusals_of_the_binding(kv):  # noqa: F811
    """A decoder without a handle, whose device is the CPU's."""
    import torch
    d = kv.Decoder.__new__(kv.Decoder)
    d.torch, d.dtype, d.handle, d._lib, d.device = torch, torch.bfloat16, None, kv.lib(), torch.device("cpu")
    d._index, d.n_q_heads, d.n_kv_heads, d.head_dim, d.max_rows = -1, 4, 2, 64, 3
    d._cache_shape, d._codes_shape, d._scales_shape = (5, 16, 2, 64), (5, 16, 2, 32), (5, 16, 2, 2, 2)
    d._qkv, d._raw_stream = 8 * 64, lambda index: 0
    i32, bf = dict(dtype=torch.int32), dict(dtype=torch.bfloat16)
    c = d.cache4()
    assert [t.shape for t in c] == [d._codes_shape] * 2 + [d._scales_shape] * 2 and not c.k.is_contiguous()
    q, table, lens, starts = torch.zeros(7, 4, 64, **bf), torch.zeros(2, 3, **i32), torch.zeros(2, **i32), torch.zeros(3, **i32)
    k = torch.zeros(5, 16, 2, 64, **bf)
    slots = torch.zeros(2, dtype=torch.int64)

    def refused(call, *a, **kw):
        with pytest.raises(kv.IsjlError) as e:
            call(*a, **kw)
        assert e.value.status == kv.ISJL_ERR_INVALID_ARG
        return str(e.value)

    # good arguments come as far as the library, which has no handle
    for call, a in ((d.prompt, (q, k, k, table, starts, lens)), (d.read4, (slots, c)), (d.attend4, (q[:2], c, table, lens)),
                    (d.append4, (torch.zeros(2, 512, **bf), None, slots, c))):
        assert "isjl_kv_" in refused(call, *a)
    for bad in (c[:3], c._replace(k=c.k.int()), c._replace(v=c.v[:4]), c._replace(k_scale=c.k_scale.half()),
                c._replace(v_scale=c.v_scale.flip(4).transpose(3, 4)), c._replace(v_scale=c.v_scale[..., :1].expand(5, 16, 2, 2, 2))):
        assert "Decoder" in refused(d.read4, slots, bad)
        assert "Decoder" in refused(d.attend4, q[:2], bad, table, lens)
    assert "Decoder" in refused(d.read4, slots.int(), c)
    assert "Decoder" in refused(d.read4, slots, c, k=torch.zeros(2, 2, 64))
    assert "Decoder" in refused(d.prompt, q.float(), k, k, table, starts, lens)
    assert "Decoder" in refused(d.prompt, q, k, k, table, starts[:2], lens)
    assert "Decoder" in refused(d.prompt, q, k, k, table[:1], starts, lens)
    assert "Decoder" in refused(d.prompt, q, k, k, table, starts, lens, window=2**31)
    assert "Decoder" in refused(d.prompt, q, k, k, torch.zeros(4, 3, **i32), torch.zeros(5, **i32), torch.zeros(4, **i32))
    assert "Decoder" in refused(d.attend4, q, c, table, lens)              # more queries than max_rows
