"""include/isjl_kv.h, the library and the binding agree; arguments that can be refused without a GPU."""
import ctypes
import os
import re
import subprocess
import tempfile

import pytest

from conftest import ROOT

HEADER = os.path.join(ROOT, "include", "isjl_kv.h")
STRUCTS = ["isjl_kv_config", "isjl_kv_cache", "isjl_kv_assign_args", "isjl_kv_append_args", "isjl_kv_attend_args"]


@pytest.fixture(scope="module")
def kv():
    from paper_2608_02244_gb300 import build, kv
    build.build()
    kv.lib()
    return kv


def test_exports(kv):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = set(re.findall(r"\b(isjl_kv_\w+)\s*\(", text))
    assert declared == set(kv.EXPORTS)
    for name in declared:
        assert hasattr(kv.lib(), name)


def test_layout(kv):
    lines = []
    for s in STRUCTS:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (s, s))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (s, f[0], s, f[0]) for f in getattr(kv, s)._fields_]
    prog = '#include <stdio.h>\n#include <stddef.h>\n#include "isjl_kv.h"\nint main(void) { %s return 0; }' % "\n".join(lines)
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "a.c"), os.path.join(d, "a")
        open(src, "w").write(prog)
        subprocess.run(["gcc", "-I", os.path.dirname(HEADER), src, "-o", exe], check=True)
        out = dict(x.split() for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for s in STRUCTS:
        cls = getattr(kv, s)
        assert int(out[s]) == ctypes.sizeof(cls)
        for f in cls._fields_:
            assert int(out["%s.%s" % (s, f[0])]) == getattr(cls, f[0]).offset, (s, f[0])


@pytest.mark.parametrize("name,packed", [("isjl_kv_cache", "_CACHE"), ("isjl_kv_assign_args", "_ASSIGN"),
                                         ("isjl_kv_append_args", "_APPEND"), ("isjl_kv_attend_args", "_ATTEND")])
def test_packed_layout(kv, name, packed):
    """The bytes that Decoder packs are the structure's: each value at its field."""
    cls, s = getattr(kv, name), getattr(kv, packed)
    assert s.size == ctypes.sizeof(cls)
    flat = []
    for f, t in cls._fields_:
        flat += [(f, i) for i in range(t._length_)] if hasattr(t, "_length_") else [(f, None)]
    a = cls.from_buffer_copy(s.pack(*range(1, len(flat) + 1)))
    for k, (f, i) in enumerate(flat):
        assert (getattr(a, f) if i is None else getattr(a, f)[i]) == k + 1, f


@pytest.mark.parametrize("change", [dict(n_blocks=0), dict(block_size=4), dict(block_size=24), dict(block_size=512),
                                    dict(n_kv_heads=0), dict(n_q_heads=12), dict(n_q_heads=2048), dict(n_q_heads=4),
                                    dict(head_dim=96), dict(head_dim=512), dict(type=2), dict(max_rows=0)])
def test_create_refuses(kv, change):
    good = dict(n_blocks=10, block_size=16, n_q_heads=16, n_kv_heads=8, head_dim=128, type=0, max_rows=4)
    with pytest.raises(kv.IsjlError) as e:
        kv.isjl_kv_create(**dict(good, **change))
    assert e.value.status == kv.ISJL_ERR_INVALID_ARG


def test_null_handles(kv):
    L = kv.lib()
    a, c = kv.isjl_kv_assign_args(), kv.isjl_kv_cache()
    assert L.isjl_kv_create(None, None) == kv.ISJL_ERR_INVALID_ARG
    assert L.isjl_kv_assign(None, ctypes.byref(a), None) == kv.ISJL_ERR_INVALID_ARG
    assert L.isjl_kv_append(None, None, ctypes.byref(c), None) == kv.ISJL_ERR_INVALID_ARG
    assert L.isjl_kv_attend(None, None, ctypes.byref(c), None) == kv.ISJL_ERR_INVALID_ARG
    assert L.isjl_kv_status(None) == kv.ISJL_ERR_INVALID_ARG
    L.isjl_kv_destroy(None)
