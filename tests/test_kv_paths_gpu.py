"""The sizes from which the decode step's calls take another kernel, grid or split: both sides of each rule are run
and compared with 64 bits, and the launches say which side it was."""
import ctypes

import numpy as np
import pytest

import kv_plain
from conftest import cuda_available
from test_kv_attend_gpu import check, decoder, inputs
from test_kv_edges_gpu import long_runs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


class KernelNode(ctypes.Structure):
    """CUDA_KERNEL_NODE_PARAMS of cuda.h (version 2)."""
    _fields_ = [("func", ctypes.c_void_p)] + [(f, ctypes.c_uint) for f in ("gx", "gy", "gz", "bx", "by", "bz", "shared")] + [
        (f, ctypes.c_void_p) for f in ("params", "extra", "kern", "ctx")]


def launches(call):
    """[(kernel's name, blocks, threads)] of a call, as a graph records them.  The call has run before."""
    import torch
    cu = ctypes.CDLL("libcuda.so.1")
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, count = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert cu.cuGraphGetNodes(raw, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert cu.cuGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    out = []
    for node in nodes:
        kind, p, name = ctypes.c_int(), KernelNode(), ctypes.c_char_p()
        assert cu.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value:
            continue                             # not a kernel
        assert cu.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(p)) == 0
        get, what = (cu.cuKernelGetName, p.kern) if p.kern else (cu.cuFuncGetName, p.func)
        assert get(ctypes.byref(name), ctypes.c_void_p(what)) == 0
        out.append((name.value.decode(), p.gx, p.bx))
    return out


def blocks_of(found, name):
    """Blocks of the kernel of that name, 0 if it was not launched."""
    at = [x for x in found if name in x[0]]
    assert len(at) <= 1
    return at[0][1] if at else 0


def sms():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("n,shared,apart", [(2, 4095, False), (2, 4096, True), (7, 682, False), (7, 683, True), (8, 219, False),
                                            (8, 220, True), (9, 191, False), (9, 192, True)])
def test_prefix_apart(n, shared, apart):
    """The prefix's own kernel from (n - 1) times its tokens = 32,768, with 8 queries or more 12,288."""
    s = inputs([20 + 7 * i for i in range(n)], 8, 2, 64, 8, shared=shared, seed=n)
    d = decoder(s)
    check(s, d)
    found = launches(lambda: d.attend(**s))
    assert (blocks_of(found, "prefix_kernel") > 0) == apart and len(found) == 2 + apart


def test_prefix_is_not_apart():
    """With a window, with heads of 256 values, with more query heads on a key head than a tile has rows."""
    for hq, hkv, dim, kw in ((8, 2, 64, dict(window=100)), (8, 2, 256, {}), (130, 1, 64, {})):
        s = inputs([9] * 20, hq, hkv, dim, 64, shared=20)
        d = decoder(s)
        check(s, d, **kw)
        assert not blocks_of(launches(lambda: d.attend(**s, **kw)), "prefix_kernel")


@pytest.mark.parametrize("n", [1, 3900, 3960, 3975, 4096])
def test_queries_that_leave_room_for_one_block_less(n):
    """Blocks of the attention hold 4 bytes a query: with the most queries one block less fits an SM."""
    s = inputs(np.arange(n) % 50 + 1, 2, 1, 128, 16, seed=n)
    d = decoder(s)
    check(s, d)
    got = blocks_of(launches(lambda: d.attend(**s)), "attend_kernel")
    assert got == (2 * sms() if n <= 3960 else sms())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,hq,hkv,shared,longest,split", [
    (128, 16, 2, 40, 256, "short"),              # 16 items of 20 tiles on 64 SMs
    (300, 128, 8, 18, 60, "short"),              # 152 items of 9 tiles: more than the SMs of a short prefix
    (128, 128, 2, 256, 3070, "fine"),            # 64 items of 128 tiles beside tables for 48 blocks of own tokens
    (128, 128, 2, 256, 60, "alone")])            # beside tables for one block
def test_shares_of_the_sms(n, hq, hkv, shared, longest, split, dim):
    """A short prefix beside own tokens on SMs of their own; a long one on all SMs but a few, with finer blocks for the
    own tokens, or on all of them where those are few."""
    s = inputs([longest] + [1 + i % 60 for i in range(n - 1)], hq, hkv, dim, 64, shared=shared, seed=n)
    d = decoder(s)
    check(s, d)
    found = launches(lambda: d.attend(**s))
    plain = blocks_of(launches(lambda: d.attend(**dict(s, prefix=None))), "attend_kernel") // sms()
    prefix, own = blocks_of(found, "prefix_kernel"), blocks_of(found, "attend_kernel")
    if split == "short":
        assert 0 < prefix <= 72 * sms() // 152 and own == plain * (sms() - prefix)
    elif split == "fine":
        assert sms() // 2 < prefix < sms() and own == 4 * plain * sms()
    else:
        assert prefix == sms() and own == plain * sms()


def test_pieces_joined_three_or_twelve_at_a_time():
    """Both joins, with and without a prefix's pieces."""
    for lens, shared, batch in (([3000], 0, 12), ([40] * 700, 0, 3), ([9] * 40, 256, 12), ([9] * 900, 40, 3)):
        s = inputs(lens, 16, 2, 64, 64, shared=shared, seed=len(lens))
        d = decoder(s)
        check(s, d)
        names = [x[0] for x in launches(lambda: d.attend(**s))]
        assert any("join_kernel" in x and "Li%dE" % batch in x for x in names) and len(names) == 2 + (shared > 0)


@pytest.mark.parametrize("n,threads", [(1, 128), (3647, 128), (3648, 32)])
def test_warps_of_a_token(n, threads):
    """append: four warps a token, one where there are 24 tokens or more for each SM."""
    import torch
    from paper_2608_02244_gb300 import kv
    assert 24 * sms() == 3648
    s = dict(qkv=torch.randn(n, 8 * 64, device="cuda").bfloat16(), slots=torch.arange(n, device="cuda"),
             k=torch.zeros(460, 8, 2, 64, device="cuda").bfloat16(), v=torch.zeros(460, 8, 2, 64, device="cuda").bfloat16())
    d = kv.Decoder(460, 8, 4, 2, 64, max_rows=1)
    q = d.append(positions=None, **s)
    assert torch.equal(q.view(n, -1), s["qkv"][:, :256]) and torch.equal(s["v"].view(-1, 128)[:n], s["qkv"][:, 384:])
    found = launches(lambda: d.append(positions=None, **s))
    assert [x[1:] for x in found] == [(n, threads)]


@pytest.mark.parametrize("rows,room,kernels", [(1024, 4096, 1), (1025, 4096, 2), (1024, 4097, 2), (1, 1, 1), (3, 9000, 2)])
def test_kernels_of_assign(rows, room, kernels):
    import torch
    from paper_2608_02244_gb300 import kv
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rng = np.random.default_rng(rows)
    lens = rng.integers(0, 17, rows)
    new = np.where(rng.random(rows) < 0.1, -1, rng.integers(0, 4, rows))
    held = -(-lens // 8)
    ids = rng.permutation(int(held.sum()) + rows)
    table = np.full((rows, 3), -1)
    table[np.arange(3)[None] < held[:, None]] = ids[:held.sum()]
    free = np.concatenate([ids[held.sum():], np.zeros(held.sum(), int)])
    d = kv.Decoder(len(free), 8, 1, 1, 64, max_rows=rows)
    t, f = i32(table), i32(free)
    p = d.assign(i32(lens), i32(new), t, f, i32([rows]), room)
    assert d.status() == 0
    want = kv_plain.assign(lens.tolist(), new.tolist(), table.tolist(), free.tolist(), rows, 8, room)
    for name in p._fields:
        assert getattr(p, name).tolist() == want[name], name
    a = [i32(lens), i32(new), i32(table), i32(free), i32([rows])]
    d.assign(*a, room)
    found = launches(lambda: d.assign(*a, room))
    assert len(found) == kernels and found[-1][0].count("assign_kernel" if kernels == 1 else "fill_kernel")


@pytest.mark.parametrize("dim,dtype", [(64, "float16"), (128, "bfloat16"), (64, "bfloat16"), (128, "float16")])
@pytest.mark.parametrize("shape", ["rising", "falling", "steps", "one late"])
def test_maxima_that_move_within_a_run(dim, dtype, shape):
    """Scores that grow along the ten tiles of a block's run, so that its sums are rescaled, some of the rows' by some
    of the tiles."""
    import torch
    s = long_runs(dim, dtype, seed=1)
    x = torch.linspace(0, 1, 40 * 64, device="cuda")
    size = {"rising": 6 * x, "falling": 6 * (1 - x), "steps": 8 * (x * 5).floor() / 5,
            "one late": torch.where(x > 0.45, 6.0, 0.3)}[shape].view(40, 64, 1, 1)
    b = s["prefix"].long()
    s["k"][b] = (s["k"][b] * size).to(s["k"].dtype)
    check(s)
