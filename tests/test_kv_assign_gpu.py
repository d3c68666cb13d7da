"""Block tables and slot maps against a stack of blocks served row by row."""
import numpy as np
import pytest

import kv_plain
from conftest import cuda_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


def step(n, block, width, pool, room, seed, fresh=0.2, ended=0.2, idle=0.2, longest=None):
    """Random rows whose held blocks fit the pool; some rows ask for more than a table row holds."""
    rng = np.random.default_rng(seed)
    longest = longest or width * block
    lens = rng.integers(0, longest + 1, n)
    held = -(-lens // block)
    while held.sum() > pool:
        lens[np.argmax(held)] //= 2
        held = -(-lens // block)
    kind = rng.random(n)
    new = np.where(kind < ended, -1, np.where(kind < ended + idle, 0, np.where(
        kind < ended + idle + fresh, rng.integers(1, longest + 2, n), 1)))
    ids = rng.permutation(pool)
    table = np.full((n, width), -1)
    table[np.arange(width)[None] < held[:, None]] = ids[:held.sum()]
    free = np.full(pool, -1)
    free[:pool - held.sum()] = ids[held.sum():]
    return lens, new, table, free, pool - int(held.sum()), room


def on_gpu(x, shape=None):
    import torch
    t = torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    return t if shape is None else t.reshape(shape)


def run(case, block, prefix=0, in_place=False, decoder=None, stream=None):
    import torch
    from paper_2608_02244_gb300 import kv
    lens, new, table, free, n_free, room = case
    d = decoder or kv.Decoder(len(free), block, 1, 1, 64, max_rows=max(1, len(lens)))
    t = [on_gpu(x) for x in (lens, new)] + [on_gpu(table, (len(lens), -1) if len(lens) else (0, 4)), on_gpu(free), on_gpu([n_free])]
    torch.cuda.synchronize()
    p = d.assign(*t, room, prefix_len=prefix, in_place=in_place, stream=stream)
    assert d.status() == 0
    got = {f: getattr(p, f).tolist() for f in p._fields}
    got.update(table=t[2].tolist(), free=t[3].tolist())
    if in_place:
        assert t[0].tolist() == got["lens"] and t[4].tolist() == got["n_free"]
    else:
        assert t[0].tolist() == list(lens) and t[4].tolist() == [n_free]
    return got


def check(case, block, **kw):
    lens, new, table, free, n_free, room = case
    want = kv_plain.assign(list(map(int, lens)), list(map(int, new)), np.asarray(table).tolist(), list(map(int, free)), n_free,
                           block, room, kw.get("prefix", 0))
    got = run(case, block, **kw)
    for f in want:
        assert got[f] == want[f], f


@pytest.mark.parametrize("n", [1, 2, 31, 33, 256, 1000, 1023, 1024, 1025, 2999, 4096, 4097, 5000])
def test_rows(n):
    check(step(n, 16, 9, 6 * n + 3, 60 * n + 5, n), 16)


@pytest.mark.parametrize("room", [1, 5, 4095, 4096, 4097, 4100])
@pytest.mark.parametrize("n", [40, 1024, 1025])
def test_around_one_kernel(n, room):
    """Both sides of the sizes up to which one kernel does it all; maps of odd lengths."""
    check(step(n, 8, 30, 20 * n, room, n + room), 8, prefix=16)


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("in_place", [False, True])
def test_blocks(block, in_place):
    check(step(77, block, 5, 300, 40000, block), block, prefix=3 * block, in_place=in_place)


@pytest.mark.parametrize("seed", range(6))
def test_pool_or_maps_too_small(seed):
    """Rows past the first that does not fit get nothing, except those that need no block."""
    case = step(300, 8, 20, 1500, 2000 if seed % 2 else 10**5, seed, fresh=0.5, ended=0.05)
    check(case, 8)


def test_long_rows():
    """Rows of many blocks and maps of many tokens: the parts that more than one block of threads fills."""
    check(step(40, 8, 4000, 90000, 700001, 3, fresh=0.6, longest=30000), 8)


def test_fill_from_nothing_and_empty():
    n = 500
    check((np.zeros(n, int), np.arange(n) % 70, np.full((n, 10), -1), np.arange(3000)[::-1].copy(), 3000, 20000), 8)
    check((np.zeros(0, int), np.zeros(0, int), np.zeros((0, 4), int), np.arange(7), 7, 5), 8)
    check((np.full(9, 64), np.full(9, -1), np.arange(72).reshape(9, 8), np.full(72, -1), 0, 3), 8)   # all end


def test_blocks_given_back_are_taken_in_the_same_step():
    lens, new = [16, 0, 24, 0], [-1, 20, -1, 30]
    table = np.array([[0, 1, -1, -1], [-1] * 4, [2, 3, 4, -1], [-1] * 4])
    check((lens, new, table, np.full(7, -1) * 1, 0, 64), 8)


def test_repeats():
    """The same inputs give the same outputs, and a step without in_place leaves its inputs as they were."""
    case = step(400, 16, 30, 9000, 30000, 9)
    assert run(case, 16) == run(case, 16)


def test_steps_follow_one_another():
    """A few steps in place keep every block in exactly one place."""
    import torch
    from paper_2608_02244_gb300 import kv
    rng = np.random.default_rng(4)
    n, block, width, pool = 64, 8, 40, 1200
    d = kv.Decoder(pool, block, 1, 1, 64, max_rows=n)
    lens, table, free, n_free = on_gpu(np.zeros(n)), on_gpu(np.full((n, width), -1)), on_gpu(rng.permutation(pool)), on_gpu([pool])
    for _ in range(30):
        have = lens.cpu().numpy()
        new = np.where(have == 0, rng.integers(0, 200, n), np.where(rng.random(n) < 0.1, -1, 1))
        d.assign(lens, on_gpu(new), table, free, n_free, 5000, in_place=True)
        assert d.status() == 0
        have, k = -(-lens.cpu().numpy() // block), int(n_free)
        held = torch.cat([table[i, :have[i]] for i in range(n)]).tolist()
        assert sorted(held + free[:k].tolist()) == list(range(pool))


def test_reports_invalid_values():
    from paper_2608_02244_gb300 import kv
    for lens, n_free in (([5, -1, 3], 2), ([5, 99, 3], 2), ([5, 2, 3], 99), ([5, 2, 3], -1)):
        d = kv.Decoder(20, 8, 1, 1, 64, max_rows=3)
        table = on_gpu(np.arange(12).reshape(3, 4))
        p = d.assign(on_gpu(lens), on_gpu([1, 1, 1]), table, on_gpu(np.arange(20)), on_gpu([n_free]), 8)
        assert d.status() == kv.ISJL_ERR_INVALID_ARG and d.status() == 0
        assert p.granted.tolist() == [1, 0 if not 0 <= lens[1] <= 32 else 1, 1]


def test_reports_more_blocks_than_there_are():
    """Rows that end with more blocks than the pool has: the list takes what it can hold, nothing beyond it is touched."""
    import torch
    from paper_2608_02244_gb300 import kv
    for n, width in ((3, 12), (1500, 40000)):                  # sums beyond the pool, and beyond 32 bits
        d = kv.Decoder(20, 256, 1, 1, 64, max_rows=n)
        lens = torch.full((n,), width * 256, dtype=torch.int32, device="cuda")
        table = torch.zeros((n, width), dtype=torch.int32, device="cuda")
        new = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        new[n // 2], lens[n // 2] = 700, 0
        p = d.assign(lens, new, table, on_gpu(np.arange(20)), on_gpu([4]), 1024)
        assert d.status() == kv.ISJL_ERR_INVALID_ARG
        assert int(p.n_free) == 17 and p.granted[n // 2] == 700 and (p.slots[:700] >= 0).all()


def test_refusals():
    import torch
    from paper_2608_02244_gb300 import kv
    d = kv.Decoder(20, 8, 1, 1, 64, max_rows=3)
    good = dict(lens=on_gpu([1, 2, 3]), new_tokens=on_gpu([1, 1, 1]), table=on_gpu(np.zeros((3, 4))), free=on_gpu(np.zeros(20)),
                n_free=on_gpu([0]), max_tokens=4)
    d.assign(**good)
    for bad in (dict(lens=good["lens"].long()), dict(lens=on_gpu([1] * 6)[::2]), dict(lens=good["lens"].cpu()), dict(max_tokens=0),
                dict(new_tokens=on_gpu([1, 1])), dict(table=on_gpu(np.zeros((2, 4)))), dict(free=on_gpu(np.zeros(19))),
                dict(n_free=on_gpu([0, 0])), dict(prefix_len=-1), dict(prefix_len=2**31 - 8)):
        with pytest.raises(kv.IsjlError) as e:
            d.assign(**dict(good, **bad))
        assert e.value.status == kv.ISJL_ERR_INVALID_ARG
    with pytest.raises(kv.IsjlError):
        d.assign(on_gpu([1] * 4), on_gpu([1] * 4), on_gpu(np.zeros((4, 4))), good["free"], good["n_free"], 4)
    torch.cuda.synchronize()
