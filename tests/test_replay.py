"""Replays of simulated schedules: table rows and new tokens by step (CPU), and the steps themselves (GPU)."""
import numpy as np
import pytest

import kv_plain
from conftest import cuda_available

gpu = [pytest.mark.gpu, pytest.mark.skipif(not cuda_available(), reason="needs a GPU")]


def schedule(seed, n=60, slots=8, horizon=300):
    """Requests that start when one of the slots is free, some not at all."""
    rng = np.random.default_rng(seed)
    start, completion = np.full(n, -1), np.full(n, -1)
    free_at = np.zeros(slots, int)
    for i in range(n):
        if rng.random() < 0.1:
            continue
        w = int(np.argmin(free_at))
        start[i] = free_at[w] + rng.integers(0, 4)
        completion[i] = start[i] + rng.integers(1, 60)
        free_at[w] = completion[i]
    return start, completion


@pytest.mark.parametrize("seed", range(8))
def test_rows_and_tokens(seed):
    from paper_2608_02244_gb300 import replay
    start, completion = schedule(seed)
    rows, count = replay.rows_of(start, completion)
    assert count <= 16                        # those running and those that have just ended
    first, last = start[rows >= 0].min(), completion.max() + 1
    new = replay.new_tokens(start, completion, rows, count, first, last)
    held = np.zeros(count, int)
    owner = np.full(count, -1)
    for k in range(first, last):
        for i in range(start.size):
            if rows[i] < 0:
                assert start[i] < 0
                continue
            x = new[k - first, rows[i]]
            if start[i] <= k < completion[i]:
                assert x == 1 and owner[rows[i]] in (-1, i)
                owner[rows[i]] = i
            elif k == completion[i]:
                assert x == -1 and owner[rows[i]] == i
        held += new[k - first] == 1
        for r in np.nonzero(new[k - first] == -1)[0]:
            i = owner[r]
            assert held[r] == completion[i] - start[i]
            held[r], owner[r] = 0, -1
    assert not held.any()


def test_fit():
    from paper_2608_02244_gb300 import replay
    running = np.array([0, 1, 2, 3, 2])
    max_r, sum_r = np.array([0, 5, 9, 4, 1]), np.array([0, 5, 12, 9, 2])
    f = replay.fit({"running": running, "max_r": max_r, "sum_r": sum_r, "seconds": 2e-5 + 3e-8 * sum_r})
    assert np.allclose(f["sum"], (2e-5, 3e-8, 1.0)) and f["max"][2] < 1


class TestGpu:
    pytestmark = gpu

    def test_every_step(self):
        """Each step of a schedule: lengths are the model's r, outputs are attention in 64 bits, all blocks return."""
        import torch
        from paper_2608_02244_gb300 import replay
        start, completion = schedule(3, n=20, slots=5)
        r = replay.Replay(start, completion, n_q_heads=8, n_kv_heads=2, head_dim=64, block_size=8, prefix=24)
        new = replay.new_tokens(start, completion, r.rows, r.n_rows, r.first, r.last)
        for k, x in enumerate(new, r.first):
            r.new.copy_(torch.from_numpy(x))
            plan, q, out = r.step()
            want = np.zeros(r.n_rows, int)
            for s, c, w in zip(start, completion, r.rows):
                if w >= 0 and s <= k < c:
                    want[w] = k - s + 1
            assert r.lens.tolist() == want.tolist()
            assert (plan.granted.cpu().numpy() == (x > 0)).all()
            if k % 7 == 0:
                w, _, size = kv_plain.attend(q, r.k, r.v, r.table, plan.visible, plan.rows, r.prefix_blocks)
                assert ((out.double() - w).abs() <= (2 * kv_plain.UNIT[out.dtype] + kv_plain.REST) * size + 2.0 ** -24).all()
        assert r.decoder.status() == 0 and int(r.n_free) == r.blocks
        assert sorted(r.free[:r.blocks].tolist()) == list(range(r.blocks))
        r.close()

    @pytest.mark.parametrize("kw", [dict(), dict(prefix=160), dict(window=40, sinks=2)])
    def test_graph_is_the_steps(self, kw):
        """The graph's steps leave what the single calls leave."""
        import torch
        from paper_2608_02244_gb300 import replay, sim, workloads
        a, p, o = workloads.generate(1)
        S = sim.Simulator(1, 200, 32)
        res = S.sweep(a, p, o, ["isjl"], [32], 2048, per_request=True)
        S.close()
        start, completion = res["start"][0, 0], res["completion"][0, 0]
        one = replay.Replay(start, completion, n_q_heads=8, n_kv_heads=2, **kw)
        two = replay.Replay(start, completion, n_q_heads=8, n_kv_heads=2, **kw)
        times = one.run(150)
        for x in replay.new_tokens(start, completion, two.rows, two.n_rows, two.first, two.first + 150):
            two.new.copy_(torch.from_numpy(x))
            plan, q, out = two.step()
        assert torch.equal(one.result[2], out) and torch.equal(one.lens, two.lens) and torch.equal(one.k, two.k)
        assert torch.equal(one.table, two.table) and int(one.n_free) == int(two.n_free)
        assert times["running"].max() <= 32 and (times["seconds"] > 0).all()
        again = one.run()
        assert again["sum_r"][:150].tolist() == times["sum_r"].tolist() and int(one.n_free) == one.blocks
        for i in (one, two):
            i.close()

    def test_command(self, capsys):
        from paper_2608_02244_gb300 import replay
        replay.main(["--workload", "1", "--policy", "fcfs", "--steps", "40", "--heads", "8", "2", "64"])
        out = capsys.readouterr().out
        assert "single-200" in out and "sum r" in out

    def test_refuses(self):
        from paper_2608_02244_gb300 import replay
        with pytest.raises(ValueError):
            replay.Replay([-1, -1], [-1, -1])
        with pytest.raises(ValueError):
            replay.Replay([0], [5], prefix=10)
