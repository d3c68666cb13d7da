"""Runs a simulated schedule on the GPU: the decode steps behind the model's costs.

The simulator charges a step c + tau * |S| * max r.  ``Replay`` performs the
steps of a schedule (start and completion steps, as the simulator returns them)
with the KV memory and the attention that they stand for: in step k every
request that runs gets its next token (r_i = k - start_i + 1 tokens so far), for
which ``kv.Decoder`` finds a slot, writes key and value, and attends over the
request's tokens.  One CUDA graph holds a step; per step only the list of new
tokens is copied.  ``fit`` then gives the card's own c and tau, and how well the
times go with |S| * max r (the model's driver) and with sum r (the tokens read).

    res = Simulator(1, 1000, B).sweep(a, p, o, ["isjl"], [64], kv_cap, per_request=True)
    r = replay.Replay(res["start"][0, 0], res["completion"][0, 0], B)
    times = r.run()
    print(replay.fit(times))

    python -m paper_2608_02244_gb300.replay --workload 1 --policy isjl --delta 32
"""
from __future__ import annotations

import numpy as np


def rows_of(start, completion):
    """A table row for each request that runs (-1: none).  A row ends in the step after its
    request's last and is taken again no earlier than in the step after that, so that one
    step never both ends and starts a row."""
    start, completion = np.asarray(start, np.int64), np.asarray(completion, np.int64)
    rows, ends, free = np.full(start.size, -1, np.int64), [], []
    count = 0
    for i in np.lexsort((np.arange(start.size), start)):
        if start[i] < 0 or completion[i] <= start[i]:
            continue
        while ends and ends[0][0] < start[i]:
            free.append(ends.pop(0)[1])
        if free:
            free.sort()
            rows[i] = free.pop(0)
        else:
            rows[i], count = count, count + 1
        ends.append((completion[i], rows[i]))
        ends.sort()
    return rows, count


def new_tokens(start, completion, rows, count, first, last):
    """[last - first, count]: 1 for a row whose request runs in the step, -1 where it ended
    with the step before, else 0."""
    out = np.zeros((last - first, count), np.int32)
    for s, c, r in zip(start, completion, rows):
        if r < 0:
            continue
        out[max(0, s - first):max(0, c - first), r] = 1
        if first <= c < last:
            out[c - first, r] = -1
    return out


class Replay:
    """The steps of one schedule.  Weights and hidden states are not simulated: the new
    tokens' projections are random numbers, the same in every step."""

    def __init__(self, start, completion, n_q_heads=32, n_kv_heads=8, head_dim=128, block_size=16, dtype=None, prefix=0,
                 window=0, sinks=0, seed=0):
        import torch
        from . import kv
        self.torch = torch
        self.start = np.asarray(start, np.int64).ravel()
        self.completion = np.asarray(completion, np.int64).ravel()
        self.rows, n = rows_of(self.start, self.completion)
        live = self.rows >= 0
        if not live.any():
            raise ValueError("no request of the schedule runs")
        if prefix % block_size:
            raise ValueError("prefix must be a multiple of block_size")
        self.first, self.last = int(self.start[live].min()), int(self.completion[live].max()) + 1
        longest = int((self.completion - self.start)[live].max())
        self.n_rows, self.block_size, self.prefix = n, block_size, prefix
        width = -(-longest // block_size)
        blocks = n * width if n * width < 4096 else self._most_blocks()
        shared = prefix // block_size
        dtype = torch.bfloat16 if dtype is None else dtype
        self.decoder = kv.Decoder(blocks + shared, block_size, n_q_heads, n_kv_heads, head_dim, dtype=dtype, max_rows=n)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rn = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
        self.k, self.v = (rn(blocks + shared, block_size, n_kv_heads, head_dim) for _ in range(2))
        self.qkv = rn(n, (n_q_heads + 2 * n_kv_heads) * head_dim)
        self.q_weight, self.k_weight = rn(head_dim), rn(head_dim)
        angle = torch.arange(prefix + longest, device="cuda")[:, None] * 10000.0 ** (
            -torch.arange(0, head_dim, 2, device="cuda") / head_dim)
        self.rope = torch.cat((angle.cos(), angle.sin()), 1).float()
        i32 = dict(dtype=torch.int32, device="cuda")
        self.prefix_blocks = torch.arange(blocks, blocks + shared, **i32) if shared else None
        self.attend_args = dict(prefix=self.prefix_blocks, window=window, sinks=sinks)
        self.lens, self.new = torch.zeros(n, **i32), torch.zeros(n, **i32)
        self.table = torch.full((n, width), -1, **i32)
        self.free = torch.zeros(blocks + shared, **i32)
        self.free[:blocks] = torch.arange(blocks - 1, -1, -1, **i32)
        self.n_free = torch.tensor([blocks], **i32)
        self.blocks = blocks
        self.graph = None

    def _most_blocks(self):
        """Blocks that the schedule holds at most: of each request ceil(r / block_size), given
        back in the step after its last."""
        change = np.zeros(self.last - self.first + 1, np.int64)
        for s, c, r in zip(self.start - self.first, self.completion - self.first, self.rows):
            if r >= 0:
                change[s:c:self.block_size] += 1
                change[c] -= -(-(c - s) // self.block_size)
        # a step's ending rows give their blocks back before its new ones are taken
        return int(np.cumsum(change).max())

    def step(self):
        """One step for the new tokens in ``new``; returns its plan, queries and outputs."""
        d = self.decoder
        plan = d.assign(self.lens, self.new, self.table, self.free, self.n_free, self.n_rows, prefix_len=self.prefix, in_place=True)
        q = d.append(self.qkv, plan.positions, plan.slots, self.k, self.v, self.rope, self.q_weight, self.k_weight)
        out = d.attend(q, self.k, self.v, self.table, plan.visible, rows=plan.rows, **self.attend_args)
        return plan, q, out

    def _capture(self):
        torch = self.torch
        self.new.zero_()                          # a step of no tokens changes nothing
        self.step()
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.result = self.step()

    def run(self, steps=None):
        """Replay the first `steps` steps (all by default) from the start.  Returns arrays by
        step: running (|S|), max_r, sum_r, seconds (of the step's kernels on the GPU)."""
        torch = self.torch
        last = self.last if steps is None else min(self.last, self.first + int(steps))
        new = new_tokens(self.start, self.completion, self.rows, self.n_rows, self.first, last)
        if self.graph is None:
            self._capture()
        self.lens.zero_()
        self.n_free.fill_(self.blocks)
        self.free[:self.blocks] = torch.arange(self.blocks - 1, -1, -1, dtype=torch.int32, device="cuda")
        plan = torch.from_numpy(new).cuda()
        events = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in new]
        for row, (a, b) in zip(plan, events):
            self.new.copy_(row)
            a.record()
            self.graph.replay()
            b.record()
        status = self.decoder.status()
        if status:
            from .sim import IsjlError
            raise IsjlError(status, "replay")
        r = np.zeros(new.shape[1], np.int64)
        running, max_r, sum_r = (np.zeros(len(new), np.int64) for _ in range(3))
        for k, x in enumerate(new):
            r[x < 0] = 0
            r += x > 0
            on = r[x > 0]
            running[k], max_r[k], sum_r[k] = on.size, on.max(initial=0), on.sum()
        return {"running": running, "max_r": max_r, "sum_r": sum_r,
                "seconds": np.array([a.elapsed_time(b) for a, b in events]) * 1e-3}

    def close(self):
        self.graph = None
        self.decoder.close()


def fit(times):
    """Least squares of the nonempty steps' times: {driver: (c, tau, r2)} for seconds = c + tau * driver with
    driver |S| * max r ("max") and sum r ("sum").  Steps of equal driver throughout give tau 0."""
    on = times["running"] > 0
    y = times["seconds"][on]
    out = {}
    for name, x in (("max", times["running"] * times["max_r"]), ("sum", times["sum_r"])):
        x = x[on].astype(np.float64)
        dx, dy = x - x.mean(), y - y.mean()
        tau = float(dx @ dy / (dx @ dx)) if dx @ dx > 0 else 0.0
        c = float(y.mean() - tau * x.mean())
        rest = dy - tau * dx
        out[name] = (c, tau, float(1 - rest @ rest / (dy @ dy)) if dy @ dy > 0 else 1.0)
    return out


def main(argv=None):
    import argparse
    from . import sim, workloads
    ap = argparse.ArgumentParser(description="Replay one simulated instance's decode steps on the GPU.")
    ap.add_argument("--workload", type=int, default=1)
    ap.add_argument("--instance", type=int, default=0)
    ap.add_argument("--policy", default="isjl", choices=sorted(sim.POLICY))
    ap.add_argument("--delta", type=int, default=None)
    ap.add_argument("--steps", type=int, default=None)
    ap.add_argument("--prefix", type=int, default=0, help="tokens of a prefix that all requests share")
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--block-size", type=int, default=16)
    ap.add_argument("--heads", type=int, nargs=3, default=(32, 8, 128), metavar=("Q", "KV", "DIM"))
    x = ap.parse_args(argv)
    wl = workloads.WORKLOADS[x.workload]
    a, p, o, count = workloads.generate(x.workload, [x.instance], with_counts=True)
    delta = wl.deltas[0] if x.delta is None else x.delta
    S = sim.Simulator(1, wl.n_per_instance, wl.B[0])
    try:
        res = S.sweep(a, p, o, [x.policy], [delta], wl.kv_caps[0], per_request=True, counts=count)
    finally:
        S.close()
    r = Replay(res["start"][0, 0], res["completion"][0, 0], *x.heads, block_size=x.block_size, prefix=x.prefix,
               window=x.window, sinks=x.sinks)
    try:
        r.run(min(x.steps or 64, 64))              # clocks and caches
        times = r.run(x.steps)
    finally:
        r.close()
    on = times["running"] > 0
    print("%s instance %d, %s delta %d: %d steps, at most %d running, %.1f us a step (median), %.3f s in all" % (
        wl.name, x.instance, x.policy, delta, on.sum(), times["running"].max(), 1e6 * np.median(times["seconds"][on]),
        times["seconds"].sum()))
    for name, (c, tau, r2) in fit(times).items():
        print("seconds = c + tau * %s: c %.3g, tau %.3g, r2 %.3f" % ({"max": "|S| max r", "sum": "sum r"}[name], c, tau, r2))


if __name__ == "__main__":
    main()
