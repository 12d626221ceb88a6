"""What a served model costs on this device, and the placement that follows.

The placement searches take each model's latency and bytes as inputs (Sec. 4.1
profiles them per configuration; Table 1 lists them).  For models that
generate, this module measures them: a decoder block whose linear layers hold
weights of 8 bits and whose requests hold caches of 4 bits, cut back to a budget
by accumulated attention weight, runs its steps on the GPU; the step's time at a
few batch sizes gives a request's latency and the batching slope, the block's
arrays give the bytes.  The budget makes both constants of the model: an
unbounded cache has no fixed size, and its step no fixed time, which the
admission rule of Sec. 4.3 needs.

`python -m paper_2302_11665_amd.served` measures two small models and prints
the placement that the partition search chooses for them.
"""
from __future__ import annotations

import dataclasses

import numpy as np

from . import sim
from .workload import gen, problems

MIB = 1 << 20


@dataclasses.dataclass(frozen=True)
class Shape:
    """A decoder of `layers` equal blocks."""
    layers: int
    hidden: int
    heads: int
    kv_heads: int
    dim: int
    inner: int          # width of the feed-forward layer
    budget: int         # tokens that a request's cache keeps
    slack: int = 64     # tokens that it may grow by before it is cut back, at least 1
    recent: int = 64    # newest tokens that a cut always keeps
    group: int = 64
    page: int = 64

    def __post_init__(self):
        if self.budget < 1 or self.slack < 1 or self.recent < 0:
            raise ValueError(f"a cache of {self.budget} tokens that grows by {self.slack}, the newest {self.recent} kept")


class Block:
    """One decoder block's weights, and its step over the caches of a batch."""

    def __init__(self, shape: Shape, seed: int = 0, device="cuda"):
        import torch
        from . import ops
        self.shape, self.device = shape, device
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(n_out, n_in):
            return ops.pack_weight(torch.randn(n_out, n_in, device=device, generator=g) * n_in ** -0.5)

        s = shape
        self.qkv = weight((s.heads + 2 * s.kv_heads) * s.dim, s.hidden)
        self.out = weight(s.hidden, s.heads * s.dim)
        self.up = weight(s.inner, s.hidden)
        self.down = weight(s.hidden, s.inner)

    @property
    def nbytes(self) -> int:
        return sum(w.nbytes for w in (self.qkv, self.out, self.up, self.down))

    def step(self, x, caches: "Caches"):
        """One token of every sequence: x [seqs, hidden] (bf16) to the block's
        output, the caches advanced by it."""
        import torch
        from . import ops
        s = self.shape
        qkv = ops.linear_i8(_normed(x), self.qkv).view(-1, 1, s.heads + 2 * s.kv_heads, s.dim)
        o = caches.attend(qkv[:, :, :s.heads], qkv[:, :, s.heads:s.heads + s.kv_heads], qkv[:, :, s.heads + s.kv_heads:])
        x = x + ops.linear_i8(o.view(-1, s.heads * s.dim), self.out)
        h = torch.nn.functional.gelu(ops.linear_i8(_normed(x), self.up))
        return x + ops.linear_i8(h, self.down)


def _normed(x):
    """Rows of mean square 1."""
    f = x.float()
    return (f * (f.square().mean(-1, keepdim=True) + 1e-6).rsqrt()).to(x.dtype)


class Caches:
    """The caches of a batch of sequences in one block: they grow token by token
    and are cut back to the budget when budget + slack is reached, into a second
    set of pages (the first is the next cut's)."""

    def __init__(self, shape: Shape, n_seqs: int, device="cuda"):
        import torch
        from . import ops
        s = self.shape = shape
        per = -(-(s.budget + s.slack) // s.page)  # pages of a sequence

        def cache():
            table = torch.arange(n_seqs * per, dtype=torch.int32, device=device).view(n_seqs, per)
            return ops.Cache.empty(n_seqs * per, s.kv_heads, s.dim, table, group=s.group, page=s.page, device=device)

        self.now, self.spare = cache(), cache()
        self.length = torch.zeros(n_seqs, dtype=torch.int32, device=device)  # tokens in the caches
        self.total = torch.zeros_like(self.length)                           # tokens so far
        self.held = 0  # length of all of them, on the host

    def bytes_per_sequence(self) -> int:
        """Of both sets of pages."""
        return 2 * self.now.bytes_per_slot * self.now.page_table.shape[1] * self.shape.page

    def attend(self, q, k, v):
        """Append one token's keys and values, attend, and cut back if due."""
        from . import ops
        s = self.shape
        if self.held == s.budget + s.slack:
            self.length.copy_(ops.cache_evict(self.now, self.spare, self.length, self.total, keep=s.budget,
                                              recent=min(s.recent, s.budget)))
            self.now, self.spare = self.spare, self.now
            self.held = s.budget
        ops.cache_append(self.now, k, v, self.length, first_pos=self.total)
        self.length.add_(1)  # in place: a captured step is replayed on the same numbers
        self.total.add_(1)
        self.held += 1
        return ops.attention_kv4(q, self.now, self.length, acc_in=self.now.acc, acc_out=self.now.acc)


@dataclasses.dataclass(frozen=True)
class Profile:
    """What the searches need to know of a model."""
    latency: float      # seconds of one request alone on one device
    slope: float        # beta of as_simulate_batched: a batch of b takes 1 + beta (b - 1) times as long
    weight_mib: int     # weights and the caches of `requests` requests


def capture_cycle(block: Block, x, caches: Caches):
    """A graph of 2 * slack steps on x from full caches on: a cut into the spare
    pages, steps until they are full, a cut back and steps until the first ones
    are full again.  Nothing is run; every replay takes the caches that far."""
    import torch
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2 * block.shape.slack):
            block.step(x, caches)
    return graph


def step_seconds(block: Block, batch: int, steps: int = 32) -> float:
    """Seconds of one step of the block at its budget's length, the cuts of the
    cache included: at least `steps` steps in a row, every `slack`-th of which
    cuts, the first one among them.  They are replayed from a graph: a step has
    some twenty launches, which take the host longer than the device."""
    import torch
    s = block.shape
    caches = Caches(s, batch, block.device)
    x = torch.randn(batch, s.hidden, device=block.device).to(torch.bfloat16)
    for _ in range(s.budget + 3 * s.slack):  # full, and a cycle before the one that is captured
        block.step(x, caches)
    graph = capture_cycle(block, x, caches)
    graph.replay()
    replays = -(-steps // (2 * s.slack))
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(replays):
        graph.replay()
    stop.record()
    torch.cuda.synchronize()
    return start.elapsed_time(stop) * 1e-3 / (replays * 2 * s.slack)


def measure(shape: Shape, tokens: int, requests: int = 8, batch: int = 8, device="cuda") -> Profile:
    """Profile of a model whose requests generate `tokens` tokens, with room
    for the caches of `requests` requests."""
    block = Block(shape, device=device)
    one, many = step_seconds(block, 1), step_seconds(block, batch)
    cache = Caches(shape, 1, device).bytes_per_sequence()
    return profile(shape, tokens, requests, block.nbytes, cache, one, many, batch)


def profile(shape: Shape, tokens: int, requests: int, block_bytes: int, cache_bytes: int, one: float, many: float,
            batch: int) -> Profile:
    """A profile from a block's bytes, one request's cache bytes in it, and the
    seconds of its step for one request and for `batch`."""
    total = shape.layers * (block_bytes + requests * cache_bytes)
    return Profile(latency=tokens * shape.layers * one,
                   slope=max(0.0, (many / one - 1.0) / (batch - 1)) if batch > 1 else 1.0,
                   weight_mib=-(-total // MIB))


def placement_problem(profiles, n_devices: int, device_mem_gb: int, rate: float, cv: float = 2.0,
                      duration: float = 60.0, slo_scale: float = 5.0, seed: int = 11,
                      partitions=((1, 1, 1), (2, 2, 1), (4, 4, 1))) -> problems.GreedyProblem:
    """The placement problem of models with these profiles: `rate` requests a
    second to each (Gamma arrivals), equal groups of (size, stages, intra-op)."""
    d = np.array([p.latency for p in profiles])
    w = np.array([p.weight_mib for p in profiles], np.int64)
    cfgs = [(S, k) for _, S, k in partitions]
    t, m = gen.trace(seed, [rate] * len(profiles), cv, duration)
    parts = []
    for c, (size, S, k) in enumerate(partitions):
        G = n_devices // size
        parts.append({"group_cfg": np.full(G, c, np.int32),
                      "group_mem_mib": np.full(G, size * device_mem_gb * problems.GIB_MIB, np.int64),
                      "label": f"{G}x(S={S},k={k})"})
    return problems.GreedyProblem("served", t, m, d, w, np.array([S for S, _ in cfgs], np.int32),
                                  np.array([k for _, k in cfgs], np.int32), problems.stage_table(d, cfgs), parts,
                                  slo_scale, {"devices": n_devices, "device_mem_mib": device_mem_gb * problems.GIB_MIB})


def place(gp: problems.GreedyProblem, device="cuda") -> dict:
    """The partition search's answer (as_partition_search)."""
    up = lambda a: sim.to_device(a, device)  # noqa: E731
    return sim.as_partition_search(up(gp.t), up(gp.model), up(gp.d_single), gp.cfg_stages, up(gp.stage_lat),
                                   gp.weight_mib, gp.partitions, gp.slo_scale)


def main():
    shapes = [Shape(layers=24, hidden=2048, heads=16, kv_heads=4, dim=128, inner=8192, budget=1024),
              Shape(layers=32, hidden=4096, heads=32, kv_heads=8, dim=128, inner=16384, budget=2048)]
    found = []
    for s in shapes:
        p = measure(s, tokens=128)
        found.append(p)
        print(f"{s.layers} layers of {s.hidden}: {p.latency:.3f} s a request of 128 tokens, batching slope "
              f"{p.slope:.3f}, {p.weight_mib} MiB", flush=True)
    profiles = [found[i % len(found)] for i in range(8)]
    gp = placement_problem(profiles, n_devices=8, device_mem_gb=16, rate=0.5 / found[-1].latency)
    r = place(gp)
    part = gp.partitions[r["best_partition"]]
    print(f"{len(profiles)} models on 8 devices of 16 GB: {part['label']}, {r['best_served']} of {len(gp.t)} requests "
          f"in time; groups of each model "
          f"{[[g for g in range(len(part['group_cfg'])) if int(m) >> g & 1] for m in r['best_mask']]}", flush=True)


if __name__ == "__main__":
    main()
