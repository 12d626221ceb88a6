"""A served block's steps, its caches' cuts, and the placement from its profile."""
import numpy as np
import pytest

import oracle
from oracle import greedy as ogreedy
from gpu_common import say

pytestmark = pytest.mark.gpu


def small(**over):
    from paper_2302_11665_amd.served import Shape
    f = dict(layers=2, hidden=256, heads=4, kv_heads=2, dim=64, inner=512, budget=40, slack=24, recent=8, page=32)
    f.update(over)
    return Shape(**f)


def run(shape, steps, seqs=3):
    import torch
    from paper_2302_11665_amd import served
    block = served.Block(shape, seed=3)
    caches = served.Caches(shape, seqs)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    outs = []
    for _ in range(steps):
        x = torch.randn(seqs, shape.hidden, device="cuda", generator=g).to(torch.bfloat16)
        outs.append(block.step(x, caches))
    return torch.stack(outs), caches


def positions(caches):
    """pos [seqs, heads, length] on the host."""
    table, page = caches.now.page_table.cpu().numpy(), caches.shape.page
    pos = caches.now.pos.cpu().numpy()
    slot = np.arange(caches.held)
    return np.stack([pos[row[slot // page], :, slot % page].T for row in table])


def test_caches_are_cut_to_the_budget():
    shape = small()
    out, caches = run(shape, 150)
    say("steps run")
    import torch
    assert torch.isfinite(out).all()
    assert caches.length.tolist() == [caches.held] * 3 and caches.total.tolist() == [150] * 3
    assert shape.budget < caches.held <= shape.budget + shape.slack
    pos = positions(caches)
    assert (np.diff(pos, axis=-1) > 0).all()  # in the order of the tokens
    since = caches.held - shape.budget        # tokens since the last cut
    newest = np.arange(150 - since - shape.recent, 150)
    assert (pos[..., -len(newest):] == newest).all()
    # a token's weight is what its queries' heads gave it: all rows of all steps
    # gave 1 in sum, and cuts only take weight away
    assert float(caches.now.acc.sum()) <= 150 * 3 * shape.heads * (1 + 1e-3)


def test_a_cut_changes_nothing_before_it():
    import torch
    cut, _ = run(small(), 64)
    free, caches = run(small(budget=200), 64)
    assert torch.equal(cut, free)
    # 64 steps of one row a head: every row gives weight 1 in sum (fp32 sums of
    # at most 64 terms)
    assert float(caches.now.acc.sum()) == pytest.approx(64 * 3 * 4, rel=1e-5)
    longer, _ = run(small(), 70)
    assert torch.equal(longer[:64], free) and torch.isfinite(longer).all()


def test_the_bytes_of_a_sequence_are_those_of_its_arrays():
    from paper_2302_11665_amd import served
    for shape in (small(), small(budget=100, dim=128, group=32, page=64)):
        caches = served.Caches(shape, 3)
        arrays = {x.data_ptr(): x.numel() * x.element_size() for c in (caches.now, caches.spare)
                  for x in (c.k, c.v, c.k_par, c.v_par, c.pos, c.acc)}
        assert len(arrays) == 12 and 3 * caches.bytes_per_sequence() == sum(arrays.values())


def test_a_step_is_timed_with_its_share_of_the_cuts(monkeypatch):
    """Cuts made slower by a known amount show in the step's time, one in `slack` steps."""
    import torch
    from paper_2302_11665_amd import ops, served
    block = served.Block(small(slack=32), seed=3)
    a = torch.randn(6000, 6000, device="cuda")

    def busy():
        for _ in range(8):
            torch.mm(a, a)

    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(2):
        start.record()
        busy()
        stop.record()
        torch.cuda.synchronize()
    extra = start.elapsed_time(stop) * 1e-3
    say("a slow cut:", extra, "s")
    plain = served.step_seconds(block, 2)
    evict = ops.cache_evict

    def slow(*args, **kw):
        busy()
        return evict(*args, **kw)

    monkeypatch.setattr(ops, "cache_evict", slow)
    cuts = served.step_seconds(block, 2)
    say("steps:", plain, cuts)
    # a 32nd of it a step; half and twice that for the clock's changes between the two
    assert extra / 32 / 2 < cuts - plain < extra / 32 * 2


def test_a_step_is_timed_without_the_host(monkeypatch):
    """What the host does between launches is no part of what a model costs on a device."""
    import time
    from paper_2302_11665_amd import served
    block = served.Block(small(slack=4), seed=3)
    step = block.step

    def slow(x, caches):
        time.sleep(3e-3)
        return step(x, caches)

    monkeypatch.setattr(block, "step", slow)
    seconds = served.step_seconds(block, 2)
    say("step:", seconds)
    assert 0 < seconds < 1.5e-3


@pytest.mark.parametrize("hidden,seqs", [(256, 3), (4096, 1), (1024, 8)])
def test_replayed_steps_are_the_steps(hidden, seqs):
    """A captured cycle of steps, replayed several times with other work between, leaves what as many steps leave."""
    import torch
    from paper_2302_11665_amd import served
    shape = small(hidden=hidden, inner=2 * hidden, slack=5, budget=60)
    block = served.Block(shape, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn(seqs, hidden, device="cuda", generator=g).to(torch.bfloat16)
    eager, caches = served.Caches(shape, seqs), served.Caches(shape, seqs)
    for c in (eager, caches):
        for _ in range(shape.budget + shape.slack):
            block.step(x, c)
    graph = served.capture_cycle(block, x, caches)

    def state(c):
        return [c.length, c.total] + [t for s in (c.now, c.spare) for t in (s.k, s.v, s.k_par, s.v_par, s.pos, s.acc)]

    for i in range(4):
        graph.replay()
        for _ in range(2 * shape.slack):
            block.step(x, eager)
        torch.cuda.synchronize()
        assert caches.held == eager.held == shape.budget + shape.slack
        for a, z in zip(state(caches), state(eager)):
            assert torch.equal(a, z), i


def test_profile_and_placement():
    from paper_2302_11665_amd import served
    shape = small()
    p = served.measure(shape, tokens=16, requests=4, batch=4)
    assert p.latency > 0 and p.slope >= 0 and p.weight_mib >= 1
    profiles = [served.Profile(latency=0.2 + 0.05 * i, slope=0.1, weight_mib=3000 + 500 * i) for i in range(6)]
    gp = served.placement_problem(profiles, n_devices=8, device_mem_gb=8, rate=2.0, duration=30.0)
    r = served.place(gp)
    best, results = ogreedy.reduced_partition_search(oracle.lib(), gp.t, gp.model, gp.d_single, gp.weight_mib,
                                                     gp.cfg_stages, gp.stage_lat, gp.partitions, gp.slo_scale)
    assert r["best_served"] == max(x["best_served"] for x in results)
    assert [int(m) for m in r["best_mask"]] == [int(m) for m in results[r["best_partition"]]["best_mask"]]
