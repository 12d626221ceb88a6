"""Requests that come and go in a served block: prompts read at once, steps of
those that run, pages given back."""
import numpy as np
import pytest
import torch

from gpu_common import say
from test_gpu_prompt_ops import ints
from test_gpu_served import small

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def block_and_prompts(lengths, behind=0, **over):
    from paper_2302_11665_amd import served
    shape = small(**over)
    block = served.Block(shape, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(lengths))
    return shape, block, torch.randn(sum(lengths) + behind, shape.hidden, device="cuda", generator=g).to(BF16)


def plain_block(shape, block, x, lengths):
    """The block's output in float64 from the definitions, without its operators;
    the weights are what their codes stand for, activations are quantised per token
    as the layers do, in exact arithmetic."""
    import ops_oracle as oo
    import prompt_oracle as po

    def weight(w):
        return w.codes.cpu().numpy()[oo.tile_index(w.n_out, w.n_in)] * w.scale.cpu().double().numpy()[:, None]

    def layer(h, w, eps=None):
        """16-bit rows (normed, with eps) through a layer."""
        if eps is None:
            c, s = oo.quantise_rows(h)
        else:
            c, s = po.norm_rows(h, None, eps)
        return round16(c * s[:, None] @ weight(w).T)

    def round16(a):
        return torch.from_numpy(a).to(BF16).double().numpy()

    h = x.cpu().double().numpy()
    qkv = layer(h, block.qkv, 1e-6).reshape(len(h), -1, shape.dim)
    o = np.zeros((len(h), shape.heads, shape.dim))
    at, per = 0, shape.heads // shape.kv_heads
    for n in lengths:
        for j in range(shape.heads if n else 0):
            k, v = qkv[at:at + n, shape.heads + j // per], qkv[at:at + n, shape.heads + shape.kv_heads + j // per]
            o[at:at + n, j] = po.attend_causal(qkv[at:at + n, j], k, v, shape.dim ** -0.5)[0]
        at += n
    h = round16(h + layer(round16(o.reshape(len(h), -1)), block.out))
    u = round16(torch.nn.functional.gelu(torch.from_numpy(layer(h, block.up, 1e-6))).numpy())
    return h, round16(h + layer(u, block.down))


@pytest.mark.parametrize("lengths", [[33], [1, 70, 0, 5], [64, 65, 130]])
def test_prompts_through_a_block(lengths):
    """Against the definitions.  The two differ where a rounding to bf16 falls
    the other way, by one unit in its last place, and where a code does, by a 127th
    of its row's largest value."""
    say("prompts", lengths)
    from paper_2302_11665_amd import served
    shape, block, x = block_and_prompts(lengths)
    requests = served.Requests(shape, len(lengths), 256)
    y = block.prompt(x, requests, ints(lengths)).cpu().double().numpy()
    h, want = plain_block(shape, block, x, lengths)
    # Outputs are near 1: layers of rows of mean square 1 and weights of size
    # inputs ** -0.5.  Codes all off by one would move one by at most the largest
    # value, below 4, times 1 / 127, in each of the four layers.
    slack = 4 * 4.0 / 127 + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(y - want) <= slack), np.max(np.abs(y - want) / slack)
    # Seven roundings to bf16 one after the other, each at most 2^-8 of what it
    # rounds and 2^-8 / sqrt(3) of it in the mean square: 2^-7.4 in all.
    assert np.sqrt(np.mean((y - want) ** 2)) <= 2.0 ** -7 * np.sqrt(np.mean(want ** 2))
    assert requests.length.tolist() == lengths


def test_packed_prompts_are_prompts_alone():
    from paper_2302_11665_amd import served
    lengths = [40, 1, 90, 33]
    shape, block, x = block_and_prompts(lengths, behind=7)
    requests = served.Requests(shape, 4, 128)
    y = block.prompt(x, requests, ints(lengths))
    at = 0
    for b, n in enumerate(lengths):
        alone = served.Requests(shape, 1, 128)
        z = block.prompt(x[at:at + n].contiguous(), alone, ints([n]))
        assert torch.equal(y[at:at + n], z), b  # the same kernels: fewer rows than change them
        for i in range(-(-n // shape.page)):
            mine, its = requests.cache.page_table[b, i], alone.cache.page_table[0, i]
            last = n - i * shape.page
            for name in ("k", "pos"):
                assert torch.equal(getattr(requests.cache, name)[mine][:, :last], getattr(alone.cache, name)[its][:, :last])
        at += n


def test_steps_after_prompts():
    """Steps append to what the prompts left, each request at its own length: the same as over a cache of its own."""
    from paper_2302_11665_amd import ops, served
    lengths = [31, 0, 64, 5]
    shape, block, x = block_and_prompts(lengths)
    requests = served.Requests(shape, 4, 128)
    block.prompt(x, requests, ints(lengths))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    table = torch.arange(16, dtype=torch.int32, device="cuda").view(4, 4)
    own = ops.Cache.empty(16, shape.kv_heads, shape.dim, table, group=shape.group, page=shape.page)
    codes, _ = ops.norm_i8(x)
    qkv = ops.linear_i8(codes, block.qkv).view(-1, shape.heads + 2 * shape.kv_heads, shape.dim)
    at = 0
    for b, n in enumerate(lengths):
        one = ops.Cache(*(getattr(own, f) for f in ("k", "v", "k_par", "v_par", "pos", "acc")), page_table=table[b:b + 1])
        kv = [z[at:at + n].unsqueeze(0) for z in (qkv[:, shape.heads:shape.heads + shape.kv_heads], qkv[:, shape.heads + shape.kv_heads:])]
        if n:
            ops.cache_append(one, *kv, ints([0]))
        at += n
    n = ints(lengths)
    for i in range(40):
        q = torch.randn(4, 1, shape.heads, shape.dim, device="cuda", generator=g).to(BF16)
        k, v = (torch.randn(4, 1, shape.kv_heads, shape.dim, device="cuda", generator=g).to(BF16) for _ in range(2))
        o = requests.attend(q, k, v)
        ops.cache_append(own, k, v, n)
        n += (n > 0).int()
        assert torch.equal(o, ops.attention_kv4(q, own, n)), i
        assert torch.equal(requests.length, n)
        assert (o[1] == 0).all()  # a place without a request
    y = block.step(torch.randn(4, shape.hidden, device="cuda").to(BF16), requests)
    assert torch.isfinite(y).all() and requests.length.tolist() == [31 + 41, 0, 64 + 41, 5 + 41]


def test_requests_that_get_no_pages():
    from paper_2302_11665_amd import served
    lengths = [64, 40, 10]
    shape, block, x = block_and_prompts(lengths)
    requests = served.Requests(shape, 3, 96, n_pages=3)  # 2 + 2 + 1 are wanted
    want = block.prompt(x, served.Requests(shape, 3, 96), ints(lengths))
    y = block.prompt(x, requests, ints(lengths))
    assert torch.equal(y, want)
    assert requests.length.tolist() == [64, 0, 0] and requests.pool.count.item() == 1
    q = torch.zeros(3, 1, shape.heads, shape.dim, dtype=BF16, device="cuda")
    k = torch.ones(3, 1, shape.kv_heads, shape.dim, dtype=BF16, device="cuda")
    requests.attend(q, k, k)
    assert requests.length.tolist() == [65, 0, 0] and requests.pool.count.item() == 0
    for _ in range(40):  # the page is full after 31 more, and there is no other
        requests.attend(q, k, k)
    assert requests.length.tolist() == [96, 0, 0]
    requests.finish(torch.tensor([True, False, False], device="cuda"))
    assert requests.length.tolist() == [0, 0, 0] and requests.pool.count.item() == 3
    block.prompt(x[64:], requests, ints([0, 40, 10]))
    assert requests.length.tolist() == [0, 40, 10] and requests.pool.count.item() == 0


def test_prompts_and_steps_replayed():
    """A captured round of prompts, steps and endings, replayed with eager rounds between, gives what it gives at once."""
    from paper_2302_11665_amd import served
    lengths = [40, 0, 33]
    shape, block, x = block_and_prompts(lengths)
    add, ended = ints(lengths), torch.ones(3, dtype=torch.bool, device="cuda")
    one = torch.randn(3, shape.hidden, device="cuda").to(BF16)
    requests = served.Requests(shape, 3, 96)

    def round_():
        y = block.prompt(x, requests, add)
        z = [block.step(one, requests) for _ in range(3)]
        n = requests.length.clone()
        requests.finish(ended)
        return [y, *z, n]

    want = [t.clone() for t in round_()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = round_()
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, z) for a, z in zip(want, got)), i
        assert all(torch.equal(a, z) for a, z in zip(want, round_())), i
        assert requests.pool.count.item() == 9 and requests.length.tolist() == [0, 0, 0]
    assert want[-1].tolist() == [43, 0, 36]


def test_a_prompt_is_counted_in_the_latency(monkeypatch):
    from paper_2302_11665_amd import served
    shape, block, _ = block_and_prompts([4])
    assert served.prompt_seconds(block, [100, 7], repeats=2) > 0
    monkeypatch.setattr(served, "step_seconds", lambda block, n: 1e-4 * (1 + n))
    monkeypatch.setattr(served, "prompt_seconds", lambda block, lengths: 1e-3 * sum(lengths) / lengths[0] * 2)
    p = served.measure(shape, tokens=10, batch=4, prompt=50)
    assert p.latency == pytest.approx(2 * (10 * 2e-4 + 2e-3)) and p.slope == pytest.approx(
        ((10 * 5e-4 + 8e-3) / (10 * 2e-4 + 2e-3) - 1) / 3)
    assert served.measure(shape, tokens=10, batch=4).latency == pytest.approx(2 * 10 * 2e-4)
