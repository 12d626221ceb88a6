"""The operators that take prompts in at sizes where they take other ways: prompts listed
by size, wide tiles of packed appends, many pages given back at once."""
import numpy as np
import pytest
import torch

from gpu_common import say
from paper_2302_11665_amd import ops
from test_gpu_ops import BF16, F16, gen, make_cache, normal
from test_gpu_prompt_ops import check_prompt, ints, prompt

pytestmark = pytest.mark.gpu


# More than 64 sequences, whose blocks of 128 rows are listed: of none to 69 blocks, in classes of their numbers.
LISTED = [([0, 1, 127, 128, 129, 700, 3000] + [5] * 70, 2, 1, 64),
          ([5] * 40 + [3000, 700, 0, 129, 128, 127, 1] + [64] * 30, 2, 2, 128),
          ([3, 1100, 0, 130] + [17] * 66, 8, 1, 128),
          ([200] * 63 + [1100, 1099, 0, 2], 8, 1, 64),
          ([(i * i * 7) % 401 for i in range(1100)], 1, 1, 64),
          ([(i * 131) % 290 for i in range(1030)], 1, 1, 128)]


@pytest.mark.parametrize("case", LISTED, ids=[str(i) for i in range(len(LISTED))])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_listed_prompts(case, dtype):
    lengths, heads, kv_heads, dim = case
    say("listed prompts", len(lengths), max(lengths), heads, kv_heads, dim, dtype)
    q, k, v, offsets = prompt(gen(sum(lengths) + heads), lengths, heads, kv_heads, dim, dtype, behind=9)
    out = torch.full(q.shape, float("nan"), dtype=dtype, device="cuda")
    ops.attention_prompt(q, k, v, offsets, out=out)
    assert torch.isnan(out[-9:]).all()
    check_prompt(q, k, v, lengths, out)
    again = ops.attention_prompt(q, k, v, offsets)
    assert torch.equal(again[:-9], out[:-9])


def arrays(c):
    """All of a cache, as whole numbers where their bits count."""
    return [c.k, c.v, c.k_par.view(torch.int16), c.v_par.view(torch.int16), c.pos, c.acc]


# 8 heads: a workgroup takes the runs of 4 tokens of 1500, and of 8, 16 and 32 of more than 2048, 4096 and 8192, on
# 256 compute units.
@pytest.mark.parametrize("t", [1500, 3000, 6000, 12000])
@pytest.mark.parametrize("dim,group,page", [(64, 32, 32), (64, 64, 64), (128, 64, 96), (128, 128, 64), (128, 32, 128)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_packed_append_of_many_tokens(t, dim, group, page, dtype):
    """Prompts from ragged starts, single tokens between them and tokens that are passed over, against appends of
    every sequence by itself; then all tokens in another order."""
    say("packed append of many tokens", t, dim, group, page, dtype)
    g, r, heads = gen(t + dim + group), np.random.default_rng(t + group), 8
    adds = []
    while sum(adds) < t:
        adds.append(int(r.choice([1, 1, 1, 1, 2, 5, 31, 32, 33, 63, 64, 65, 100, 700])))
    starts = r.integers(0, 70, len(adds)).tolist()
    a = make_cache(g, [s + n for s, n in zip(starts, adds)], heads, dim, group, page, spare=2)
    table = a.page_table[torch.tensor([0] * 3)]  # three sequences more, on no page
    a = ops.Cache(a.k, a.v, a.k_par, a.v_par, a.pos, a.acc, torch.cat([a.page_table, torch.full_like(table, -1)]))
    b, c = (ops.Cache(*(x.clone() for x in (a.k, a.v, a.k_par, a.v_par, a.pos, a.acc, a.page_table))) for _ in range(2))
    seq, slot = [], []
    for i, (s, n) in enumerate(zip(starts, adds)):
        seq += [i] * n
        slot += range(s, s + n)
        if i % 3 == 0:  # passed over: no sequence, no slot, no page, none of the cache's sequences
            seq += [-1, i, len(adds) + i % 2, len(adds) + 3]
            slot += [int(slot[-1]) + 1, -1, 0, 3]
    seq, slot = ints(seq), ints(slot)
    n = len(seq)
    both = normal(g, n, 2 * heads, dim, dtype=dtype)
    k, v = both[:, :heads], both[:, heads:]
    held = ops.cache_append_packed(a, k, v, seq, slot, held=True)
    at = 0
    for i, (s, m) in enumerate(zip(starts, adds)):
        one = ops.Cache(b.k, b.v, b.k_par, b.v_par, b.pos, b.acc, b.page_table[i:i + 1])
        want = ops.cache_append(one, k[at:at + m].unsqueeze(0), v[at:at + m].unsqueeze(0), ints([s]), held=True)
        for x, z in zip(held, want):
            assert torch.equal(x[at:at + m], z[0]), i
        at += m + (4 if i % 3 == 0 else 0)
    assert at == n
    for x, z in zip(arrays(a), arrays(b)):
        assert torch.equal(x, z)
    order = torch.randperm(n, device="cuda", generator=g)
    ops.cache_append_packed(c, k[order], v[order], seq[order], slot[order])
    for x, z in zip(arrays(c), arrays(b)):
        assert torch.equal(x, z)


def check_release(lengths, which, page, max_pages, n_pages, count):
    """Pages go onto the stack in the order of sequences and of their pages, as many as it has room for."""
    r = np.random.default_rng(len(lengths))
    table = r.permutation(len(lengths) * max_pages).reshape(-1, max_pages).astype(np.int32)
    around = np.full(n_pages + 64, 7, np.int32)
    want = around.copy()
    pages = np.concatenate([table[b, :-(-lengths[b] // page)] for b in range(len(lengths)) if which[b]] + [[]])
    fit = int(min(len(pages), n_pages - count))
    want[32 + count:32 + count + fit] = pages[:fit]
    stack = torch.tensor(around, device="cuda")
    pool, length = ops.PagePool(stack[32:32 + n_pages], ints([count])), ints(lengths)
    ops.pages_release(pool, torch.tensor(table, device="cuda"), page, length, torch.tensor(which, device="cuda"))
    assert pool.count.item() == count + fit and np.array_equal(stack.cpu().numpy(), want)
    assert length.tolist() == [0 if w else n for n, w in zip(lengths, which)]


@pytest.mark.parametrize("seqs,most,part,at_least", [(1024, 150, 0.6, 1024), (1024, 500, 0.9, 4096), (2500, 700, 0.8, 9000),
                                                     (300, 5000, 1.0, 16384)])
@pytest.mark.parametrize("short", [0, 1, 1000])
def test_release_of_many_pages(seqs, most, part, at_least, short):
    """More pages from a run of 1024 sequences than threads, and than four times those; sequences of none between; and
    lengths that ask for more than there is room for."""
    say("release of many pages", seqs, most, short)
    r = np.random.default_rng(seqs + most)
    lengths = np.where(r.random(seqs) < 0.2, 0, r.integers(1, most + 1, seqs)).tolist()
    which = (r.random(seqs) < part).tolist()
    asked = sum(-(-n // 32) for n, w in zip(lengths, which) if w)
    assert asked > at_least
    check_release(lengths, which, 32, -(-most // 32), 100 + asked + (50 if short == 0 else -short), 100)
