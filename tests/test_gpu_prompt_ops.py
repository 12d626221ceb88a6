"""The operators that take prompts in, on the GPU, against their 64-bit
definitions.  Tolerances are first-order bounds of the roundings that the
operators state, worked out beside each."""
import dataclasses

import numpy as np
import pytest
import torch

import ops_oracle as oo
import prompt_oracle as po
from gpu_common import say
from paper_2302_11665_amd import ops, sim
from test_gpu_ops import BF16, F16, F32, HALF_ULP, TINY, check_linear, f64, gen, host, make_cache, normal

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------- norm, 8 bits

NORM = [(1, 1), (3, 2), (2, 15), (3, 127), (16, 128), (17, 129), (1, 4096), (5, 4097), (33, 9000), (2, 16384),
        (2, 16400), (3, 33000), (2, 70001), (1, 131072), (2047, 65), (2050, 900), (2100, 1500), (2049, 2111),
        (2048, 4096), (2060, 8192), (2055, 8200)]


def check_norm(x, residual, gain, eps, result):
    codes, total, held = result
    rows, cols = x.reshape(-1, x.shape[-1]).shape
    h = x if residual is None else (x.cpu().float() + residual.cpu().float()).to(x.dtype)
    assert torch.equal(total.cpu().view(torch.int16), h.cpu().view(torch.int16))
    c, scale = po.norm_rows(f64(h).reshape(rows, cols), None if gain is None else gain.cpu().numpy(), eps)
    got = codes.codes.cpu().numpy()[oo.tile_index(rows, cols)]
    assert np.array_equal(got, c)
    # Squares are summed in fp32 in at most (columns / 1024 + 86) additions one after the
    # other (a lane's 16 four times over, or for every 16,384 columns; 6 between lanes, 16
    # between wavefronts), of numbers that are not negative: 2^-24 of the sum each, half of
    # it of its root; the scale is rounded once.
    tol = ((cols / 1024 + 86) / 2 + 1) * 2.0 ** -24
    s = f64(codes.scale)
    assert np.array_equal(np.isnan(s), np.isnan(scale))
    fine = ~np.isnan(scale)
    assert np.all(np.abs(s - scale)[fine] <= tol * np.abs(scale[fine]) + TINY[F32])
    with np.errstate(invalid="ignore"):
        want = got.astype(np.float32) * codes.scale.cpu().numpy()[:, None]
    assert np.array_equal(held.cpu().numpy().reshape(rows, cols), want, equal_nan=True)
    # columns behind the last are 0
    padded = -(-cols // 128) * 128
    assert not codes.codes.cpu().numpy()[oo.tile_index(rows, padded)][:, cols:].any()


@pytest.mark.parametrize("rows,cols", NORM)
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("add,gained", [(False, False), (True, False), (False, True), (True, True)])
def test_norm(rows, cols, dtype, add, gained):
    say("norm", rows, cols, dtype, add, gained)
    g = gen(rows * 5 + cols)
    x = normal(g, rows, cols, dtype=dtype)
    r = (normal(g, rows, cols) * 3).to(dtype) if add else None
    gain = 1 + 0.5 * normal(g, cols) if gained else None
    if cols > 2 and not add and not gained:
        x[0] = 0
        x[rows - 1, 1] = x[rows - 1].abs().max() * 0.5  # half of the largest: the tie 63.5
    check_norm(x, r, gain, 1e-6, ops.norm_i8(x, r, gain, held=True))


@pytest.mark.parametrize("rows,cols", [(3, 200), (2, 17000), (2049, 300), (2, 40000)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_norm_of_rows_at_the_ends_of_the_range(rows, cols, dtype):
    """Squares that fp32 does not hold, rows of zeros without eps, and rows that are not finite."""
    say("norm ends", rows, cols, dtype)
    g = gen(cols)
    large, small = (1e30, 1e-30) if dtype == BF16 else (6e3, 1e-6)
    for size in (large, small):
        x = (normal(g, rows, cols) * size).to(dtype)
        x[1] = 0
        for eps in (0.0, 1e-6):
            for gain in (None, torch.rand(cols, device="cuda", generator=g)):
                check_norm(x, None, gain, eps, ops.norm_i8(x, gain=gain, eps=eps, held=True))
    x = normal(g, rows, cols, dtype=dtype)
    x[0, cols - 1] = float("inf")
    x[1, 3] = float("nan")
    codes, _, held = ops.norm_i8(x, held=True)
    assert torch.isnan(codes.scale[:2]).all() and torch.isfinite(codes.scale[2:]).all()
    assert torch.isnan(held[:2]).all() and torch.isfinite(held[2:]).all()
    # a sum or a gain that leaves the range: its row alone
    top = torch.finfo(dtype).max
    x = torch.ones(rows, cols, device="cuda", dtype=dtype)
    r = torch.ones_like(x)
    x[0, 5] = r[0, 5] = top
    codes, total = ops.norm_i8(x, r)
    assert torch.isinf(total[0, 5]) and torch.isnan(codes.scale[0]) and torch.isfinite(codes.scale[1:]).all()
    gain = torch.full((cols,), 3e38, device="cuda")
    x = torch.full((rows, cols), 0.5, device="cuda", dtype=dtype)
    x[1] = 4
    codes, _ = ops.norm_i8(x, gain=gain)
    assert torch.isfinite(codes.scale[0]) and torch.isnan(codes.scale[1])


@pytest.mark.parametrize("rows,cols", [(1, 300), (7, 130), (2100, 257)])
def test_norm_in_place_and_of_strided_rows(rows, cols):
    say("norm strides", rows, cols)
    g = gen(8)
    wide = normal(g, rows, 2 * cols + 3, dtype=BF16)
    x, r = wide[:, :cols], wide[:, cols + 1:2 * cols + 1]
    want = ops.norm_i8(x.contiguous(), r.contiguous(), held=True)
    check_norm(x, r, None, 1e-6, ops.norm_i8(x, r, held=True))
    for pick in (0, 1):  # the sum in x's place, in the residual's
        both = wide.clone()
        xs, rs = both[:, :cols], both[:, cols + 1:2 * cols + 1]
        c, total, held = ops.norm_i8(xs, rs, out=(xs, rs)[pick], held=True)
        assert total.data_ptr() == (xs, rs)[pick].data_ptr() and torch.equal(total, want[1])
        assert torch.equal(held, want[2]) and torch.equal(c.scale, want[0].scale)
        left = (rs, xs)[pick]
        assert torch.equal(left, (r, x)[pick]) and torch.equal(both[:, 2 * cols + 1:], wide[:, 2 * cols + 1:])
    one = wide[:1, :cols].expand(rows, cols)  # one row for all tokens
    c, _, held = ops.norm_i8(one, held=True)
    assert torch.equal(held, ops.norm_i8(one.contiguous(), held=True)[2])
    x3 = normal(g, 2, 5, cols, dtype=F16)
    c, total, held = ops.norm_i8(x3, x3, held=True)
    assert total.shape == x3.shape == held.shape and c.n_rows == 10
    none, _ = ops.norm_i8(x3[:0])
    assert none.n_rows == 0 and ops.linear_i8(none, ops.pack_weight(normal(g, 9, cols))).shape == (0, 9)


@pytest.mark.parametrize("rows,cols", [(3101, 8203), (5200, 5000), (1700, 17003)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_norm_of_many_rows_is_that_of_a_few(rows, cols, dtype):
    """Calls that go past the caches, against rows by themselves; the sum in place."""
    say("norm, many rows", rows, cols, dtype)
    g = gen(rows)
    x, r, gain = normal(g, rows, cols, dtype=dtype), normal(g, rows, cols, dtype=dtype), 1 + 0.2 * normal(g, cols)
    taken = [0, 1, 14, 15, 16, 17, rows // 2, rows - 2, rows - 1]
    few = ops.norm_i8(x[taken], r[taken], gain, held=True)
    codes, total, held = ops.norm_i8(x, r, gain, held=True)
    assert torch.equal(total, x + r)
    # The sums of squares may be taken in another order, each as far off as `check_norm`
    # says: twice that between two of them.
    tol = 2 * ((cols / 1024 + 86) / 2 + 1) * 2.0 ** -24
    assert np.all(np.abs(f64(codes.scale[taken]) - f64(few[0].scale)) <= tol * f64(few[0].scale))
    tiles = torch.from_numpy(oo.tile_index(rows, cols)[taken]).cuda()
    mine = torch.from_numpy(oo.tile_index(len(taken), cols)).cuda()
    assert torch.equal(codes.codes[tiles], few[0].codes[mine])
    assert torch.equal(held[taken], few[0].codes[mine].float() * codes.scale[taken, None])
    codes2, total2 = ops.norm_i8(x, r, gain, out=r)
    assert total2.data_ptr() == r.data_ptr() and torch.equal(r, total)
    assert torch.equal(codes2.scale, codes.scale) and torch.equal(codes2.codes[tiles], codes.codes[tiles])


@pytest.mark.parametrize("t,k,n", [(1, 300, 77), (5, 4096, 130), (16, 512, 256), (17, 129, 4097), (40, 2048, 96),
                                   (64, 1024, 1024), (100, 640, 300), (777, 1500, 2777), (2100, 900, 33),
                                   (333, 100, 8200), (385, 260, 5555)])
@pytest.mark.parametrize("dtype,y_dtype,bias", [(BF16, BF16, False), (F16, F32, True), (BF16, F16, True)])
def test_linear_of_codes(t, k, n, dtype, y_dtype, bias):
    say("linear of codes", t, k, n, dtype, y_dtype)
    g = gen(t + k)
    x, r, gain = normal(g, t, k, dtype=dtype), normal(g, t, k, dtype=dtype), 1 + 0.2 * normal(g, k)
    w = ops.pack_weight(normal(g, n, k))
    b = normal(g, n) if bias else None
    c, _ = ops.norm_i8(x, r, gain)
    y = ops.linear_i8(c, w, bias=b, dtype=y_dtype)
    codes = c.codes.cpu().numpy()[oo.tile_index(t, k)]
    prod = (codes.astype(np.float64) @ w.codes.cpu().numpy()[oo.tile_index(n, k)].astype(np.float64).T
            * f64(c.scale)[:, None] * f64(w.scale)[None, :])
    exact = prod + (f64(b)[None, :] if bias else 0.0)
    # the sum to fp32, two products, the bias: 2^-24 each of what they round
    slack = 4 * 2.0 ** -24 * (np.abs(prod) + np.abs(exact))
    slack += HALF_ULP[y_dtype] * (np.abs(exact) + slack) + TINY[y_dtype]
    assert y.dtype == y_dtype and np.all(np.abs(f64(y) - exact) <= slack)
    assert ops.linear_i8(c, w).dtype == dtype
    wide = torch.full((t, n + 5), 7.0, dtype=y_dtype, device="cuda")
    ops.linear_i8(c, w, bias=b, out=wide[:, 2:n + 2])
    assert torch.equal(wide[:, 2:n + 2], y) and (wide[:, :2] == 7).all() and (wide[:, n + 2:] == 7).all()


def test_linear_of_codes_is_linear_of_their_rows():
    """Codes of plain rows, as as_quantize_i8 writes them, give what the layer gives that quantises by itself."""
    g = gen(3)
    for t, k, n in ((1, 300, 40), (33, 1000, 200), (2100, 640, 260)):
        x, w = normal(g, t, k, dtype=F16), ops.pack_weight(normal(g, n, k))
        p = ops.pack_weight(x)
        y = ops.linear_i8(ops.Codes(p.codes, p.scale, t, k, F16), w)
        assert torch.equal(y, ops.linear_i8(x, w))


# ------------------------------------------------------- attention of prompts

def check_prompt(q, k, v, lengths, out, scale=None):
    t, heads, dim = q.shape
    per = heads // k.shape[1]
    sc = dim ** -0.5 if scale is None else scale
    qd, kd, vd, got = f64(q), f64(k), f64(v), f64(out)
    u = HALF_ULP[q.dtype]
    at = 0
    for b, n in enumerate(lengths):
        rows = slice(at, at + n)
        at += n
        for j in range(heads if n else 0):
            qs, ks, vs = qd[rows, j], kd[rows, j // per], vd[rows, j // per]
            o, p, a = po.attend_causal(qs, ks, vs, sc)
            # A logit sums dim products in fp32: as many roundings of 2^-24 of the
            # sum of magnitudes; scaling it and taking the reference off, two of
            # the logit's and the reference's (which is one of the row's logits, or
            # 2^8 below it) size; scale log2 e as one number, two more.
            size = np.abs(qs) @ np.abs(ks).T * sc
            seen = np.arange(n)[None, :] <= np.arange(n)[:, None]
            biggest = np.where(seen, np.abs(a), 0.0).max(1, initial=0.0)
            delta = (np.where(seen, dim * 2.0 ** -24 * size, 0.0).max(1, initial=0.0)
                     + 4 * 2.0 ** -24 * (2 * biggest + 8))
            # weights: that twice (over their sum), exp2 and the division 2^-22; one
            # rounding to the type; fp32 sums of a term each 16 slots
            rel = 2 * delta + 2.0 ** -22 + u + (n / 8 + 16) * 2.0 ** -24
            slack = rel[:, None] * (p @ np.abs(vs))
            if q.dtype == F16:  # weights below 2^-14 of the largest are subnormal in fp16
                slack += 2.0 ** -25 * np.cumsum(np.abs(vs), axis=0)
            slack += u * (np.abs(o) + slack) + TINY[q.dtype]
            off = np.abs(got[rows, j] - o)
            assert np.all(off <= slack), (b, j, n, np.max(off / slack))


def prompt(g, lengths, heads, kv_heads, dim, dtype, behind=0):
    t = sum(lengths) + behind
    qkv = normal(g, t, heads + 2 * kv_heads, dim)
    qkv[:, :heads] *= 1.5
    qkv = qkv.to(dtype)
    offsets = ints([0] + np.cumsum(lengths).tolist())
    return qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], offsets


PROMPTS = [
    # lengths, query heads, key/value heads, dim
    ([1], 1, 1, 64),
    ([2, 1, 3], 2, 1, 128),
    ([0, 1, 0, 31, 32, 33, 0], 4, 2, 64),
    ([63, 64, 65], 8, 1, 128),
    ([127, 128, 129, 130], 3, 3, 64),
    ([255, 257, 5], 6, 2, 128),
    ([511, 1, 90], 5, 1, 64),
    ([700], 7, 1, 128),
    ([1025], 2, 2, 128),
    ([40] * 70 + [0, 3], 4, 4, 64),
    ([1 + i % 17 for i in range(300)], 6, 2, 64),
    ([0] * 200 + [90, 0, 1], 1, 1, 128),
    ([300, 2, 450], 40, 8, 64),
    ([9, 150], 64, 1, 128),       # a group of more rows than a wavefront has
    ([33, 70], 300, 1, 64),       # and than a workgroup has
]


@pytest.mark.parametrize("case", PROMPTS, ids=[str(i) for i in range(len(PROMPTS))])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompt(case, dtype):
    lengths, heads, kv_heads, dim = case
    say("prompt", case, dtype)
    q, k, v, offsets = prompt(gen(sum(lengths) + heads), lengths, heads, kv_heads, dim, dtype)
    check_prompt(q, k, v, lengths, ops.attention_prompt(q, k, v, offsets))


def test_prompt_of_many_sequences():
    """More sequences than a workgroup has threads, each compared with itself alone."""
    g = gen(11)
    lengths = [(7 * i) % 40 for i in range(1500)]
    q, k, v, offsets = prompt(g, lengths, 4, 2, 64, BF16)
    out = ops.attention_prompt(q, k, v, offsets)
    at = np.concatenate([[0], np.cumsum(lengths)])
    for b in list(range(0, 1500, 97)) + [1499, 1, 6]:
        s = slice(int(at[b]), int(at[b + 1]))
        check_prompt(q[s], k[s], v[s], [lengths[b]], out[s])


@pytest.mark.parametrize("n,heads,kv_heads,dim,dtype", [(5000, 2, 1, 128, BF16), (9001, 1, 1, 64, F16),
                                                        (3000, 16, 2, 128, F16)])
def test_long_prompt(n, heads, kv_heads, dim, dtype):
    say("long prompt", n, heads, dim)
    q, k, v, offsets = prompt(gen(n), [n, 10], heads, kv_heads, dim, dtype)
    out = ops.attention_prompt(q, k, v, offsets)
    per = heads // kv_heads
    for j in {0, heads - 1}:
        kk, vv = k[:n, j // per:j // per + 1], v[:n, j // per:j // per + 1]
        check_prompt(q[:n, j:j + 1], kk, vv, [n], out[:n, j:j + 1])
    check_prompt(q[n:], k[n:], v[n:], [10], out[n:])


@pytest.mark.parametrize("lengths,heads,kv_heads", [([1200], 32, 8), ([500, 3, 700, 0, 40], 32, 8), ([900, 333], 30, 10)])
def test_prompt_of_as_many_blocks_as_run_at_once(lengths, heads, kv_heads):
    say("two blocks a unit", lengths, heads)
    q, k, v, offsets = prompt(gen(heads), lengths, heads, kv_heads, 128, BF16)
    check_prompt(q, k, v, lengths, ops.attention_prompt(q, k, v, offsets))


@pytest.mark.parametrize("way", ["up", "down", "flat"])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompt_where_the_maximum_moves(way, dtype):
    """Logits that rise or fall by hundreds along the keys, or are all the same."""
    g = gen(2)
    n, dim = 900, 64
    q, k, v = (normal(g, n, 1, dim) * 0.1 for _ in range(3))
    ramp = torch.linspace(0, 40, n, device="cuda").view(n, 1)
    q[..., 0] = 8.0
    k[..., 0] = ramp if way == "up" else ramp.flip(0) if way == "down" else 3.0
    if way == "flat":
        q[..., 1:] = 0
    q, k, v = (x.to(dtype) for x in (q, k, v))
    offsets = ints([0, 500, n])
    check_prompt(q, k, v, [500, n - 500], ops.attention_prompt(q, k, v, offsets, scale=1.0), scale=1.0)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_prompt_of_the_largest_logits(dtype, dim, sign):
    """Eight values of logits up to 2^30 (bf16) and 2^24 (fp16), far apart: the largest
    that a row sees share its weight."""
    g, n = gen(5), 300
    q, k = torch.zeros(n, 1, dim, device="cuda"), torch.zeros(n, 1, dim, device="cuda")
    v = normal(g, n, 1, dim).to(dtype)
    q[..., 3] = 1.0 if dtype == BF16 else 2.0 ** 8
    steps = torch.randint(0, 8, (n,), device="cuda", generator=g) * 30 + 45
    k[:, 0, 3] = sign * steps * (2.0 ** 22 if dtype == BF16 else 2.0 ** 8)
    out = ops.attention_prompt(q.to(dtype), k.to(dtype), v, ints([0, n]), scale=1.0)
    with np.errstate(over="ignore"):  # of what is masked
        o, p, a = po.attend_causal(f64(q)[:, 0], f64(k)[:, 0], f64(v)[:, 0], 1.0)
    assert abs(a).max() > (2 ** 29.9 if dtype == BF16 else 2 ** 23.9) and ((p > 0).sum(1) > 5).any()
    # logits are exact, so equal ones have equal weights 2^c, |c| half a unit in the last
    # place of a logit log2 e; one rounding of it to the type, exp2 and the division
    # 2^-22, fp32 sums of a term each 16 slots
    u = HALF_ULP[dtype]
    slack = (u + 2.0 ** -22 + (n / 8 + 16) * 2.0 ** -24) * (p @ np.abs(f64(v)[:, 0]))
    slack += u * (np.abs(o) + slack) + TINY[dtype]
    assert np.all(np.abs(f64(out)[:, 0] - o) <= slack)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [1, 3])
def test_prompt_does_not_see_what_is_masked(dtype, dim, heads):
    """Infinities and NaN in later tokens, in other sequences and behind the last one change nothing before them."""
    say("masked", dtype, dim, heads)
    g = gen(dim)
    lengths = [70, 200, 1, 130]
    q, k, v, offsets = prompt(g, lengths, heads, 1, dim, dtype, behind=40)
    want = ops.attention_prompt(q, k, v, offsets)
    at = np.cumsum([0] + lengths).tolist()
    for value in (float("nan"), float("inf"), -float("inf")):
        for bad in (45, at[1] + 3, at[1] + 100, at[1] + 199, at[3] + 64, at[4], at[4] + 39):
            seq = next((b for b in range(4) if at[b] <= bad < at[b + 1]), None)
            end = bad if seq is None else at[seq + 1]
            for which in ("k", "v", "both"):
                kk, vv = k.clone(), v.clone()
                if which != "v":
                    kk[bad] = value
                if which != "k":
                    vv[bad, 0, ::3] = value
                out = ops.attention_prompt(q, kk, vv, offsets)
                clean = [i for i in range(at[4]) if not bad <= i < end]
                # (a query's sums depend on no other query)
                assert torch.equal(out[clean], want[clean]), (value, bad, which)
                if which == "v" and seq is not None:
                    hit, rest = out[bad:end, :, ::3], torch.ones(dim, dtype=torch.bool)
                    rest[::3] = False
                    assert (hit == value).all() if value == value and end - bad < 60 else not torch.isfinite(hit).any()
                    assert torch.equal(out[bad:end][:, :, rest], want[bad:end][:, :, rest])
                if which != "v" and seq is not None and value != value:
                    assert torch.isnan(out[bad:end]).all()
    # rows of no sequence keep what they hold
    out = torch.full_like(want, 5.0)
    ops.attention_prompt(q, k, v, offsets, out=out)
    assert torch.equal(out[:at[4]], want[:at[4]]) and (out[at[4]:] == 5).all()


# Few heads and long prompts: blocks are split, and the last part takes what the host did not expect.
SPLIT = [([1500], 1, 1, 128), ([4000, 30, 0, 700], 1, 1, 64), ([40, 0, 3300, 1], 6, 2, 128), ([900] * 7, 1, 1, 64),
         ([64 * 30], 1, 1, 128), ([2049], 3, 1, 64)]


@pytest.mark.parametrize("case", SPLIT, ids=[str(i) for i in range(len(SPLIT))])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_split_prompt(case, dtype):
    lengths, heads, kv_heads, dim = case
    say("split prompt", case, dtype)
    assert ops.lib().as_attention_prompt_workspace(sum(lengths), heads, kv_heads, len(lengths)) > 0
    q, k, v, offsets = prompt(gen(sum(lengths) + heads), lengths, heads, kv_heads, dim, dtype)
    out = ops.attention_prompt(q, k, v, offsets)
    check_prompt(q, k, v, lengths, out)
    graph, held = torch.cuda.CUDAGraph(), torch.zeros_like(out)
    with torch.cuda.graph(graph):
        ops.attention_prompt(q, k, v, offsets, out=held)
    for _ in range(3):
        held.zero_()
        graph.replay()
        again = ops.attention_prompt(q, k, v, offsets)
        torch.cuda.synchronize()
        assert torch.equal(held, out) and torch.equal(again, out)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 128])
def test_split_prompt_does_not_see_what_is_masked(dtype, dim):
    say("split, masked", dtype, dim)
    g = gen(dim + 1)
    lengths = [1700, 300]
    q, k, v, offsets = prompt(g, lengths, 2, 1, dim, dtype, behind=40)
    assert ops.lib().as_attention_prompt_workspace(2040, 2, 1, 2) > 0
    want = ops.attention_prompt(q, k, v, offsets)
    for value in (float("nan"), float("inf"), -float("inf")):
        for bad, end in ((45, 1700), (255, 1700), (256, 1700), (1023, 1700), (1699, 1700), (1800, 2000), (2010, 2040)):
            for which in ("k", "v"):
                kk, vv = k.clone(), v.clone()
                if which == "k":
                    kk[bad] = value
                else:
                    vv[bad, 0, ::3] = value
                out = ops.attention_prompt(q, kk, vv, offsets)
                clean = [i for i in range(2000) if not bad <= i < end]
                assert torch.equal(out[clean], want[clean]), (value, bad, which)
                if which == "v" and end <= 2000:
                    rest = torch.ones(dim, dtype=torch.bool)
                    rest[::3] = False
                    assert not torch.isfinite(out[bad:end][:, :, ::3]).any()
                    assert torch.equal(out[bad:end][:, :, rest], want[bad:end][:, :, rest])
                if which == "k" and end <= 2000 and value != value:
                    assert torch.isnan(out[bad:end]).all()


def test_prompt_of_opposite_infinities():
    """A row that sees both signs is NaN there, one that sees one of them has it."""
    g = gen(4)
    q, k, v, offsets = prompt(g, [50], 2, 1, 64, BF16)
    v = v.clone()
    v[10, 0, 5], v[20, 0, 5] = float("inf"), -float("inf")
    out = ops.attention_prompt(q, k, v, offsets)
    assert torch.isfinite(out[:10]).all() and (out[10:20, :, 5] == float("inf")).all()
    assert torch.isnan(out[20:, :, 5]).all() and torch.isfinite(out[:, :, :5]).all() and torch.isfinite(out[:, :, 6:]).all()


def test_prompt_of_strided_rows():
    g = gen(7)
    lengths = [37, 90]
    q, k, v, offsets = prompt(g, lengths, 4, 2, 64, F16)
    want = ops.attention_prompt(q.contiguous(), k.contiguous(), v.contiguous(), offsets)
    assert torch.equal(ops.attention_prompt(q, k, v, offsets), want)
    odd = torch.empty(127 * (8 * 64 + 3) + 9, dtype=F16, device="cuda")
    rows = odd[1:1 + 127 * (8 * 64 + 3)].view(127, -1)[:, :8 * 64].unflatten(1, (8, 64))  # at odd addresses
    rows.copy_(torch.cat([q, k, v], 1))
    assert torch.equal(ops.attention_prompt(rows[:, :4], rows[:, 4:6], rows[:, 6:], offsets), want)
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]  # heads outermost
    assert torch.equal(ops.attention_prompt(*turned, offsets), want)
    one = k[:1].expand(127, 2, 64)  # one key for all tokens: every weight is the same
    got = ops.attention_prompt(q, one, v, offsets)
    check_prompt(q, one.contiguous(), v, lengths, got)
    single = [x[:1] for x in (q, k, v)]
    assert torch.equal(ops.attention_prompt(*single, ints([0, 1])), v[:1].repeat_interleave(2, 1))
    assert ops.attention_prompt(q[:0], k[:0], v[:0], ints([0, 0])).shape == (0, 4, 64)
    assert ops.attention_prompt(q, k, v, ints([0]), out=torch.zeros_like(want)).eq(0).all()


def test_prompt_with_offsets_that_make_no_sense():
    """Clipped to the rows that there are; nothing else is touched."""
    g = gen(9)
    q, k, v, _ = prompt(g, [100], 2, 1, 64, BF16)
    for offsets in ([-5, 1000], [50, 20, 90], [0, 2 ** 31 - 1, -2 ** 31, 60], [101, 200], [-1, -1, -1]):
        out = torch.full((300, 2, 64), 5.0, dtype=BF16, device="cuda")
        ops.attention_prompt(q, k, v, ints(offsets), out=out[100:200])
        torch.cuda.synchronize()
        assert (out[:100] == 5).all() and (out[200:] == 5).all(), offsets


# ------------------------------------------------------------------- pages

def check_reserve(stack, count, table, page, length, add, n_tokens):
    s, t = np.array(stack, np.int32), np.array(table, np.int32)
    pool = ops.PagePool(ints(stack), ints([count]))
    dt, dl, da = ints(table), ints(length), ints(add)
    left, after = ints([-7]), torch.full_like(dl, -7)
    places = ops.pages_reserve(pool, dt, page, dl, da, n_tokens, new_length=after, new_count=left)
    want_count, want_length, offsets, seq, slot = po.reserve(s, count, t, page, length, add, n_tokens)
    assert left.item() == want_count and after.tolist() == want_length
    assert places.offsets.tolist() == offsets and places.seq.tolist() == seq and places.slot.tolist() == slot
    assert np.array_equal(dt.cpu().numpy(), t)
    assert pool.count.item() == count and dl.tolist() == list(length)  # left alone
    again = ops.PagePool(pool.stack, pool.count.clone())
    ops.pages_reserve(again, dt, page, dl, da, n_tokens)  # in place
    assert again.count.item() == want_count and dl.tolist() == want_length
    return want_count, want_length, t


@pytest.mark.parametrize("seqs,page,add_hi,part", [(1, 32, 1, 1.0), (3, 32, 40, 0.7), (48, 64, 1, 0.9), (100, 96, 300, 0.3),
                                                   (1023, 32, 5, 0.5), (1024, 64, 90, 0.5), (1025, 32, 64, 0.8),
                                                   (2500, 128, 200, 0.4), (5000, 32, 1, 0.9), (9000, 32, 2, 0.02),
                                                   (9000, 64, 700, 0.01), (7, 32, 5000, 0.9)])
@pytest.mark.parametrize("short", [0, 3])
def test_reserve(seqs, page, add_hi, part, short):
    say("reserve", seqs, page, add_hi, short)
    r = np.random.default_rng(seqs + add_hi)
    max_pages = -(-(200 + add_hi) // page)
    length = r.integers(0, 200, seqs)
    add = np.where(r.random(seqs) < part, r.integers(1, add_hi + 1, seqs), 0)
    need = (-(-(length + add) // page) + length * 0) - -(-length // page)
    free = max(0, int(need.sum()) - short) if short else int(need.sum()) + 2
    stack = r.permutation(free + 10)
    table = r.integers(-1, 99999, (seqs, max_pages))
    check_reserve(stack.tolist(), free, table.tolist(), page, length.tolist(), add.tolist(), int(add.sum()))


@pytest.mark.parametrize("page", [4064, 4096, 2016, 1312])
def test_reserve_far_along(page):
    """Lengths up to 2^30 slots: quotients by the page stay whole."""
    most = 2 ** 30 // page
    r = np.random.default_rng(page)
    ends = np.array([most, most, most - 1, most // 2 + 1, 3]) * page  # where pages begin, or the cache ends
    length = ends - [70, 1, 1, 40, page]
    add = [70, 1, 2, 90, page + 1]
    table = r.integers(-1, 99, (5, most))
    check_reserve(r.permutation(20).tolist(), 12, table, page, length.tolist(), add, int(sum(add)))


def test_reserve_refuses_what_does_not_fit():
    table = [[7, -1, -1]] * 6
    stack = list(range(100, 120))
    # too long for its row; exactly its row; nothing asked; less than nothing; rows that are not there
    check_reserve(stack, 20, table, 32, [10, 90, 96, 5, 40, 0], [87, 6, 1, 0, -3, 20], 114)
    check_reserve(stack, 20, table, 32, [0, 0, 0, 0, 0, 0], [10, 10, 10, 10, 10, 10], 35)
    check_reserve(stack, 20, table, 32, [0] * 6, [10] * 6, 80)  # more rows than tokens
    check_reserve(stack, 2, table, 32, [0, 30, 0, 0, 31, 0], [64, 2, 33, 32, 1, 1], 133)  # no overtaking for pages
    check_reserve(stack, 0, table, 32, [31, 32, 0, 5, 0, 64], [1, 1, 0, 20, 1, 2], 25)
    check_reserve([], 0, table, 32, [0] * 6, [1] * 6, 6)
    check_reserve(stack, 20, table, 32, [2 ** 31 - 1, -2 ** 31, 3, 3, 3, 3], [2 ** 31 - 1] * 2 + [5] * 4, 20)
    check_reserve(stack, 20, table * 800, 32, [40, 2 ** 31 - 1, -2 ** 31, 95, 0, 3] * 800, [1, 2 ** 31 - 1, 0, -9, 96, 2 ** 30] * 800, 7000)
    check_reserve(stack, 20, table * 800, 32, [40, 32, 5, 1, 7, 0] * 800, ([1, 5, 0, 3, 0, 0] + [0] * 594) * 8, 5000)
    check_reserve(stack, 20, [[]] * 3, 32, [0, 0, 0], [1, 0, 2], 3)
    check_reserve(stack, 20, table, 32, [3] * 6, [0] * 6, 0)
    pool = ops.PagePool.full(4)
    none = ops.pages_reserve(pool, ints([[0]] * 2)[:0], 32, ints([]), ints([]), 3)
    assert none.offsets.tolist() == [0] and none.seq.tolist() == [-1] * 3 and pool.count.item() == 4
    none = ops.pages_reserve(pool, ints([[0]] * 2)[:0], 32, ints([]), ints([]), 9000)
    assert none.offsets.tolist() == [0] and (none.seq == -1).all() and (none.slot == -1).all()
    for count in (-5, 1000):  # a count that the stack does not have
        pool = ops.PagePool(ints(stack), ints([count]))
        n = ints([0, 0])
        ops.pages_reserve(pool, ints([[-1], [-1]]), 32, n, ints([1, 1]), 2)
        assert (pool.count.item(), n.tolist()) == ((0, [0, 0]) if count < 0 else (18, [1, 1]))


@pytest.mark.parametrize("seqs,page,rounds", [(5, 32, 30), (200, 64, 12), (1500, 32, 6)])
def test_requests_come_and_go(seqs, page, rounds):
    """Rounds of releases and reservations: no page is ever of two sequences, and none is lost."""
    say("come and go", seqs, page)
    r = np.random.default_rng(seqs)
    pages, max_pages = 3 * seqs, 6
    pool, length = ops.PagePool.full(pages), ints([0] * seqs)
    table = torch.full((seqs, max_pages), -1, dtype=torch.int32, device="cuda")
    stack, t, n, count = pool.stack.cpu().numpy(), table.cpu().numpy(), [0] * seqs, pages
    assert stack.tolist() == list(range(pages))[::-1]
    for i in range(rounds):
        which = r.random(seqs) < 0.3
        add = np.where(r.random(seqs) < 0.7, r.integers(1, 3 * page, seqs), 0)
        ops.pages_release(pool, table, page, length, torch.tensor(which, device="cuda"))
        count, n = po.release(stack, count, t, page, n, which)
        assert pool.count.item() == count and length.tolist() == n and np.array_equal(pool.stack.cpu().numpy(), stack)
        places = ops.pages_reserve(pool, table, page, length, ints(add), int(add.sum()))
        count, n, offsets, seq, slot = po.reserve(stack, count, t, page, n, add, int(add.sum()))
        assert pool.count.item() == count and length.tolist() == n and np.array_equal(table.cpu().numpy(), t)
        assert places.seq.tolist() == seq and places.slot.tolist() == slot
        held = [int(p) for b in range(seqs) for p in t[b, :-(-n[b] // page)]]
        assert sorted(held + stack[:count].tolist()) == list(range(pages)), i


def test_release_leaves_alone_and_stays_inside():
    table = [[1, 2], [3, 4], [5, 6]]
    pool, length = ops.PagePool(ints([9, 0, 0, 0, 0, 0]), ints([1])), ints([33, 64, 1])
    after, left = ints([-7] * 3), ints([-7])
    ops.pages_release(pool, ints(table), 32, length, torch.tensor([1, 0, 1], dtype=torch.uint8, device="cuda"),
                      new_length=after, new_count=left)
    assert pool.stack.tolist() == [9, 1, 2, 5, 0, 0] and left.item() == 4 and after.tolist() == [0, 64, 0]
    assert length.tolist() == [33, 64, 1] and pool.count.item() == 1
    # lengths beyond the row, below 0, and more pages than the pool has
    both = ints([9, 0, 0, 0, 77, 77])
    pool = ops.PagePool(both[:4], ints([1]))
    n = ints([2 ** 31 - 1, -5, 64])
    ops.pages_release(pool, ints(table), 32, n, torch.ones(3, dtype=torch.bool, device="cuda"))
    assert both.tolist() == [9, 1, 2, 5, 77, 77] and pool.count.item() == 4 and n.tolist() == [0, 0, 0]
    ops.pages_release(pool, ints(table)[:0], 32, n[:0], torch.ones(0, dtype=torch.bool, device="cuda"))
    assert pool.count.item() == 4


# ------------------------------------------------------------ packed appends

def check_packed(c, before, k, v, seq, slot, pos, held):
    """Every array of the cache after an append: the tokens' places hold what
    their quantisation gives, and nothing else changed."""
    after = host(c)
    page, group, heads, dim = c._c.page, c._c.group, c._c.n_heads, c._c.dim
    want = {n: a.copy() for n, a in before.items()}
    kd, vd = f64(k), f64(v)
    hk, hv = f64(held[0]), f64(held[1])
    kc, kdl, kml = oo.quantise_token(kd, group)
    vc, vdl, vml = oo.quantise_token(vd, group)
    wk, wv = want["k"].view(np.uint32), want["v"].view(np.uint32)
    ch = np.arange(dim)
    for t in range(len(seq)):
        b, s = int(seq[t]), int(slot[t])
        if b < 0 or b >= c._c.n_seqs or s < 0 or s >= c._c.max_pages * page:
            continue
        p, at = int(before["page_table"][b, s // page]), s % page
        if p < 0 or p >= c._c.n_pages:
            continue
        for h in range(heads):
            words = np.zeros((4, dim // 32), np.uint32)
            np.bitwise_or.at(words, (ch // 8 % 4, ch // 32), kc[t, h].astype(np.uint32) << np.array(
                [oo.nibble(e) for e in ch % 8], np.uint32))
            wk[p, h, at] = words
            e = 4 * (at % 32 // 16) + at % 4
            cell = (p, h, at // 32, at // 4 % 4, ch % 16, ch // 16)
            wv[cell] = wv[cell] & ~np.uint32(15 << oo.nibble(e)) | (vc[t, h].astype(np.uint32) << np.uint32(oo.nibble(e)))
            want["k_par"][p, h, :, at, 0], want["k_par"][p, h, :, at, 1] = kdl[t, h], kml[t, h]
            want["v_par"][p, h, :, at, 0], want["v_par"][p, h, :, at, 1] = vdl[t, h], vml[t, h]
            want["pos"][p, h, at] = s if pos is None else pos[t]
            want["acc"][p, h, at] = 0
            for got, code, d, m in ((hk, kc, kdl, kml), (hv, vc, vdl, vml)):
                value = code[t, h] * np.repeat(d[t, h].astype(np.float64), group) + np.repeat(
                    m[t, h].astype(np.float64), group)
                assert np.all(np.abs(got[t, h] - value) <= 2.0 ** -23 * (np.abs(value) + 15 * np.abs(
                    np.repeat(d[t, h].astype(np.float64), group))))
    for n in want:
        a, z = after[n], want[n]
        if a.dtype == np.float16:
            a, z = a.view(np.int16), z.view(np.int16)
        assert np.array_equal(a, z), n


def packed_places(lengths, adds):
    seq = [b for b, a in enumerate(adds) for _ in range(a)]
    slot = [n + i for n, a in zip(lengths, adds) for i in range(a)]
    return seq, slot


PACKED = [
    # tokens held, tokens added, heads, dim, group, page
    ([0], [1], 1, 64, 64, 32),
    ([5, 0, 31, 32], [1, 1, 1, 1], 2, 64, 32, 32),
    ([0, 3, 40], [70, 1, 29], 2, 128, 64, 32),
    ([10, 0, 0, 63, 1], [1, 0, 100, 2, 33], 1, 128, 128, 96),
    ([i % 40 for i in range(70)], [1] * 70, 1, 64, 64, 64),
    ([0, 17, 31, 0], [33, 31, 1, 200], 3, 128, 32, 128),
    ([30, 62, 1], [4, 4, 64], 2, 64, 64, 32),
]


@pytest.mark.parametrize("case", PACKED, ids=[str(i) for i in range(len(PACKED))])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_packed_append(case, dtype):
    lengths, adds, heads, dim, group, page = case
    say("packed append", case, dtype)
    g = gen(sum(adds) + dim)
    c = make_cache(g, [n + a for n, a in zip(lengths, adds)], heads, dim, group, page, spare=1)
    seq, slot = packed_places(lengths, adds)
    t = len(seq)
    both = normal(g, t, 2 * heads, dim, dtype=dtype) * torch.exp(normal(g, 1, 2 * heads, dim)).to(dtype)
    k, v = both[:, :heads], both[:, heads:]
    before = host(c)
    held = ops.cache_append_packed(c, k, v, ints(seq), ints(slot), held=True)
    check_packed(c, before, k, v, seq, slot, None, held)
    again = host(c)
    pos = [1000 + 3 * i for i in range(t)]
    assert ops.cache_append_packed(c, k.contiguous(), v, ints(seq), ints(slot), pos=ints(pos)) is None
    check_packed(c, again, k, v, seq, slot, pos, held)


def test_packed_append_passes_over():
    """Tokens without a place, and places that do not exist, write nothing."""
    g = gen(5)
    c = make_cache(g, [60, 40], 2, 64, 32, 32, spare=2)
    table = c.page_table.clone()
    table[1, 1] = 9999
    c = dataclasses.replace(c, page_table=table)
    seq = [0, 0, -1, 1, 1, 1, 2, 0, 5, 0, -1, 0, 0, 0, 1]
    slot = [3, 4, 7, 30, 31, 32, 0, 5, 1, -1, -1, 64, 2 ** 31 - 1, 50, 33]
    k, v = normal(g, 15, 2, 64, dtype=F16), normal(g, 15, 2, 64, dtype=F16)
    before = host(c)
    held = ops.cache_append_packed(c, k, v, ints(seq), ints(slot), held=True)
    for x in held:  # rows that are passed over are not written; the check reads the others alone
        assert torch.isfinite(x[[0, 1, 3, 4, 7, 13]]).all()
    check_packed(c, before, k, v, seq, slot, None, held)
    ops.cache_append_packed(c, k[:0], v[:0], ints([]), ints([]))


@pytest.mark.parametrize("dim,t", [(64, 500), (128, 3000)])
def test_packed_append_in_any_order(dim, t):
    """Tokens of a few blocks dealt out over all workgroups."""
    g = gen(t)
    heads = 2
    a = make_cache(g, [t, t], heads, dim, 64, 64)
    k, v = normal(g, 2 * t, heads, dim, dtype=F16), normal(g, 2 * t, heads, dim, dtype=F16)
    seq, slot = (ints(x) for x in packed_places([0, 0], [t, t]))
    b = ops.Cache(*(x.clone() for x in (a.k, a.v, a.k_par, a.v_par, a.pos, a.acc, a.page_table)))
    ops.cache_append_packed(a, k, v, seq, slot)
    order = torch.randperm(2 * t, device="cuda", generator=g)
    ops.cache_append_packed(b, k[order], v[order], seq[order], slot[order])
    for x, z in zip((a.k, a.v, a.pos, a.acc, a.k_par, a.v_par), (b.k, b.v, b.pos, b.acc, b.k_par, b.v_par)):
        assert torch.equal(x, z)


@pytest.mark.parametrize("dim,group,page,starts,t", [(64, 32, 32, [0, 5, 64], 300), (128, 64, 96, [31, 0, 7], 90)])
def test_packed_append_is_an_append(dim, group, page, starts, t):
    """Every sequence's tokens packed one after the other, and given side by side."""
    g = gen(t)
    a = make_cache(g, [s + t for s in starts], 4, dim, group, page)
    b = ops.Cache(*(x.clone() for x in (a.k, a.v, a.k_par, a.v_par, a.pos, a.acc, a.page_table)))
    k, v = normal(g, 3, t, 4, dim, dtype=BF16), normal(g, 3, t, 4, dim, dtype=BF16)
    k[0, 2, 1, 5], v[1, 3, 0, 7], v[2, 0, 3] = float("nan"), float("inf"), 2.0
    ha = ops.cache_append(a, k, v, ints(starts), held=True)
    seq, slot = packed_places(starts, [t] * 3)
    hb = ops.cache_append_packed(b, k.view(-1, 4, dim), v.view(-1, 4, dim), ints(seq), ints(slot), held=True)
    for x, z in zip((a.k, a.v, a.pos, a.acc, a.k_par.view(torch.int16), a.v_par.view(torch.int16)),
                    (b.k, b.v, b.pos, b.acc, b.k_par.view(torch.int16), b.v_par.view(torch.int16))):
        assert torch.equal(x, z)
    for x, z in zip(ha, hb):
        assert torch.equal(x.view(-1).view(torch.int32), z.view(-1).view(torch.int32))


# ------------------------------------------------------ as they are used together

def test_a_prompt_on_another_stream_and_in_a_graph():
    """Pages, norm, product, attention and append on a side stream, and replayed from a graph, give what they give at
    once."""
    g = gen(31)
    heads, kv, dim, hidden, page = 4, 2, 64, 256, 32
    lengths = [70, 0, 33, 1]
    t = sum(lengths) + 5  # rows behind the last prompt
    w = ops.pack_weight(normal(g, (heads + 2 * kv) * dim, hidden))
    back = ops.pack_weight(normal(g, hidden, heads * dim))
    x = normal(g, t, hidden, dtype=BF16)
    gain = 1 + 0.1 * normal(g, hidden)
    add, ended = ints(lengths), torch.tensor([True, False, True, True], device="cuda")
    table = torch.full((4, 4), -1, dtype=torch.int32, device="cuda")
    cache = ops.Cache.empty(8, kv, dim, table, page=page)
    pool, length = ops.PagePool.full(8), ints([0] * 4)
    out = torch.zeros(t, heads, dim, dtype=BF16, device="cuda")

    def step():
        places = ops.pages_reserve(pool, table, page, length, add, t)
        c, _ = ops.norm_i8(x, gain=gain)
        qkv = ops.linear_i8(c, w).view(t, heads + 2 * kv, dim)
        ops.cache_append_packed(cache, qkv[:, heads:heads + kv], qkv[:, heads + kv:], places.seq, places.slot)
        ops.attention_prompt(qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], places.offsets, out=out)
        o = ops.linear_i8(out.view(t, -1), back)
        c, s = ops.norm_i8(o, x, gain=gain)
        y = ops.linear_i8(c, w)
        last = ops.attention_kv4(qkv[:4, :heads].unsqueeze(1), cache, length)
        ops.pages_release(pool, table, page, length, ended)
        return out, s, y, last, places.offsets, places.seq, places.slot

    def state():
        return [cache.k, cache.v, cache.k_par, cache.v_par, cache.pos, table, length, pool.count]

    got = step()
    torch.cuda.synchronize()
    want = [x.clone() for x in got]
    assert length.tolist() == [0, 0, 0, 0] and pool.count.item() == 8
    # (pages given back are taken again from the last one on, in the opposite order every time: two steps are a cycle)
    step()
    torch.cuda.synchronize()
    rest = [x.clone() for x in state()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = [x.clone() for x in step()]
        second = step()
    torch.cuda.synchronize()
    for a, z, y in zip(want, first, second):
        assert torch.equal(a, z) and torch.equal(a, y)
    assert all(torch.equal(a, z) for a, z in zip(rest, state()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        held = step()
    for i in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, z in zip(want, held):
            assert torch.equal(a, z), i
        assert all(torch.equal(a, z) for a, z in zip(rest, state())), i
        step()  # eager work between the replays
        assert torch.equal(step()[1], want[1])


def test_refusals():
    g = gen(1)
    x, gain = normal(g, 4, 64, dtype=BF16), normal(g, 64)
    w = ops.pack_weight(normal(g, 32, 64))
    codes, _ = ops.norm_i8(x)
    q, k = normal(g, 10, 4, 64, dtype=BF16), normal(g, 10, 2, 64, dtype=BF16)
    n = ints([0, 10])
    c = make_cache(g, [40], 2, 64, 64, 32)
    pool, table, length = ops.PagePool.full(4), ints([[0, 1]]), ints([3])
    wide = normal(g, 4, 80, dtype=BF16)
    bad = [
        lambda: ops.norm_i8(x.float()),
        lambda: ops.norm_i8(x.cpu()),
        lambda: ops.norm_i8(x, x[:3]),
        lambda: ops.norm_i8(x, x.half()),
        lambda: ops.norm_i8(x, gain=gain[:63]),
        lambda: ops.norm_i8(x, gain=gain.half()),
        lambda: ops.norm_i8(x, eps=-1.0),
        lambda: ops.norm_i8(x, eps=float("nan")),
        lambda: ops.norm_i8(x, out=torch.empty_like(x)),
        lambda: ops.norm_i8(x, x, out=x.expand(2, 4, 64)[0][:3]),
        lambda: ops.norm_i8(x, x, out=x[:1].expand(4, 64)),
        lambda: ops.norm_i8(wide[:, :64], x, out=wide[:, 8:72]),
        lambda: ops.norm_i8(x, wide[:, :64], out=wide[:, 16:]),
        lambda: ops.norm_i8(x[:, :0]),
        lambda: ops.linear_i8(codes, ops.pack_weight(normal(g, 32, 65))),
        lambda: ops.linear_i8(ops.Codes(codes.codes[:-1], codes.scale, 4, 64, BF16), w),
        lambda: ops.linear_i8(ops.Codes(codes.codes, codes.scale[:3], 4, 64, BF16), w),
        lambda: ops.linear_i8(ops.Codes(codes.codes, codes.scale, 17, 64, BF16), w),
        lambda: ops.linear_i8(codes, w, out=torch.empty(3, 32, dtype=BF16, device="cuda")),
        lambda: ops.attention_prompt(q, k, k[:9], n),
        lambda: ops.attention_prompt(q, k, k.half(), n),
        lambda: ops.attention_prompt(q[:, :3], k, k, n),
        lambda: ops.attention_prompt(q, k[..., :32], k[..., :32], n),
        lambda: ops.attention_prompt(q[..., :32], k[..., :32], k[..., :32], n),
        lambda: ops.attention_prompt(q, k, k, n.long()),
        lambda: ops.attention_prompt(q, k, k, n[:0]),
        lambda: ops.attention_prompt(q, k, k, n, scale=0.0),
        lambda: ops.attention_prompt(q, k, k, n, scale=float("inf")),
        lambda: ops.attention_prompt(q, k, k, n, out=q[:9]),
        lambda: ops.attention_prompt(q, k, k, n, out=q),
        lambda: ops.attention_prompt(q.float(), k.float(), k.float(), n),
        lambda: ops.pages_reserve(pool, table, 48, length, length, 3),
        lambda: ops.pages_reserve(pool, table, 32, length, ints([1, 2]), 3),
        lambda: ops.pages_reserve(pool, table.long(), 32, length, length, 3),
        lambda: ops.pages_reserve(pool, table, 32, length, length.long(), 3),
        lambda: ops.pages_reserve(pool, table, 32, length, length, -1),
        lambda: ops.pages_reserve(pool, table, 1 << 33, length, length, 3),
        lambda: ops.pages_reserve(pool, table, 32, length, length, 3, new_count=ints([])),
        lambda: ops.pages_release(pool, table, 32, length, length),
        lambda: ops.pages_release(pool, table, 0, length, torch.ones(1, dtype=torch.bool, device="cuda")),
        lambda: ops.cache_append_packed(c, k[:, :1], k[:, :1], ints([0] * 10), ints(range(10))),
        lambda: ops.cache_append_packed(c, k, k, ints([0] * 9), ints(range(10))),
        lambda: ops.cache_append_packed(c, k, k, ints([0] * 10), ints(range(10)).long()),
        lambda: ops.cache_append_packed(c, k, k.half(), ints([0] * 10), ints(range(10))),
        lambda: ops.cache_append_packed(c, k, k, ints([0] * 10), ints(range(10)), pos=ints([1])),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(sim.SimError):
            f()
            print("not refused:", i)
