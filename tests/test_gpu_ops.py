"""The operators of a served model's step on the GPU against their 64-bit
definitions.  Tolerances are first-order bounds of the roundings that the
operators state, worked out beside each."""
import dataclasses

import numpy as np
import pytest
import torch

import ops_oracle as oo
from gpu_common import kernels_run, say
from paper_2302_11665_amd import ops, sim

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}  # unit roundoff: significands of 8, 11 and 24 bits
TINY = {BF16: 2.0 ** -134, F16: 2.0 ** -25, F32: 2.0 ** -150}   # half the spacing of subnormals


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def f64(x):
    return x.detach().cpu().double().numpy()


# ------------------------------------------------------------------- 8 bits

@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (16, 128), (17, 129), (40, 1000), (5, 4100)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_quantised_rows(rows, cols, dtype):
    say("quantise", rows, cols, dtype)
    x = normal(gen(rows * 7 + cols), rows, cols, dtype=dtype)
    if cols > 2:
        x[0, :] = 0
        x[rows - 1, 1] = x[rows - 1].abs().max() * 0.5  # half of the largest: the tie 63.5
    w = ops.pack_weight(x)
    # With fp32 values, 127 x is rounded once and then divided: the definition
    # is stated for that product.
    top = f64(x.abs().amax(1))
    if dtype == F32:
        prod = f64(x * 127.0)
        codes = np.rint((prod / np.where(top > 0, top, 1.0)[:, None]).astype(np.float32).astype(np.float64))
        codes = codes.astype(np.int64)
    else:
        codes, _ = oo.quantise_rows(f64(x))
    got = w.codes.cpu().numpy()[oo.tile_index(rows, cols)]
    assert np.array_equal(got, codes)
    assert np.allclose(f64(w.scale), top / 127.0, rtol=2.0 ** -24, atol=0)
    pad = np.ones(w.codes.numel(), bool)
    padded = -(-cols // 128) * 128
    pad[oo.tile_index(rows, padded)[:, :cols]] = False
    pad_rows = np.zeros(w.codes.numel(), bool)
    pad_rows[oo.tile_index(rows, padded)] = True
    assert not w.codes.cpu().numpy()[pad & pad_rows].any()  # columns beyond the last are 0


LINEAR = [(1, 1, 1), (1, 64, 16), (1, 4096, 1024), (2, 300, 77), (7, 1000, 130), (16, 512, 256), (17, 129, 4097),
          (33, 2048, 96), (64, 1024, 1024), (100, 640, 300), (129, 256, 520), (257, 1500, 777), (1000, 200, 300),
          (300, 4224, 640), (2050, 900, 33), (2049, 1500, 40), (2048, 3001, 24), (2100, 6100, 17), (2060, 8200, 20),
          (4100, 260, 4200), (2, 9000, 60), (15, 5000, 8500), (64, 130, 9000)]


def check_linear(x, w, u, bias, y, y_dtype):
    codes, s = oo.quantise_rows(f64(x))
    acc = codes.astype(np.float64) @ w.astype(np.float64).T
    prod = acc * s[:, None] * u[None, :]
    exact = prod + (bias[None, :] if bias is not None else 0.0)
    # roundings of the sum to fp32, of the scale, of two products (and of the
    # last sum): 2^-24 each of what they round
    slack = 5 * 2.0 ** -24 * (np.abs(prod) + np.abs(exact))
    slack += HALF_ULP[y_dtype] * (np.abs(exact) + slack) + TINY[y_dtype]
    got = f64(y)
    assert got.shape == exact.shape
    assert np.array_equal(np.isnan(got), np.isnan(exact))
    fine = ~np.isnan(exact)
    assert np.all(np.abs(got - exact)[fine] <= slack[fine]), np.max((np.abs(got - exact) / slack)[fine])


@pytest.mark.parametrize("t,k,n", LINEAR)
@pytest.mark.parametrize("x_dtype,y_dtype,bias", [(BF16, BF16, False), (F16, F16, True), (BF16, F32, True),
                                                  (F16, BF16, False)])
def test_linear(t, k, n, x_dtype, y_dtype, bias):
    say("linear", t, k, n, x_dtype, y_dtype, bias)
    g = gen(t + 3 * k + n)
    x = normal(g, t, k, dtype=x_dtype)
    wf = normal(g, n, k)
    w = ops.pack_weight(wf)
    b = normal(g, n) if bias else None
    y = ops.linear_i8(x, w, bias=b, dtype=y_dtype)
    assert y.dtype == y_dtype
    codes = w.codes.cpu().numpy()[oo.tile_index(n, k)]
    check_linear(x, codes, f64(w.scale), f64(b) if bias else None, y, y_dtype)


def test_linear_rows_that_are_not_finite():
    g = gen(5)
    x = normal(g, 20, 200, dtype=BF16)
    x[0, 3] = float("inf")
    x[7, 199] = float("nan")
    x[19] = 0
    w = ops.pack_weight(normal(g, 40, 200))
    y = ops.linear_i8(x, w, dtype=F32)
    codes = w.codes.cpu().numpy()[oo.tile_index(40, 200)]
    with np.errstate(invalid="ignore"):
        check_linear(x, codes, f64(w.scale), None, y, F32)
    assert torch.isnan(y[0]).all() and torch.isnan(y[7]).all() and (y[19] == 0).all()


@pytest.mark.parametrize("t,k,n", [(4090, 130, 4081), (4096, 256, 4096), (2050, 200, 4097), (1111, 130, 2111), (200, 130, 610)])
@pytest.mark.parametrize("x_dtype,y_dtype,bias", [(BF16, BF16, True), (F16, F16, False), (BF16, F32, True)])
def test_linear_tiles_to_outputs_at_odd_places(t, k, n, x_dtype, y_dtype, bias):
    say("linear tiles", t, k, n, x_dtype, y_dtype, bias)
    g = gen(t + k + n)
    x = normal(g, t, k, dtype=x_dtype)
    w = ops.pack_weight(normal(g, n, k))
    b = normal(g, n) if bias else None
    y = torch.full((t, n + 3), 7.0, device="cuda", dtype=y_dtype)
    ops.linear_i8(x, w, bias=b, out=y[:, 1:n + 1])
    assert (y[:, 0] == 7.0).all() and (y[:, n + 1:] == 7.0).all()
    codes = w.codes.cpu().numpy()[oo.tile_index(n, k)]
    check_linear(x, codes, f64(w.scale), f64(b) if bias else None, y[:, 1:n + 1], y_dtype)


# Outputs of a vocabulary's size: two and four channel tiles to a workgroup, the
# tokens quantised there or before, one to four tiles of them.
MANY_OUTPUTS = [(1, 300, 16400), (7, 130, 17001), (16, 640, 20000), (20, 200, 16385), (40, 129, 30011), (64, 300, 17000),
                (1, 700, 32801), (2, 64, 40000), (13, 200, 33333), (16, 128, 65536), (17, 130, 32800), (33, 250, 33001),
                (64, 100, 34567), (65, 100, 34567)]


@pytest.mark.parametrize("t,k,n", MANY_OUTPUTS)
@pytest.mark.parametrize("x_dtype,y_dtype,bias", [(BF16, F32, False), (F16, F16, True)])
def test_linear_to_very_many_outputs(t, k, n, x_dtype, y_dtype, bias):
    test_linear(t, k, n, x_dtype, y_dtype, bias)


@pytest.mark.parametrize("t", [1, 5, 40, 300])
def test_linear_strides_and_shapes(t):
    g = gen(t)
    big = normal(g, t, 403, dtype=F16)
    w = ops.pack_weight(normal(g, 50, 300))
    codes = w.codes.cpu().numpy()[oo.tile_index(50, 300)]
    x = big[:, 3:303]  # rows neither aligned nor packed
    y = torch.full((t, 64), 7.0, dtype=F16, device="cuda")
    assert ops.linear_i8(x, w, out=y[:, :50]).data_ptr() == y.data_ptr()
    check_linear(x, codes, f64(w.scale), None, y[:, :50], F16)
    assert (y[:, 50:] == 7.0).all()
    z = ops.linear_i8(x.reshape(t, 1, 300), w)
    assert z.shape == (t, 1, 50) and torch.equal(z[:, 0], y[:, :50])
    assert ops.linear_i8(x[:0], w).shape == (0, 50)


@pytest.mark.parametrize("t", [2, 8, 40, 300, 2100])
def test_linear_of_overlapping_rows(t):
    """A row broadcast to all tokens, and windows of one line."""
    g = gen(t + 1)
    line = normal(g, 200 + 3 * t, dtype=BF16)
    w = ops.pack_weight(normal(g, 40, 200))
    codes = w.codes.cpu().numpy()[oo.tile_index(40, 200)]
    one, windows = line[:200].expand(t, 200), line.unfold(0, 200, 3)[:t]
    for x in (one, windows):
        check_linear(x, codes, f64(w.scale), None, ops.linear_i8(x, w), BF16)
        packed, apart = ops.pack_weight(x), ops.pack_weight(x.contiguous())
        at = torch.from_numpy(oo.tile_index(t, 256)).cuda()  # (rows beyond the last hold anything)
        assert torch.equal(packed.codes[at], apart.codes[at]) and torch.equal(packed.scale, apart.scale)
    y = ops.linear_i8(line[:200].view(1, 1, 200).expand(t, 2, 200), w)
    assert y.shape == (t, 2, 40) and torch.equal(y, ops.linear_i8(line[None, :200], w).expand(t, 2, 40))
    for out in (torch.zeros(1, 40, dtype=BF16, device="cuda").expand(t, 40),
                torch.zeros(40 + t, dtype=BF16, device="cuda").unfold(0, 40, 1)[:t]):
        with pytest.raises(sim.SimError):
            ops.linear_i8(one, w, out=out)


@pytest.mark.parametrize("t", [3, 40, 2100])
def test_linear_of_values_at_the_ends_of_the_range(t):
    """Rows of very large and very small values, subnormal ones too, and rows
    whose values tie between two codes."""
    g = gen(t)
    w = ops.pack_weight(normal(g, 24, 320))
    codes = w.codes.cpu().numpy()[oo.tile_index(24, 320)]
    for dtype, sizes in ((BF16, (3e38, 1e37, 1e30, 2e-38, 5e-39, 1e-40)), (F16, (6e4, 1e-4, 3e-6, 6e-8))):
        for size in sizes:
            x = (torch.rand(t, 320, device="cuda", generator=g) * 2 - 1) * size
            x = x.to(dtype)
            assert np.array_equal(ops.pack_weight(x).codes.cpu().numpy()[oo.tile_index(t, 320)],
                                  oo.quantise_rows(f64(x))[0])
            if not 2e-36 < size < 1e35:
                continue  # scales that are subnormal, sums beyond fp32 once scaled
            check_linear(x, codes, f64(w.scale), None,
                         ops.linear_i8(x, w, dtype=F32), F32)
    x = torch.randint(-254, 255, (t, 320), device="cuda", generator=g)  # codes k + 0.5 where odd
    x[:, 0] = 254
    for dtype in (BF16, F16):
        check_linear(x.to(dtype), codes, f64(w.scale), None, ops.linear_i8(x.to(dtype), w, dtype=F32), F32)
        check_linear((x * 0.75).to(dtype), codes, f64(w.scale), None,
                     ops.linear_i8((x * 0.75).to(dtype), w, dtype=F32), F32)


# -------------------------------------------------------------------- cache

def make_cache(g, lengths, heads, dim, group, page, spare=0, scale=1.0):
    """A cache of random codes and parameters on shuffled pages."""
    counts = [-(-n // page) for n in lengths]
    pages = sum(counts) + spare
    table = torch.full((len(lengths), max(counts + [1])), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, device="cuda", generator=g).int()
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    c = ops.Cache.empty(pages, heads, dim, table, group=group, page=page)
    for x in (c.k, c.v):
        x.copy_(torch.randint(-2 ** 31, 2 ** 31, x.shape, device="cuda", generator=g))
    for x in (c.k_par, c.v_par):
        x[..., 0] = (torch.rand(x.shape[:-1], device="cuda", generator=g) * 0.3 + 0.05) * scale
        x[..., 1] = (torch.rand(x.shape[:-1], device="cuda", generator=g) * -3.0 - 0.5) * scale
    c.acc.copy_(torch.rand(c.acc.shape, device="cuda", generator=g) * 3)
    return c


def host(c):
    return {n: getattr(c, n).cpu().numpy() for n in ("k", "v", "k_par", "v_par", "pos", "acc", "page_table")}


def check_attention(c, q, lengths, out, scale=None, acc_in=None, acc_out=None, before=None):
    h = host(c)
    b_, t, hq, dim = q.shape
    heads, page = c._c.n_heads, c._c.page
    per = hq // heads
    sc = dim ** -0.5 if scale is None else scale
    got, qd = f64(out), f64(q)
    for b, n in enumerate(lengths):
        for j in range(heads):
            kc, vc, kp, vp = oo.read_cache(h["k"], h["v"], h["k_par"], h["v_par"], h["page_table"][b], j, n, page, dim,
                                           c._c.group)
            k, v = oo.values(kc, kp), oo.values(vc, vp)
            rows = qd[b, :, j * per:(j + 1) * per].reshape(t * per, dim)
            seen = np.arange(n)[None, :] < (n - t + 1 + np.arange(t).repeat(per))[:, None]
            o, p = oo.attend(rows, k, v, seen, sc)
            mine = got[b, :, j * per:(j + 1) * per].reshape(t * per, dim)
            # A logit sums dim products of |q| (16 + c) d, c <= 15, and terms
            # |q m|, each in fp32: (dim + 8) roundings of 2^-24 of the sum of
            # magnitudes, and three of the scaled logit.
            size = np.abs(rows) @ (31.0 * kp[..., 0] + np.abs(kp[..., 1])).T * sc
            delta = np.where(seen, (dim + 8) * 2.0 ** -24 * size, 0.0).max(axis=1, initial=0.0) + 2.0 ** -21 * np.where(
                seen, np.abs(rows @ k.T * sc), 0.0).max(axis=1, initial=0.0)
            # probabilities: twice that, exp and division; p d as two bf16
            # numbers 2^-17; sums over the slots of fp32
            rel = 2 * delta + 2.0 ** -17 + (n / 16 + 64) * 2.0 ** -24
            mag = p @ (31.0 * vp[..., 0] + np.abs(vp[..., 1]))
            slack = rel[:, None] * mag
            slack += HALF_ULP[q.dtype] * (np.abs(o) + slack) + TINY[q.dtype]
            off = np.abs(mine - o)
            assert np.all(off <= slack), (b, j, np.max(off / slack), n)
            if acc_out is not None:
                want = p.sum(0)
                slot = np.arange(n)
                pg, at = h["page_table"][b][slot // page], slot % page
                was = acc_in[pg, j, at].astype(np.float64) if acc_in is not None else np.zeros(n)
                new = acc_out[pg, j, at].astype(np.float64)
                slack_w = (p * (2 * delta + (n / 16 + 64 + t * per) * 2.0 ** -24)[:, None]).sum(0)
                slack_w += 2.0 ** -23 * (np.abs(was) + want) + 1e-37
                assert np.all(np.abs(new - was - want) <= slack_w), (b, j, np.max(np.abs(new - was - want) / slack_w))


ATTEND = [
    # lengths, queries, query heads, heads, dim, group, page
    ([1], 1, 1, 1, 64, 64, 32),
    ([0, 1, 2, 31, 32, 33], 1, 4, 2, 64, 32, 32),
    ([63, 64, 65, 0, 200], 1, 8, 1, 128, 64, 64),
    ([257, 1023], 1, 16, 2, 128, 32, 96),
    ([5, 700], 1, 40, 2, 128, 128, 128),
    ([2000], 1, 3, 1, 64, 64, 4096),
    ([3, 4, 50, 1], 4, 6, 2, 64, 32, 64),   # rows that see nothing
    ([300, 17, 129], 5, 6, 2, 128, 64, 32),
    ([150, 40], 40, 3, 1, 64, 64, 64),
    ([90], 90, 8, 2, 128, 128, 32),
    ([3000], 2, 8, 8, 64, 64, 64),
]


# Tables too long, or heads too many, for one workgroup to a head: the slots
# are dealt out in shares.
ATTEND += [
    ([5200], 1, 8, 2, 64, 32, 32),
    ([6000, 0, 1, 5300, 33], 1, 16, 2, 128, 64, 64),
    ([40, 7000], 1, 5, 1, 128, 128, 96),
    ([5500, 3, 90], 4, 6, 2, 64, 64, 128),
    ([5400, 60], 25, 2, 1, 128, 32, 64),       # 50 rows, several groups
    ([1500, 5200], 70, 3, 3, 64, 64, 32),
    ([31 + 7 * i for i in range(70)], 1, 4, 4, 64, 64, 32),  # more than 64 sequences
    ([0] * 66 + [100, 0, 0, 64], 2, 8, 4, 128, 64, 32),
    ([20] * 90, 20, 6, 3, 64, 32, 32),
    ([2500, 130], 100, 4, 1, 128, 64, 64),     # 400 rows: the codes expanded once for 128
    ([700, 3000, 65], 65, 2, 1, 64, 64, 32),
    ([1900], 33, 3, 1, 128, 32, 96),
]


@pytest.mark.parametrize("case", ATTEND, ids=[str(i) for i in range(len(ATTEND))])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("weights", [False, True])
def test_attention(case, dtype, weights):
    lengths, t, hq, heads, dim, group, page = case
    say("attend", case, dtype, weights)
    g = gen(sum(lengths) + t + dim)
    c = make_cache(g, lengths, heads, dim, group, page, spare=2)
    q = (normal(g, len(lengths), t, hq, dim) * 0.7).to(dtype)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if not weights:
        return check_attention(c, q, lengths, ops.attention_kv4(q, c, n))
    out = torch.full_like(c.acc, -5.0)
    o = ops.attention_kv4(q, c, n, acc_in=c.acc, acc_out=out)
    got = out.cpu().numpy()
    check_attention(c, q, lengths, o, acc_in=c.acc.cpu().numpy(), acc_out=got)
    # slots beyond the lengths keep what they held
    untouched = np.ones(got.shape, bool)
    table = c.page_table.cpu().numpy()
    for b, m in enumerate(lengths):
        slot = np.arange(m)
        untouched[table[b][slot // page], :, slot % page] = False
    assert (got[untouched] == -5.0).all()
    # in place, and without a starting weight
    again = torch.zeros_like(c.acc)
    ops.attention_kv4(q, c, n, acc_out=again)
    ops.attention_kv4(q, c, n, acc_in=c.acc, acc_out=c.acc)
    live = torch.from_numpy(~untouched).cuda()
    assert torch.equal(c.acc[live], out[live])
    assert torch.all((again[live] >= 0) & (again[live] <= t * hq / heads * (1 + 1e-3)))


# Many rows over short tables, a segment to a workgroup, with weights or not; some
# of one unseen sequence, of tables without pages, of rows that see nothing, and
# of more segments than two to a compute unit over tables of up to 2048 slots.
SHORT = [([0, 1, 40, 226], 33, 10, 2, 64, 64, 64), ([0, 0], 120, 2, 2, 64, 64, 32), ([300, 7], 128, 8, 8, 128, 64, 128),
         ([129, 130, 500], 100, 4, 2, 128, 128, 256), ([64, 81, 3], 64, 10, 2, 128, 32, 64), ([96], 25, 4, 2, 64, 32, 32),
         ([700, 10, 333, 0, 1500, 901, 64, 65], 96, 128, 16, 64, 64, 64)]


@pytest.mark.parametrize("case", SHORT, ids=[str(i) for i in range(len(SHORT))])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_of_many_rows_over_short_tables(case, dtype, weights):
    test_attention(case, dtype, weights)


# Few heads over long contexts, the parts of a row joined by sixteen wavefronts
# (64 parts and more); prompts of more than eight groups of 128 rows.
LONG = [([17001], 1, 1, 1, 64, 64, 64), ([9000, 8300], 1, 8, 2, 128, 64, 128), ([20011, 5], 2, 3, 1, 128, 32, 256),
        ([12345], 1, 5, 1, 64, 32, 32), ([11000], 1, 16, 1, 128, 128, 4096), ([2600, 900], 700, 4, 1, 128, 64, 64),
        ([1500], 1100, 2, 1, 64, 32, 32), ([1300], 1300, 1, 1, 128, 32, 64)]


@pytest.mark.parametrize("case", LONG, ids=[str(i) for i in range(len(LONG))])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_of_long_contexts_and_prompts(case, dtype, weights):
    test_attention(case, dtype, weights)


def with_room(c, slots):
    """The cache with a table for so many slots; its entries behind those of the lengths are anything."""
    g = gen(slots)
    t = c.page_table
    wide = torch.randint(-3, 10 ** 6, (t.shape[0], -(-slots // c._c.page)), dtype=torch.int32, device="cuda", generator=g)
    wide[:, :t.shape[1]] = t
    return dataclasses.replace(c, page_table=wide)


# A server's tables: far wider than the present contexts.
ROOM = [([300, 0, 1, 900], 1, 8, 2, 64, 64, 64, 32000), ([40, 33], 1, 16, 2, 128, 64, 32, 131072),
        ([5, 700, 64], 4, 6, 2, 128, 32, 96, 2000), ([500, 3], 130, 2, 1, 64, 32, 64, 32000),
        ([129, 250, 7], 96, 16, 4, 128, 128, 256, 2048), ([1, 1, 0], 20, 3, 3, 128, 64, 4096, 262144)]


@pytest.mark.parametrize("case", ROOM, ids=[str(i) for i in range(len(ROOM))])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_over_tables_with_room_to_grow(case, dtype, weights):
    lengths, t, hq, heads, dim, group, page, slots = case
    say("room", case, dtype, weights)
    g = gen(sum(lengths) + t)
    c = with_room(make_cache(g, lengths, heads, dim, group, page, spare=1), slots)
    q = (normal(g, len(lengths), t, hq, dim) * 0.7).to(dtype)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if not weights:
        return check_attention(c, q, lengths, ops.attention_kv4(q, c, n))
    out = torch.full_like(c.acc, -5.0)
    o = ops.attention_kv4(q, c, n, acc_in=c.acc, acc_out=out)
    check_attention(c, q, lengths, o, acc_in=c.acc.cpu().numpy(), acc_out=out.cpu().numpy())


@pytest.mark.parametrize("way", ["up", "down", "both"])
@pytest.mark.parametrize("rows,n", [(1, 700), (1, 6000), (40, 3000), (130, 3000)])
def test_attention_where_the_maximum_moves(way, rows, n):
    """Logits that rise or fall by hundreds along the context, exact in fp32, so
    that only the scaling of what was summed so far can be wrong."""
    say("maximum", way, rows, n)
    g = gen(n + rows)
    dim = 64
    c = make_cache(g, [n], 1, dim, 64, 64)
    for x in (c.k_par, c.v_par):
        x[..., 0] = 0.25
        x[..., 1] = -2.0
    # codes 15 where a channel counts, the more of them the further along
    slot = torch.arange(n, device="cuda")
    along = {"up": slot, "down": n - 1 - slot, "both": (2 * slot - n).abs()}[way] / (n - 1)
    codes = torch.where(torch.rand(n, dim, device="cuda", generator=g) < along[:, None], 15, 0).cpu().numpy()
    words = np.zeros((n, 4, 2), np.uint32)
    for ch in range(dim):
        words[:, ch // 8 % 4, ch // 32] |= codes[:, ch].astype(np.uint32) << np.uint32(oo.nibble(ch % 8))
    table = c.page_table[0].long()
    c.k[table[slot // 64], 0, slot % 64] = torch.from_numpy(words.view(np.int32)).cuda()
    q = torch.randint(1, 4, (1, 1, rows, dim), device="cuda", generator=g).to(F16)
    got = f64(ops.attention_kv4(q, c, torch.tensor([n], dtype=torch.int32, device="cuda"), scale=3.0))[0, 0]
    h = host(c)
    kc, vc, kp, vp = oo.read_cache(h["k"], h["v"], h["k_par"], h["v_par"], h["page_table"][0], 0, n, 64, dim, 64)
    assert np.array_equal(kc, codes)
    k, v, qd = oo.values(kc, kp), oo.values(vc, vp), f64(q)[0, 0]
    o, p = oo.attend(qd, k, v, np.ones((rows, n), bool), 3.0)
    # the logits are exact, scaled ones are rounded four times (the scale, its
    # product with log2 e, theirs with the logit, the difference); p twice that
    # much, p d as two bf16 numbers, sums of fp32
    rel = 8 * 2.0 ** -24 * np.abs(3.0 * qd @ k.T).max(1) + 2.0 ** -17 + (n / 16 + 64) * 2.0 ** -24
    slack = rel[:, None] * (p @ (31.0 * vp[..., 0] + np.abs(vp[..., 1])))
    slack += HALF_ULP[F16] * (np.abs(o) + slack) + TINY[F16]
    assert np.all(np.abs(got - o) <= slack), np.max(np.abs(got - o) / slack)


def test_attention_ignores_what_it_does_not_see():
    """Slots beyond a length, and slots after a query, may hold infinities and
    NaN; pages that do not exist hold no slots."""
    g = gen(9)
    lengths = [70, 33]
    c = make_cache(g, lengths, 2, 64, 64, 64, spare=1)
    q = normal(g, 2, 3, 4, 64, dtype=BF16)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want = ops.attention_kv4(q, c, n)
    for b, m in enumerate(lengths):
        for s in range(m, (m + 63) // 64 * 64):
            pg = int(c.page_table[b, s // 64])
            c.k_par[pg, :, :, s % 64] = float("nan")
            c.v_par[pg, :, :, s % 64] = float("inf")
    assert torch.equal(ops.attention_kv4(q, c, n), want)
    # the last slot is seen by the last query alone
    pg, at = int(c.page_table[0, 69 // 64]), 69 % 64
    c.v_par[pg, :, :, at] = float("nan")
    got = ops.attention_kv4(q, c, n)
    assert torch.isnan(got[0, 2]).all() and torch.equal(got[0, :2], want[0, :2]) and torch.equal(got[1], want[1])
    c.k_par[pg, :, :, at] = float("nan")
    got = ops.attention_kv4(q, c, n)
    assert torch.isnan(got[0, 2]).all() and torch.equal(got[0, :2], want[0, :2]) and torch.equal(got[1], want[1])
    c.page_table[:] = torch.where(c.page_table >= 0, 10 ** 6, -7)
    assert (ops.attention_kv4(q, c, n) == 0).all()
    # lengths beyond the table and below zero stay inside it
    assert (ops.attention_kv4(q, c, torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device="cuda")) == 0).all()


def test_attention_over_extreme_logits():
    """Logits far apart and large: the maximum moves many times."""
    g = gen(11)
    lengths = [900]
    c = make_cache(g, lengths, 1, 64, 32, 32, scale=8.0)
    q = (normal(g, 1, 1, 5, 64) * 4).to(F16)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    check_attention(c, q, lengths, ops.attention_kv4(q, c, n, scale=0.02), scale=0.02)
    o = ops.attention_kv4(q, c, n, scale=3.0)
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("dim,group,seqs,heads,n", [(64, 64, 1024, 1, 262144), (128, 32, 768, 2, 131072),
                                                    (64, 64, 512, 128, 65536), (128, 64, 512, 128, 40000)])
def test_attention_sums_over_long_runs(dim, group, seqs, heads, n):
    """Nearly flat attention over many slots, one segment to a workgroup: what is
    added up by one wavefront is far larger than the result.  All sequences
    share one sequence's pages."""
    say("long runs", dim, group, seqs, heads, n)
    g = gen(n + dim)
    c = make_cache(g, [n], 1, dim, group, 4096)
    for x in (c.k_par, c.v_par):  # values of mean 0, of one size
        x[..., 0] = 0.1370
        x[..., 1] = -7.5 * 0.1370
    shared = ops.Cache(c.k, c.v, c.k_par, c.v_par, c.pos, c.acc, c.page_table.expand(seqs, -1).contiguous())
    q = (normal(g, seqs, 1, heads, dim) * 0.2).to(F16)
    out = ops.attention_kv4(q, shared, torch.full((seqs,), n, dtype=torch.int32, device="cuda"))
    h = host(c)
    kc, vc, kp, vp = oo.read_cache(h["k"], h["v"], h["k_par"], h["v_par"], h["page_table"][0], 0, n, 4096, dim, group)
    k, v = oo.values(kc, kp), oo.values(vc, vp)
    pick = np.arange(0, seqs, seqs // 8)
    rows = f64(q)[pick, 0, :2].reshape(-1, dim)
    o, _ = oo.attend(rows, k, v, np.ones((len(rows), n), bool), dim ** -0.5)
    off = f64(out)[pick, 0, :2].reshape(-1, dim) - o
    # Rounding to fp16 is off by 2^-11 at most, 2^-11 / sqrt(3) in the mean of
    # squares where all significands were 1.  Before it, sums of at most 8 blocks
    # of 32 slots of p d (16 + c), c <= 15, are rounded twice a block, by 2^-25 of
    # 8 * 32 * 31 p d at most, as if at random, against a result of
    # sqrt(n) times the codes' spread, 4.6 p d: sqrt(2 n / 32) 2^-25 7936 /
    # (4.6 sqrt(n)) = 1.3e-5 for any n.  2^-14 leaves four times that and p d's
    # 17 bits.
    assert np.linalg.norm(off) <= (2.0 ** -11 / 3 ** 0.5 + 2.0 ** -14) * np.linalg.norm(o), np.linalg.norm(
        off) / np.linalg.norm(o)


@pytest.mark.parametrize("rows,n", [(1, 100), (1, 3000), (40, 3000), (130, 1000)])
def test_attention_over_the_largest_logits(rows, n):
    """All logits far below zero, or above, up to 2^30: the largest one takes all, its value comes out as it is."""
    say("largest logits", rows, n)
    g = gen(n + rows)
    c = make_cache(g, [n], 1, 64, 64, 64)
    for x in (c.k_par, c.v_par):
        x[..., 0] = 0.25
        x[..., 1] = 0.5  # keys of 0.5 to 4.25: every logit has the sign of q
    h = host(c)
    kc, vc, kp, vp = oo.read_cache(h["k"], h["v"], h["k_par"], h["v_par"], h["page_table"][0], 0, n, 64, 64, 64)
    k, v = oo.values(kc, kp), oo.values(vc, vp)
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    for size, scale in ((-2.0 ** 18, 1.0), (2.0 ** 18, 1.0), (-1.0, 2.0 ** 18), (-2.0 ** -90, 2.0 ** 108), (2.0 ** 21, 0.125), (-0.01, 3.0)):
        q = (size * 2.0 ** torch.randint(0, 3, (1, 1, rows, 64), device="cuda", generator=g)).to(BF16)
        out = f64(ops.attention_kv4(q, c, lengths, scale=scale))[0, 0]
        weights = torch.zeros_like(c.acc)
        assert np.array_equal(f64(ops.attention_kv4(q, c, lengths, scale=scale, acc_out=weights))[0, 0], out)
        a = f64(q)[0, 0] @ k.T * scale
        assert np.abs(a).max() < 2.0 ** 30
        got = np.argsort(-a, axis=1)
        first, second = (np.take_along_axis(a, got[:, i:i + 1], 1)[:, 0] for i in (0, 1))
        # fp32 sums of 64 products tell them apart where they differ by 2^-16 of their size
        clear = first - second > 2.0 ** -16 * np.abs(first) + 40.0  # (e^-40 of another value is nothing)
        assert clear.any() or abs(size * scale) < 1.0
        # all weight on one slot: the output's rounding, and p d as two bf16 numbers
        want = v[got[:, 0]]
        assert np.all(np.abs(out - want)[clear] <= 2.0 ** -8 * np.abs(want)[clear] + 2.0 ** -17 * (31 * 0.25 + 0.5)), (
            size, scale)
        pg = h["page_table"][0][np.arange(n) // 64]
        assert weights.cpu().numpy()[pg, 0, np.arange(n) % 64].sum() == pytest.approx(rows, rel=1e-5)


def test_attention_query_strides():
    g = gen(13)
    lengths = [50, 20, 77]
    c = make_cache(g, lengths, 2, 64, 64, 32)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    qkv = normal(g, 3, 2, 8, 64, dtype=BF16)  # queries, keys and values side by side
    q = qkv[:, :, :4]
    want = ops.attention_kv4(q.contiguous(), c, n)
    assert torch.equal(ops.attention_kv4(q, c, n), want)
    odd = torch.empty(3 * 2 * 4 * 64 + 1, dtype=BF16, device="cuda")[1:].view(3, 2, 4, 64)
    odd.copy_(q)
    assert torch.equal(ops.attention_kv4(odd, c, n), want)


def test_attention_of_one_token_at_any_stride():
    g = gen(14)
    c = make_cache(g, [50], 2, 64, 64, 32)
    n = torch.tensor([50], dtype=torch.int32, device="cuda")
    line = normal(g, 2048, dtype=F16)
    want = ops.attention_kv4(line[:256].view(1, 1, 4, 64), c, n)
    for strides in ((1003, 256, 64, 1), (1003, 77, 64, 1), (0, 0, 64, 1)):
        assert torch.equal(ops.attention_kv4(line.as_strided((1, 1, 4, 64), strides), c, n), want)
    two = line[256:].as_strided((1, 2, 4, 64), (5, 300, 64, 1))  # 300 is no multiple of 8
    assert torch.equal(ops.attention_kv4(two, c, n), ops.attention_kv4(two.clone(memory_format=torch.contiguous_format), c, n))


@pytest.mark.parametrize("dim,group,page", [(64, 32, 32), (64, 64, 64), (128, 32, 96), (128, 64, 32), (128, 128, 64)])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("starts,t", [([0, 5, 31], 1), ([0, 32, 40], 33), ([7, 0, 90], 70)])
def test_append(dim, group, page, dtype, starts, t):
    say("append", dim, group, page, dtype, starts, t)
    g = gen(dim + group + t)
    heads = 3
    lengths = [s + t for s in starts]
    c = make_cache(g, lengths, heads, dim, group, page)
    before = host(c)
    k, v = normal(g, 3, t, heads, dim, dtype=dtype), normal(g, 3, t, heads, dim, dtype=dtype)
    k[0, 0, 0, :group] = 2.5  # all alike: scale 0
    k[1, 0, 1, 3] = 60000.0
    if dtype == BF16:
        v[1, 0, 2, 5] = 1e30  # clamped
        v[2, 0, 0, 1] = float("-inf")
    k[2, 0, 2, 0] = float("nan")
    start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    first = torch.tensor([100, 7, 0], dtype=torch.int32, device="cuda")
    hk, hv = ops.cache_append(c, k, v, start, first_pos=first, held=True)
    after = host(c)
    for b in range(3):
        for j in range(heads):
            n = starts[b] + t
            old = oo.read_cache(*(before[x] for x in ("k", "v", "k_par", "v_par")), before["page_table"][b], j, n, page,
                                dim, group)
            new = oo.read_cache(*(after[x] for x in ("k", "v", "k_par", "v_par")), before["page_table"][b], j, n, page,
                                dim, group)
            for a, z in zip(old, new):  # older tokens stay
                assert np.array_equal(a[:starts[b]], z[:starts[b]])
            for x, codes, par, held in ((k, new[0], new[2], hk), (v, new[1], new[3], hv)):
                want, d, m = oo.quantise_token(f64(x[b, :, j]), group)
                bad = np.isnan(f64(x[b, :, j])).reshape(t, -1, group).any(-1).repeat(group, -1)
                d, m = (np.where(bad, np.nan, y.astype(np.float64).repeat(group, -1)) for y in (d, m))
                want = np.where(bad, 0, want)
                got_c, got_p = codes[starts[b]:], par[starts[b]:]
                assert np.array_equal(got_p[..., 0], d, equal_nan=True)
                assert np.array_equal(got_p[..., 1], m, equal_nan=True)
                assert np.array_equal(got_c, want)
                # code * d is exact, the sum rounded once
                assert np.array_equal(f64(held[b, :, j]), (want * d + m).astype(np.float32).astype(np.float64),
                                      equal_nan=True)
            slot = starts[b] + np.arange(t)
            pg, at = before["page_table"][b][slot // page], slot % page
            assert np.array_equal(after["pos"][pg, j, at], int(first[b]) + np.arange(t))
            assert (after["acc"][pg, j, at] == 0).all()
    # nothing else changed
    for x in ("pos", "acc"):
        same = np.ones(before[x].shape, bool)
        for b in range(3):
            slot = starts[b] + np.arange(t)
            same[before["page_table"][b][slot // page], :, slot % page] = False
        assert np.array_equal(before[x][same], after[x][same])


@pytest.mark.parametrize("dim,group,page,starts,t", [(64, 32, 32, [0, 5, 64], 1000), (128, 64, 96, [31, 0, 7], 517),
                                                     (128, 128, 4096, [100, 2, 33], 800), (64, 64, 64, [1, 0, 0], 1)])
def test_append_of_prompts(dim, group, page, starts, t):
    for dtype in (BF16, F16):
        test_append(dim, group, page, dtype, starts, t)


def test_append_beyond_the_table_writes_nothing_there():
    g = gen(3)
    c = make_cache(g, [40, 40], 1, 64, 64, 32, spare=1)
    before = host(c)
    k = normal(g, 2, 6, 1, 64, dtype=F16)
    c.page_table[1, 1] = 999
    start = torch.tensor([61, 30], dtype=torch.int32, device="cuda")
    ops.cache_append(c, k, k, start)
    after = host(c)
    table = before["page_table"]
    used = np.zeros(before["acc"].shape, bool)
    used[table[0, 1], :, 29:32] = True
    used[table[1, 0], :, 30:32] = True
    assert np.array_equal(before["acc"][~used], after["acc"][~used]) and (after["acc"][used] == 0).all()
    kept = ~used.any(axis=(1, 2))
    assert np.array_equal(before["k"][kept], after["k"][kept]) and np.array_equal(before["v"][kept], after["v"][kept])


def test_sequences_that_share_their_first_pages():
    """Attention without weights, and a cut out of shared pages, as with pages of
    their own; weights with pages of their own."""
    g = gen(6)
    lengths, shared = [150, 97, 64, 300], 2  # 64 slots in common
    own = make_cache(g, lengths, 2, 64, 32, 32, spare=1)
    table = own.page_table.clone()
    table[1:, :shared] = table[0, :shared]
    c = dataclasses.replace(own, page_table=table)
    for name in ("k", "v", "k_par", "v_par", "pos", "acc"):
        x = getattr(own, name)
        x[own.page_table[1:, :shared].long()] = x[table[1:, :shared].long()]
    q = normal(g, 4, 3, 6, 64, dtype=F16)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    o = ops.attention_kv4(q, c, n)
    check_attention(c, q, lengths, o)
    weights = torch.zeros_like(own.acc)
    assert torch.equal(ops.attention_kv4(q, own, n, acc_out=weights), o)
    check_attention(own, q, lengths, o, acc_out=weights.cpu().numpy())
    at = torch.arange(own.pos.shape[0] * 32, device="cuda").view(-1, 1, 32).expand(-1, 2, 32).int()
    own.pos.copy_(at)
    own.pos[own.page_table[1:, :shared].long()] = own.pos[table[1:, :shared].long()]
    kept = []
    for src in (c, own):
        dst = ops.Cache.empty(12, 2, 64, torch.arange(12, dtype=torch.int32, device="cuda").view(4, 3), group=32, page=32)
        new = ops.cache_evict(src, dst, n, torch.full_like(n, 10 ** 6), keep=80, recent=0)
        kept.append([new, dst.k, dst.v, dst.k_par, dst.v_par, dst.pos, dst.acc])
    assert all(torch.equal(a, z) for a, z in zip(*kept)) and kept[0][0].tolist() == [80, 80, 64, 80]


def test_a_longer_table_makes_another_cache():
    g = gen(4)
    c = make_cache(g, [40, 64], 2, 64, 64, 32, spare=3)
    q = normal(g, 2, 1, 4, 64, dtype=BF16)
    n = torch.tensor([40, 64], dtype=torch.int32, device="cuda")
    want = ops.attention_kv4(q, c, n)
    wide = torch.cat([c.page_table, torch.full((2, 9), -1, dtype=torch.int32, device="cuda")], 1)
    with pytest.raises(AttributeError):
        c.page_table = wide
    d = dataclasses.replace(c, page_table=wide)
    assert d.k is c.k and d.bytes_per_slot == c.bytes_per_slot and torch.equal(ops.attention_kv4(q, d, n), want)
    free = torch.tensor(sorted(set(range(c.k.shape[0])) - set(c.page_table.flatten().tolist())))
    d.page_table[0, 2] = int(free[0])
    ops.cache_append(d, normal(g, 2, 1, 2, 64, dtype=BF16), normal(g, 2, 1, 2, 64, dtype=BF16),
                     torch.tensor([64, 300], dtype=torch.int32, device="cuda"))
    assert (c.acc[int(free[0]), :, 0] == 0).all() and torch.equal(ops.attention_kv4(q, d, n), want)


# ----------------------------------------------------------------- eviction

EVICT = [
    # lengths, heads, dim, group, source page, destination page, keep, recent
    ([1, 0, 5], 1, 64, 64, 32, 32, 1, 0),
    ([33, 64, 31, 32], 2, 64, 32, 32, 64, 32, 5),
    ([100, 300, 1000], 3, 128, 64, 64, 32, 77, 77),
    ([2500, 10], 2, 128, 128, 96, 64, 1000, 100),
    ([5000], 1, 64, 64, 256, 128, 64, 0),
    ([9000, 12000], 2, 64, 64, 64, 64, 4097, 1),
]


@pytest.mark.parametrize("case", EVICT, ids=[str(i) for i in range(len(EVICT))])
@pytest.mark.parametrize("kind", ["plain", "ties", "special"])
def test_evict(case, kind):
    lengths, heads, dim, group, page, dpage, keep, recent = case
    say("evict", case, kind)
    g = gen(sum(lengths) + keep)
    src = make_cache(g, lengths, heads, dim, group, page, spare=1)
    if kind == "ties":
        src.acc.copy_((src.acc * 1.3).floor())
    if kind == "special":
        pick = torch.rand(src.acc.shape, device="cuda", generator=g)
        for lo, val in ((0.0, float("nan")), (0.05, float("inf")), (0.1, -0.0), (0.2, 0.0), (0.3, -1.5),
                        (0.35, float("-inf")), (0.4, 1e-42)):
            src.acc[(pick >= lo) & (pick < lo + 0.05)] = val
    # positions with gaps, in slot order, differing by head
    table = src.page_table.cpu().numpy()
    rng = np.random.default_rng(len(lengths))
    total = []
    for b, n in enumerate(lengths):
        last = 0
        pos = []
        for j in range(heads):
            p = np.cumsum(rng.integers(1, 3, n)) - 1
            pos.append(p)
            last = max(last, int(p[-1]) + 1 if n else 0)
        total.append(last)
        for j in range(heads):
            p = pos[j] + (last - 1 - pos[j][-1] if n else 0)
            slot = np.arange(n)
            src.pos[torch.from_numpy(table[b][slot // page].astype(np.int64)).cuda(), j,
                    torch.from_numpy(slot % page).cuda()] = torch.from_numpy(p.astype(np.int32)).cuda()
    dst = make_cache(g, [keep] * len(lengths), heads, dim, group, dpage, spare=1)
    before, there = host(src), host(dst)
    new = ops.cache_evict(src, dst, torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                          torch.tensor(total, dtype=torch.int32, device="cuda"), keep=keep, recent=recent)
    assert new.tolist() == [min(n, keep) for n in lengths]
    after, same = host(dst), host(src)
    for x in before:
        assert before[x].tobytes() == same[x].tobytes(), x  # the source stays
    written = np.zeros(there["acc"].shape, bool)
    for b, n in enumerate(lengths):
        for j in range(heads):
            slot = np.arange(n)
            pg, at = table[b][slot // page], slot % page
            acc, pos = before["acc"][pg, j, at], before["pos"][pg, j, at]
            stay = oo.keep_slots(acc, pos, total[b], keep, recent)
            m = len(stay)
            to = np.arange(m)
            dpg, dat = there["page_table"][b][to // dpage], to % dpage
            written[dpg, j, dat] = True
            assert np.array_equal(after["pos"][dpg, j, dat], pos[stay]), (b, j)
            assert np.array_equal(after["acc"][dpg, j, dat].view(np.uint32), acc[stay].view(np.uint32))
            a = oo.read_cache(*(before[x] for x in ("k", "v", "k_par", "v_par")), table[b], j, n, page, dim, group)
            full = -(-m // 32) * 32
            z = oo.read_cache(*(after[x] for x in ("k", "v", "k_par", "v_par")), there["page_table"][b], j, full, dpage,
                              dim, group)
            for x, y in zip(a, z):
                assert np.array_equal(x[stay], y[:m])
            assert not z[1][m:].any()  # values' codes behind the last one
    assert np.array_equal(there["acc"][~written], after["acc"][~written])
    assert np.array_equal(there["pos"][~written], after["pos"][~written])


# Longer than 16,384 slots, and than the 65,536 that a workgroup's registers hold:
# ties on both sides of the border, one slot behind it, all before it.
LONG_EVICT = [([20000, 33], 2, 64, 64, 64, 128, 5000, 100), ([70001], 1, 64, 32, 4096, 64, 69000, 7),
              ([66000, 300], 1, 128, 64, 256, 64, 500, 3), ([65537, 65536], 1, 64, 64, 128, 32, 65500, 65000),
              ([140000], 1, 64, 64, 4096, 4096, 20000, 0)]


@pytest.mark.parametrize("case", LONG_EVICT, ids=[str(i) for i in range(len(LONG_EVICT))])
@pytest.mark.parametrize("kind", ["plain", "ties", "special"])
def test_evict_of_long_caches(case, kind):
    test_evict(case, kind)


@pytest.mark.parametrize("slots", [3000, 20000, 140000])
def test_evict_from_tables_with_room_to_grow(slots):
    """As from a table of the present length."""
    g = gen(slots)
    lengths = [700, 5, 0, 1300]
    src = make_cache(g, lengths, 2, 64, 32, 64, spare=1)
    src.pos.copy_(torch.randperm(src.pos.numel(), device="cuda", generator=g).view_as(src.pos))
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    found = []
    for c in (src, with_room(src, slots)):
        table = torch.arange(4 * 13, dtype=torch.int32, device="cuda").view(4, 13)
        dst = ops.Cache.empty(4 * 13, 2, 64, table, group=32, page=32)
        new = ops.cache_evict(c, dst, n, torch.full_like(n, src.pos.numel()), keep=400, recent=100)
        found.append([new, dst.k, dst.v, dst.k_par, dst.v_par, dst.pos, dst.acc])
    assert all(torch.equal(a, z) for a, z in zip(*found)) and found[0][0].tolist() == [400, 5, 0, 400]


def test_the_long_cases_reach_their_kernels():
    """Those that only many outputs, long tables or few long segments choose (on a device of 256 compute units)."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the sizes are for 256 compute units")
    g = gen(2)

    def names(f):
        return " ".join(kernels_run(f))

    for t, n, want in ((3, 17001, "0, 2, 1, true>"), (3, 32801, "0, 4, 1, true>"), (40, 17001, "0, 2, 3, false>"),
                       (40, 33001, "0, 4, 3, false>")):
        x, w = normal(g, t, 130, dtype=BF16), ops.pack_weight(normal(g, n, 130))
        assert f"product_few<0, {want}" in names(lambda: ops.linear_i8(x, w)), (t, n)
    for n in (17001, 70001):
        src, dst = make_cache(g, [n], 1, 64, 64, 4096), make_cache(g, [64], 1, 64, 64, 32)
        lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
        assert "evict_select<16>" in names(lambda: ops.cache_evict(src, dst, lengths, lengths, keep=64, recent=3)), n
        q = normal(g, 1, 1, 1, 64, dtype=BF16)
        assert "join<0, 64, 1, 1024>" in names(lambda: ops.attention_kv4(q, src, lengths)), n


# --------------------------------------------------------- streams and graphs

def test_a_step_on_another_stream_and_in_a_graph():
    """linear, append, attention with weights and eviction on a side stream and
    replayed from a graph give what they give at once."""
    g = gen(21)
    lengths = [300, 45]
    w = ops.pack_weight(normal(g, 3 * 4 * 64, 256))
    x = normal(g, 2, 256, dtype=BF16)
    base = make_cache(g, [n + 1 for n in lengths], 4, 64, 64, 32)
    base.pos.copy_(torch.arange(32, device="cuda").expand_as(base.pos))
    start = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    after = start + 1
    acc = torch.zeros_like(base.acc)
    dst = ops.Cache.empty(4, 4, 64, torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2), page=32)

    def step():
        qkv = ops.linear_i8(x, w).view(2, 1, 12, 64)
        ops.cache_append(base, qkv[:, :, 4:8], qkv[:, :, 8:], start)
        o = ops.attention_kv4(qkv[:, :, :4], base, after, acc_in=base.acc, acc_out=acc)
        n = ops.cache_evict(base, dst, after, after, keep=64, recent=8)
        return o, n

    o, n = step()
    torch.cuda.synchronize()
    want = [o.clone(), n.clone(), acc.clone(), dst.k.clone(), dst.v.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (acc, dst.k, dst.v):
        t.zero_()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        o, n = step()
    torch.cuda.synchronize()
    for a, z in zip(want, [o, n, acc, dst.k, dst.v]):
        assert torch.equal(a, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go, gn = step()
    for i in range(4):
        for t in (acc, go, dst.k, dst.v):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, z in zip(want, [go, gn, acc, dst.k, dst.v]):
            assert torch.equal(a, z), i
        assert torch.equal(step()[0], want[0])  # eager work between the replays


def test_refusals():
    g = gen(1)
    w = ops.pack_weight(normal(g, 32, 64))
    x = normal(g, 4, 64, dtype=BF16)
    c = make_cache(g, [40], 2, 64, 64, 32)
    q = normal(g, 1, 1, 4, 64, dtype=BF16)
    n = torch.tensor([40], dtype=torch.int32, device="cuda")
    bad = [
        lambda: ops.linear_i8(x.float(), w),
        lambda: ops.linear_i8(x[:, :63], w),
        lambda: ops.linear_i8(x.cpu(), w),
        lambda: ops.linear_i8(x, w, dtype=torch.float64),
        lambda: ops.linear_i8(x, w, bias=normal(g, 31)),
        lambda: ops.linear_i8(x, w, out=torch.empty(4, 31, dtype=BF16, device="cuda")),
        lambda: ops.linear_i8(x, ops.PackedWeight(w.codes[:-1], w.scale, 32, 64)),
        lambda: ops.attention_kv4(q[..., :32], c, n),
        lambda: ops.attention_kv4(q[:, :, :3], c, n),
        lambda: ops.attention_kv4(q, c, n.long()),
        lambda: ops.attention_kv4(q, c, n, scale=0.0),
        lambda: ops.attention_kv4(q, c, n, scale=float("nan")),
        lambda: ops.attention_kv4(q, c, n, acc_in=c.acc),
        lambda: ops.attention_kv4(q, c, n, acc_out=c.acc[:1]),
        lambda: ops.attention_kv4(q, c, torch.cat([n, n])),
        lambda: ops.cache_append(c, q[:, :, :2], q[:, :, :2].half(), n),
        lambda: ops.cache_append(c, q, q, n),
        lambda: ops.cache_evict(c, c, n, n, keep=0, recent=0),
        lambda: ops.cache_evict(c, c, n, n, keep=65, recent=0),
        lambda: ops.cache_evict(c, c, n, n, keep=8, recent=9),
        lambda: ops.Cache(k=c.k, v=c.v, k_par=c.k_par, v_par=c.v_par, pos=c.pos[:, :1], acc=c.acc,
                          page_table=c.page_table),
        lambda: ops.Cache(k=c.k, v=c.v[..., :1], k_par=c.k_par, v_par=c.v_par, pos=c.pos, acc=c.acc,
                          page_table=c.page_table),
    ]
    for f in bad:
        with pytest.raises(sim.SimError):
            f()
