"""Attention over packed prompts at the ends of its values' range, on the GPU, against
the 64-bit definition."""
import numpy as np
import pytest
import torch

import prompt_oracle as po
from gpu_common import say
from paper_2302_11665_amd import ops
from test_gpu_ops import BF16, F16, HALF_ULP, TINY, f64, gen, normal
from test_gpu_prompt_ops import ints, prompt

pytestmark = pytest.mark.gpu


def check_rows(q, k, v, lengths, out, scale, skip=()):
    """Rows of sequences but those in `skip`, whose logits are exact or small."""
    qd, kd, vd, got = f64(q), f64(k), f64(v), f64(out)
    per, u, dim = q.shape[1] // k.shape[1], HALF_ULP[q.dtype], q.shape[2]
    at = 0
    for b, n in enumerate(lengths):
        rows = slice(at, at + n)
        at += n
        for j in range(q.shape[1] if n and b not in skip else 0):
            ks, vs = kd[rows, j // per], vd[rows, j // per]
            with np.errstate(over="ignore"):  # of what is masked
                o, p, a = po.attend_causal(qd[rows, j], ks, vs, scale)
            # A logit: dim products in fp32, 2^-24 each of the sum of magnitudes; its scaling, the
            # reference and scale log2 e, four of its size.  0 where logits are 0 or one exact product.
            size = np.abs(qd[rows, j]) @ np.abs(ks).T * scale
            delta = (dim * size.max() + 8 * (np.abs(a).max() + 4)) * 2.0 ** -24 if np.abs(a).max() < 1000 else 0.0
            # A weight: twice that, exp2 2^-23, its quotient by the sum and the output's by
            # theirs, four roundings of 2^-24; once to the type.  Sums: a term each 16 slots.
            rel = 2 * delta + 2.0 ** -23 + 4 * 2.0 ** -24 + u + (n / 8 + 16) * 2.0 ** -24
            slack = rel * (p @ np.abs(vs))
            if q.dtype == F16:  # weights below 2^-14 of the largest are subnormal in fp16
                slack += 2.0 ** -25 * np.cumsum(np.abs(vs), axis=0)
            slack += u * (np.abs(o) + slack) + TINY[q.dtype]
            off = np.abs(got[rows, j] - o)
            assert np.all(off <= slack), (b, j, n, np.nanmax(off / slack), np.isfinite(off).all())


# Blocks found by a search, listed, and split in parts that are joined.
LARGE = [([4], 1, 1, 64), ([1, 70, 0, 300], 4, 2, 128), ([200, 3], 6, 2, 64), ([33] * 66 + [200], 2, 1, 64),
         ([2, 0, 140] * 23, 2, 2, 128), ([1700, 300], 2, 1, 128), ([2049], 3, 1, 64)]


@pytest.mark.parametrize("case", LARGE, ids=[str(i) for i in range(len(LARGE))])
@pytest.mark.parametrize("logits", ["equal", "random", "largest"])
def test_prompt_of_large_values(case, logits):
    """Sums of values times weights would pass fp32's range, results do not; small values beside them stay."""
    lengths, heads, kv_heads, dim = case
    say("large values", case, logits)
    g = gen(sum(lengths) + dim)
    q, k, v, offsets = (x.clone() for x in prompt(g, lengths, heads, kv_heads, dim, BF16))
    if logits != "random":
        q.zero_()
    if logits == "largest":
        q[..., 3], k[..., 3] = 1.0, (torch.randint(0, 8, k.shape[:2], device="cuda", generator=g) * 30 + 45) * 2.0 ** 22
    sign = torch.randint(0, 2, (1, *v.shape[1:]), device="cuda", generator=g) * 2 - 1  # most channels of one sign
    v = ((1e38 + 2.2e38 * torch.rand(v.shape, device="cuda", generator=g)) * sign).to(BF16)
    v[..., 5] = (1e-30 * normal(g, *v.shape[:2])).to(BF16)
    out = ops.attention_prompt(q, k, v, offsets, scale=0.125)
    check_rows(q, k, v, lengths, out, 0.125)


@pytest.mark.parametrize("case", LARGE[1:], ids=[str(i) for i in range(1, len(LARGE))])
def test_prompt_of_large_values_beside_others_that_are_not_finite(case):
    lengths, heads, kv_heads, dim = case
    say("large values, not finite", case)
    g = gen(sum(lengths) + dim)
    q, k, v, offsets = (x.clone() for x in prompt(g, lengths, heads, kv_heads, dim, BF16))
    v = (1e38 + 2.2e38 * torch.rand(v.shape, device="cuda", generator=g)).to(BF16)
    b = int(np.argmax(lengths))
    begin, end = sum(lengths[:b]), sum(lengths[:b + 1])
    bad = begin + lengths[b] // 2
    for value in (float("nan"), float("inf"), -float("inf")):
        w = v.clone()
        w[bad, :, ::3] = value
        out = ops.attention_prompt(q, k, w, offsets)
        hit, rest = torch.zeros(dim, dtype=torch.bool), slice(begin, bad)
        hit[::3] = True
        assert not torch.isfinite(out[bad:end][:, :, hit]).any()
        assert torch.isfinite(out[bad:end][:, :, ~hit]).all() and torch.isfinite(out[rest]).all()
        check_rows(q[rest], k[rest], v[rest], [bad - begin], out[rest], dim ** -0.5)
        check_rows(q[:begin], k[:begin], v[:begin], lengths[:b], out[:begin], dim ** -0.5)


def test_prompt_of_large_values_in_fp16():
    g = gen(8)
    lengths = [300, 5]
    q, k, v, offsets = (x.clone() for x in prompt(g, lengths, 2, 1, 64, F16))
    q.zero_()
    v = (65000.0 - 3000 * torch.rand(v.shape, device="cuda", generator=g)).to(F16)
    check_rows(q, k, v, lengths, ops.attention_prompt(q, k, v, offsets, scale=1.0), 1.0)


def test_prompt_with_many_offsets_that_make_no_sense():
    """Sequences that all have all tokens: 2^33 blocks of rows, of which those that can be are worked on, inside the
    arrays."""
    g = gen(4)
    t, heads, seqs = 8192, 256, 1 << 20
    q, k, v = normal(g, t, heads, 64, dtype=BF16), normal(g, t, 1, 64, dtype=BF16), normal(g, t, 1, 64, dtype=BF16)
    offsets = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    offsets[1::2] = t
    out = torch.full((t + 64, heads, 64), 5.0, dtype=BF16, device="cuda")
    say("offsets that make no sense", seqs)
    ops.attention_prompt(q, k, v, offsets, out=out[32:-32])
    torch.cuda.synchronize()
    assert (out[:32] == 5).all() and (out[-32:] == 5).all()
    offsets[:-1] = torch.randint(-t, 2 * t, (seqs,), device="cuda", generator=g)
    ops.attention_prompt(q, k, v, offsets[-5000:].contiguous(), out=out[32:-32])
    torch.cuda.synchronize()
    assert (out[:32] == 5).all() and (out[-32:] == 5).all()
