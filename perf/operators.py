"""The operators of a served model's step, as cases to be timed.

The placement searches plan with what a model costs on a device: its bytes and
its time per step.  For a model that generates, these operators set both:
  linear  matrix product in 8-bit integers, activations quantised per token,
          weights per output channel
  attend  attention of a step's queries over a paged cache held in 4 bits,
          with the attention weight of every cached token where asked for
  step    a step's new tokens appended to that cache, then attended
  evict   a cache cut to a budget: the newest tokens, and of the others those
          of the largest accumulated attention weight

Where `own` is false the plain forms run: elementary torch operations in 32
bits.  Where it is true the package's operators run.  Both read the same state.
Codes of a cache that `evict` moves come back as the words that hold them:
they are whole numbers that are moved, not computed, and have to be equal.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # One token of one request through a square projection: the smallest
        # call of a step, where launches count.
        dict(name="linear_token", kind="linear", tokens=1, inputs=4096, outputs=4096, type="bf16", out="bf16",
             bias=False),
        # A batch of requests' tokens through a wide projection: the weights'
        # bytes count.
        dict(name="linear_batch", kind="linear", tokens=48, inputs=4096, outputs=16384, type="f16", out="f16",
             bias=True),
        # Sizes that fit no tile, with a bias and 32-bit results (a last
        # projection).
        dict(name="linear_odd", kind="linear", tokens=333, inputs=1500, outputs=2777, type="bf16", out="f32",
             bias=True),
        # Prompts of several requests through a large projection: the matrix
        # rate counts.
        dict(name="linear_prompt", kind="linear", tokens=4096, inputs=8192, outputs=8192, type="bf16", out="bf16",
             bias=False),
        # One request's token over a short context: latency.
        dict(name="attend_one", kind="attend", seqs=1, queries=1, heads=32, kv_heads=8, dim=128, group=64, page=64,
             len_lo=4100, len_hi=4100, type="bf16", weights=False),
        # Drafted tokens of a few requests checked together, small heads, few
        # channels to a scale, with the cached tokens' weights.
        dict(name="attend_draft", kind="attend", seqs=6, queries=5, heads=24, kv_heads=8, dim=64, group=32, page=32,
             len_lo=1001, len_hi=30000, type="f16", weights=True),
        # A part of a prompt (300 tokens of each of two requests) over what
        # came before it: compute counts.
        dict(name="attend_chunk", kind="attend", seqs=2, queries=300, heads=32, kv_heads=8, dim=128, group=128,
             page=128, len_lo=5003, len_hi=12000, type="bf16", weights=False),
        # A few requests with very long contexts: the cache's bytes count.
        dict(name="attend_long", kind="attend", seqs=4, queries=1, heads=64, kv_heads=8, dim=128, group=64, page=256,
             len_lo=180007, len_hi=260000, type="bf16", weights=False),
        # A step of a small batch on one device.
        dict(name="step_few", kind="step", seqs=3, queries=1, heads=16, kv_heads=4, dim=64, group=64, page=64,
             len_lo=300, len_hi=1900, type="f16"),
        # A step of a full batch with ragged contexts, weights accumulated.
        dict(name="step_batch", kind="step", seqs=40, queries=1, heads=64, kv_heads=8, dim=128, group=64, page=64,
             len_lo=700, len_hi=16000, type="bf16"),
        # Caches of a few requests cut back to their budget after a while of
        # generating.
        dict(name="evict_steady", kind="evict", seqs=5, kv_heads=4, dim=128, group=64, page=64, len_lo=1040,
             len_hi=1300, keep=1024, recent=128),
        # Long prompts' caches cut to an eighth once they are read.
        dict(name="evict_prompts", kind="evict", seqs=12, kv_heads=8, dim=128, group=64, page=64, len_lo=20011,
             len_hi=65000, keep=6000, recent=500),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, n if n != 3072 else n + 1))


def draw(rng):
    kind = rng.choice(["linear", "attend", "step", "evict"])
    if kind == "linear":
        while True:
            case = dict(kind=kind, tokens=_log(rng, 1, 4096), inputs=_log(rng, 256, 8192),
                        outputs=_log(rng, 256, 16384), type=rng.choice(["bf16", "f16"]), bias=rng.random() < 0.5)
            case["out"] = rng.choice([case["type"], case["type"], "f32"])
            if case["tokens"] * case["inputs"] * case["outputs"] <= 4096 * 8192 * 8192:
                return case
    dim = rng.choice([64, 128])
    case = dict(kind=kind, dim=dim, group=rng.choice([g for g in (32, 64, 128) if g <= dim]),
                page=rng.choice([32, 64, 128, 256]))
    if kind == "evict":
        case["kv_heads"] = rng.choice([1, 2, 4, 8])
        case["len_hi"] = _log(rng, 40, 65000)
        case["len_lo"] = rng.randint(max(1, case["len_hi"] // 4), case["len_hi"])
        case["keep"] = _log(rng, max(1, case["len_hi"] // 20), case["len_hi"])
        case["recent"] = rng.randint(0, case["keep"])
        case["seqs"] = _log(rng, 1, max(1, min(64, 12 * 8 * 65000 // (case["len_hi"] * case["kv_heads"]))))
        return case
    case["type"] = rng.choice(["bf16", "f16"])
    case["kv_heads"] = rng.choice([1, 2, 4, 8])
    case["heads"] = case["kv_heads"] * rng.choice([1, 2, 5, 7, 8])
    case["queries"] = rng.choice([1, 1, 1, _log(rng, 2, 8), _log(rng, 9, 300)])
    case["len_hi"] = max(case["queries"], _log(rng, 17, 200000 if case["queries"] <= 8 else 12000))
    case["len_lo"] = rng.randint(max(case["queries"], case["len_hi"] // 16), case["len_hi"])
    # the cache's tokens and heads of the longest listed case, the products of
    # the one with the most queries
    room = min(4 * 8 * 260000 // (case["len_hi"] * case["kv_heads"]),
               2 * 300 * 32 * 12000 // (case["len_hi"] * case["heads"] * case["queries"]) if case["queries"] > 8 else 64)
    case["seqs"] = _log(rng, 1, max(1, min(64, room)))
    if kind == "attend":
        case["weights"] = rng.random() < 0.4
    return case


def _lengths(case):
    """Tokens of each sequence's cache: ragged, the longest among them."""
    lo, hi = case["len_lo"], case["len_hi"]
    return [hi - int((hi - lo + 1) * ((0.618 * b) % 1.0)) if hi > lo else hi for b in range(case["seqs"])]


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if case["kind"] == "linear":
        t, k, n = case["tokens"], case["inputs"], case["outputs"]
        return {"bytes": t * k * size[case["type"]] + n * k + 4 * n * (2 if case["bias"] else 1)
                + t * n * size[case["out"]], "flops": 2 * t * k * n}
    total = sum(_lengths(case))
    token = case["dim"] + 8 * (case["dim"] // case["group"])  # K and V codes and scales of one token and head
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in _lengths(case))
        # the weights and positions of all tokens read; the kept ones' codes,
        # scales, weights and positions read and written
        return {"bytes": case["kv_heads"] * (8 * total + kept * (2 * token + 8)), "flops": case["kv_heads"] * total}
    b, t = case["seqs"], case["queries"]
    moved = total * case["kv_heads"] * token + 2 * b * t * case["heads"] * case["dim"] * 2
    if case["kind"] == "step":
        moved += b * t * case["kv_heads"] * (2 * case["dim"] * 2 + 2 * case["dim"] * 4)
    if case["kind"] == "step" or case["weights"]:
        moved += 8 * total * case["kv_heads"]
    pairs = sum(t * n - t * (t - 1) // 2 for n in _lengths(case))
    return {"bytes": moved, "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------- the cache's storage, in torch

# A word holds 8 codes of 4 bits; element e of the word is at nibble e/2 + 4 (e%2).
_NIBBLE = [4 * (e // 2 + 4 * (e % 2)) for e in range(8)]


def _words(codes):
    """int32 words of the codes [..., 8]."""
    shift = torch.tensor(_NIBBLE, dtype=torch.int32, device=codes.device)
    return (codes.to(torch.int32) << shift).sum(-1, dtype=torch.int32)


def _codes(words):
    """The codes [..., 8] of int32 words, as int8."""
    shift = torch.tensor(_NIBBLE, dtype=torch.int32, device=words.device)
    return ((words.unsqueeze(-1) >> shift) & 15).to(torch.int8)


def _pack_k(codes):
    """[pages, heads, page, dim] codes as K's words [pages, heads, page, 4, dim/32]."""
    n, h, p, d = codes.shape
    return _words(codes.view(n, h, p, d // 32, 4, 8).transpose(3, 4))


def _pack_v(codes):
    """[pages, heads, page, dim] codes as V's words [pages, heads, page/32, 4, 16, dim/16]."""
    n, h, p, d = codes.shape
    blocks = codes.view(n, h, p // 32, 2, 4, 4, d // 16, 16).permute(0, 1, 2, 4, 7, 6, 3, 5)
    return _words(blocks.reshape(n, h, p // 32, 4, 16, d // 16, 8))


def _unpack_k(words):
    n, h, p, _, i = words.shape
    return _codes(words).transpose(3, 4).reshape(n, h, p, 32 * i)


def _unpack_v(words):
    n, h, c, _, _, i = words.shape
    return _codes(words).view(n, h, c, 4, 16, i, 2, 4).permute(0, 1, 2, 6, 3, 7, 5, 4).reshape(n, h, 32 * c, 16 * i)


def _quantise(x, group):
    """Codes of x [..., dim] and the (scale, minimum) [..., dim/group, 2] of
    each group of channels, in 16 bits."""
    g = x.float().clamp(-65504.0, 65504.0).unflatten(-1, (-1, group))
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    base = low.half()
    scale = ((high - low) / 15.0).half()
    code = ((g - base.float()) / scale.float()).round().clamp(0, 15)
    code = torch.where(scale == 0, torch.zeros_like(code), code)
    return code.flatten(-2).to(torch.int8), torch.cat([scale, base], -1)


def _values(codes, par, group):
    """What codes [..., dim] with (scale, minimum) [..., dim/group, 2] stand for."""
    g = codes.unflatten(-1, (-1, group)).float()
    return (g * par[..., :1].float() + par[..., 1:].float()).flatten(-2)


# ----------------------------------------------------------------- the inputs

def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _pages(case, lengths, gen):
    """A table of shuffled pages that hold `lengths` tokens, and their number."""
    counts = [(n + case["page"] - 1) // case["page"] for n in lengths]
    total = sum(counts)
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((len(lengths), max(counts)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return table, total


def _cache(case, lengths, gen):
    """A cache whose tokens have keys and values with channels of unequal
    size, as models' keys have."""
    table, pages = _pages(case, lengths, gen)
    h, p, d = case["kv_heads"], case["page"], case["dim"]
    out = {"page_table": table}
    for name, pack in (("k", _pack_k), ("v", _pack_v)):
        channel = torch.exp(0.4 * _normal(gen, h, 1, d))
        x = _normal(gen, pages, h, p, d) * channel
        codes, par = _quantise(x, case["group"])
        del x
        out[name] = pack(codes)
        out[name + "_par"] = par.permute(0, 1, 3, 2, 4).contiguous()  # [pages, heads, groups, page, 2]
    # What earlier steps left: a few tokens hold most of the weight.
    out["acc"] = torch.exp(2.0 * _normal(gen, pages, h, p)) * 0.05
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] == "linear":
        t, k, n = case["tokens"], case["inputs"], case["outputs"]
        # Activations with a few large channels; weights as a per-channel
        # quantiser leaves them.
        x = _normal(gen, t, k) * torch.exp(0.7 * _normal(gen, 1, k))
        w = (_normal(gen, n, k) * 36.0).round().clamp(-127, 127).to(torch.int8)
        return {"case": case, "x": x.to(DTYPES[case["type"]]), "w": w,
                "packed": _pack_rows(w), "scale": torch.rand(n, device="cuda", generator=gen) * 2e-3 + 1e-4,
                "bias": _normal(gen, n) if case["bias"] else None}
    lengths = _lengths(case)
    if case["kind"] == "evict":
        state = {"case": case, "cache": _cache(case, lengths, gen)}
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        # Older tokens were evicted before: positions have gaps, in slot order.
        cap = state["cache"]["page_table"].shape[1] * case["page"]
        gaps = torch.randint(0, 3, (case["seqs"], case["kv_heads"], cap), device="cuda", generator=gen) // 2
        pos = torch.arange(cap, device="cuda") + gaps.cumsum(-1)
        last = pos.gather(-1, (state["lengths"].long() - 1).view(-1, 1, 1).expand(-1, case["kv_heads"], 1))
        total = last.amax((1, 2)) + 1
        pos = pos + (total.view(-1, 1, 1) - 1 - last)  # every head holds the newest token
        state["total"] = total.to(torch.int32)
        state["cache"]["pos"] = _to_pages(pos.to(torch.int32), state["cache"]["page_table"],
                                          state["cache"]["acc"].shape, case["page"])
        held = [min(n, case["keep"]) for n in lengths]
        table, pages = _pages(case, [max(held)] * len(held), gen)
        shape = lambda a: (pages,) + tuple(a.shape[1:])  # noqa: E731
        state["dst"] = {name: torch.zeros(shape(a), dtype=a.dtype, device="cuda")
                        for name, a in state["cache"].items() if name != "page_table"}
        state["dst"]["page_table"] = table
        return state
    b, t, d = case["seqs"], case["queries"], case["dim"]
    kind = DTYPES[case["type"]]
    state = {"case": case, "cache": _cache(case, lengths, gen),
             "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
             # Larger queries than unit ones: attention that picks tokens out.
             "q": (_normal(gen, b, t, case["heads"], d) * 1.5).to(kind)}
    state["cache"]["pos"] = torch.zeros_like(state["cache"]["acc"], dtype=torch.int32)
    state["acc_out"] = torch.zeros_like(state["cache"]["acc"])
    if case["kind"] == "step":
        state["start"] = state["lengths"] - t
        state["k"] = _normal(gen, b, t, case["kv_heads"], d).to(kind)
        state["v"] = _normal(gen, b, t, case["kv_heads"], d).to(kind)
    return state


def _pack_rows(w):
    """int8 [n, k] as the operands of matrix instructions: tiles of 16 rows by
    64 columns [n/16][k/64][4][16][16], both padded with zeros (k to 128)."""
    n, k = w.shape
    w = torch.nn.functional.pad(w, (0, -k % 128, 0, -n % 16))
    return w.view(w.shape[0] // 16, 16, w.shape[1] // 64, 4, 16).permute(0, 2, 3, 1, 4).contiguous()


def _to_pages(x, table, shape, page):
    """x [seqs, heads, slots] laid into a pool [pages, heads, page]."""
    out = torch.zeros(shape, dtype=x.dtype, device=x.device)
    blocks = x.unflatten(-1, (-1, page)).transpose(1, 2)  # [seqs, pages, heads, page]
    out[table[table >= 0].long()] = blocks[table >= 0]
    return out


# ------------------------------------------------------------ the plain forms

def _by_slot(pool, table):
    """A pool [pages, heads, page, ...] read through the table: [seqs, heads, slots, ...]."""
    x = pool[table.clamp(min=0).long()].transpose(1, 2)  # [seqs, heads, pages, page, ...]
    return x.flatten(2, 3)


def _plain_linear(s):
    x = s["x"].float()
    top = x.abs().amax(-1, keepdim=True)
    codes = torch.where(top > 0, (x * 127.0 / top).round(), torch.zeros_like(x))
    y = (codes @ s["w"].float().t()) * (top / 127.0) * s["scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[s["case"]["out"]])


def _plain_attend(s, step):
    case, cache, table = s["case"], s["cache"], s["cache"]["page_table"]
    b, t, hq, d = s["q"].shape
    h = case["kv_heads"]
    k, v = (_values(_by_slot(unpack(cache[n]), table), _by_slot(cache[n + "_par"].transpose(2, 3), table),
                    case["group"]) for n, unpack in (("k", _unpack_k), ("v", _unpack_v)))
    acc = _by_slot(cache["acc"], table)
    slots = k.shape[2]
    held = []
    if step:
        new = s["start"].long().view(b, 1, 1) + torch.arange(t, device=k.device).view(1, 1, t)
        at = new.expand(b, h, t)
        for_dims = at.unsqueeze(-1).expand(b, h, t, d)
        ks, vs = (_values(*_quantise(s[n], case["group"]), case["group"]) for n in ("k", "v"))
        held = [ks, vs]
        k = k.scatter(2, for_dims, ks.transpose(1, 2))
        v = v.scatter(2, for_dims, vs.transpose(1, 2))
        acc = acc.scatter(2, at, torch.zeros_like(acc[:, :, :t]))
    q = s["q"].float().view(b, t, h, hq // h, d).permute(0, 2, 3, 1, 4).reshape(b, h, hq // h * t, d)
    logits = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    first = s["lengths"].long().view(b, 1) - t + 1 + torch.arange(t, device=k.device)  # slots that query i sees
    seen = torch.arange(slots, device=k.device).view(1, 1, slots) < first.unsqueeze(-1)
    seen = seen.view(b, 1, 1, t, slots).expand(b, 1, hq // h, t, slots).reshape(b, 1, hq // h * t, slots)
    logits = torch.where(seen, logits, torch.full_like(logits, -math.inf))
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = p @ v
    o = o.view(b, h, hq // h, t, d).permute(0, 3, 1, 2, 4).reshape(b, t, hq, d).to(s["q"].dtype)
    if not step and not case["weights"]:
        return [o]
    valid = torch.arange(slots, device=k.device).view(1, 1, slots) < s["lengths"].view(b, 1, 1)
    acc = torch.where(valid, acc + p.sum(2), torch.zeros_like(acc))
    return [o, _to_pages(acc, table, cache["acc"].shape, case["page"])] + held


def _plain_evict(s):
    case, cache, dst = s["case"], s["cache"], s["dst"]
    src, to = cache["page_table"], dst["page_table"]
    acc, pos = _by_slot(cache["acc"], src), _by_slot(cache["pos"], src)
    b, h, slots = acc.shape
    valid = torch.arange(slots, device=acc.device) < s["lengths"].view(b, 1, 1)
    newest = pos >= (s["total"] - case["recent"]).view(b, 1, 1)
    key = torch.where(newest, torch.full_like(acc, math.inf), acc)
    key = torch.where(valid, key, torch.full_like(acc, -math.inf))
    room = to.shape[1] * case["page"]
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :min(case["keep"], slots)]
    count = s["lengths"].clamp(max=case["keep"])
    filled = torch.arange(order.shape[-1], device=acc.device) < count.view(b, 1, 1)
    order = torch.sort(torch.where(filled, order, torch.full_like(order, slots)), dim=-1).values
    order = torch.nn.functional.pad(order, (0, room - order.shape[-1]), value=slots)
    filled = order < slots
    order = order.clamp(max=slots - 1)

    def moved(x):
        """The kept tokens of x [seqs, heads, slots, ...], zeros behind them, in the destination's pages."""
        at, ok = order, filled
        if x.dim() == 4:
            at, ok = order.unsqueeze(-1).expand(b, h, room, x.shape[-1]), filled.unsqueeze(-1)
        y = torch.where(ok, x.gather(2, at), torch.zeros((), dtype=x.dtype, device=x.device))
        y = y.unflatten(2, (-1, case["page"])).transpose(1, 2)  # [seqs, pages, heads, page, ...]
        out = torch.zeros((dst["acc"].shape[0],) + tuple(y.shape[2:]), dtype=x.dtype, device=x.device)
        out[to[to >= 0].long()] = y[to >= 0]
        return out

    def scales(pool):
        x = moved(_by_slot(pool.transpose(2, 3), src).flatten(3))
        return x.unflatten(3, (-1, 2)).transpose(2, 3).contiguous()

    return {"k": _pack_k(moved(_by_slot(_unpack_k(cache["k"]), src))),
            "v": _pack_v(moved(_by_slot(_unpack_v(cache["v"]), src))),
            "k_par": scales(cache["k_par"]), "v_par": scales(cache["v_par"]),
            "pos": moved(pos), "acc": moved(acc), "lengths": count}


# ------------------------------------------------------------------- one pass

def _handle(ops, c):
    return ops.Cache(k=c["k"], v=c["v"], k_par=c["k_par"], v_par=c["v_par"], pos=c["pos"], acc=c["acc"],
                     page_table=c["page_table"])


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        if kind == "linear":
            return _plain_linear(state)
        return _plain_evict(state) if kind == "evict" else _plain_attend(state, kind == "step")
    from paper_2302_11665_amd import ops
    if kind == "linear":
        w = ops.PackedWeight(state["packed"], state["scale"], case["outputs"], case["inputs"])
        return ops.linear_i8(state["x"], w, bias=state["bias"], dtype=DTYPES[case["out"]])
    if kind == "evict":
        dst = state["dst"]
        count = ops.cache_evict(_handle(ops, state["cache"]), _handle(ops, dst), state["lengths"], state["total"],
                                keep=case["keep"], recent=case["recent"])
        return {"k": dst["k"], "v": dst["v"], "k_par": dst["k_par"], "v_par": dst["v_par"], "pos": dst["pos"],
                "acc": dst["acc"], "lengths": count}
    cache = _handle(ops, state["cache"])
    held = []
    if kind == "step":
        held = list(ops.cache_append(cache, state["k"], state["v"], state["start"], held=True))
    elif not case["weights"]:
        return [ops.attention_kv4(state["q"], cache, state["lengths"])]
    o = ops.attention_kv4(state["q"], cache, state["lengths"], acc_in=cache.acc, acc_out=state["acc_out"])
    return [o, state["acc_out"]] + held


# ------------------------------------------------- the definitions, in 64 bits

def exact(case, seed):
    if case["kind"] == "evict":
        return None  # whole numbers, and values that are moved
    s = prepare(case, seed)
    if case["kind"] == "linear":
        x = s["x"].double()
        top = x.abs().max(dim=1, keepdim=True).values
        codes = torch.round(127.0 * x / torch.where(top == 0, torch.ones_like(top), top))
        y = torch.mm(codes, s["w"].double().t().contiguous()) * (top / 127.0) * s["scale"].double()[None, :]
        return y if s["bias"] is None else y + s["bias"].double()
    cache, page, group, d = s["cache"], case["page"], case["group"], case["dim"]
    t, h, per = case["queries"], case["kv_heads"], case["heads"] // case["kv_heads"]
    step = case["kind"] == "step"
    dev = s["q"].device

    def held(new):
        """The new tokens' values [seqs, queries, heads, dim] as 4 bits hold them."""
        x = new.double().reshape(*new.shape[:-1], d // group, group)
        low, high = x.min(-1).values, x.max(-1).values
        base, scale = low.to(torch.float16).double(), ((high - low) / 15.0).to(torch.float16).double()
        code = torch.round((x - base[..., None]) / scale[..., None]).clamp(0, 15)
        return (code * scale[..., None] + base[..., None]).reshape(new.shape)

    # Where the dims of a K word, and the tokens and dims of a V word, are.
    nib = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=dev)
    out = torch.empty(case["seqs"], t, case["heads"], d, dtype=torch.float64, device=dev)
    acc = torch.zeros(cache["acc"].shape, dtype=torch.float64, device=dev)
    new_k, new_v = (held(s["k"]), held(s["v"])) if step else (None, None)
    for b, n in enumerate(_lengths(case)):
        pages = cache["page_table"][b, :(n + page - 1) // page].long()
        for j in range(h):
            kw, vw = cache["k"][pages, j].long(), cache["v"][pages, j].long()
            kc = (kw[..., None] >> nib) & 15  # [pages, page, 4, dim/32, 8]
            k = kc.permute(0, 1, 3, 2, 4).reshape(-1, d).double()
            vc = (vw[..., None] >> nib) & 15  # [pages, page/32, 4, 16, dim/16, 8]
            vc = vc.reshape(*vc.shape[:-1], 2, 4)  # tokens 16 a + 4 g + r
            v = vc.permute(0, 1, 5, 2, 6, 4, 3).reshape(-1, d).double()
            kp, vp = (cache[m][pages, j].double().transpose(0, 1).reshape(d // group, -1, 2) for m in ("k_par", "v_par"))
            for c in range(d // group):
                sl = slice(c * group, (c + 1) * group)
                k[:, sl] = k[:, sl] * kp[c, :, :1] + kp[c, :, 1:]
                v[:, sl] = v[:, sl] * vp[c, :, :1] + vp[c, :, 1:]
            k, v = k[:n], v[:n]
            was = cache["acc"][pages, j].reshape(-1)[:n].double()
            if step:
                k[n - t:], v[n - t:], was[n - t:] = new_k[b, :, j], new_v[b, :, j], 0.0
            weight = torch.zeros(n, dtype=torch.float64, device=dev)
            sees = torch.arange(n, device=dev)[None, :] <= (n - t + torch.arange(t, device=dev))[:, None]
            for g in range(per):
                a = torch.mm(s["q"][b, :, j * per + g].double(), k.t().contiguous()) / math.sqrt(d)
                p = torch.softmax(a.masked_fill(~sees, -math.inf), dim=-1)
                out[b, :, j * per + g] = torch.mm(p, v)
                weight += p.sum(0)
            full = torch.zeros(len(pages) * page, dtype=torch.float64, device=dev)
            full[:n] = was + weight
            acc[pages, j] = full.view(len(pages), page)
    if not step and not case["weights"]:
        return [out]
    return [out, acc] + ([new_k, new_v] if step else [])
