"""The operators that take prompts into a served model, as cases to be timed.

A request's cost begins with its prompt.  A model's block reads the prompts of
several requests at once, packed one after the other, and leaves their keys and
values in a paged cache of 4 bits:
  norm     a residual added, the rows brought to mean square 1, times a gain,
           and held in 8 bits with a scale per token
  project  the same, then a linear layer with 8-bit weights from these codes
  prompt   causal attention of every token over its own prompt, query heads
           in groups that share a key/value head
  pages    a step's bookkeeping: pages of requests that ended go back to the
           pool, new tokens get pages, and every packed token its sequence and
           slot
  append   packed tokens, of prompts and of single steps, put into the cache

Where `own` is false the plain forms run: elementary torch operations in 32
bits.  Where it is true the package's operators run.  Both read the same state.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # One token of one request before a projection: the smallest call of a
        # step, where launches count.
        dict(name="norm_token", kind="norm", tokens=1, cols=4096, type="bf16", residual=True, gain=True),
        # Long prompts of a wide model: bytes count.
        dict(name="norm_prompts", kind="norm", tokens=8192, cols=8192, type="f16", residual=True, gain=False),
        # A batch of requests' tokens into a block's first projection.
        dict(name="project_batch", kind="project", tokens=24, cols=4096, outputs=6144, type="bf16", out="bf16",
             residual=True, gain=True),
        # Sizes that fit no tile, 32-bit results (a last projection).
        dict(name="project_odd", kind="project", tokens=777, cols=1500, outputs=2777, type="f16", out="f32",
             residual=False, gain=True),
        # One short prompt of a small model: latency.
        dict(name="prompt_short", kind="prompt", seqs=1, len_lo=33, len_hi=33, heads=8, kv_heads=2, dim=64,
             type="bf16"),
        # Prompts of very unequal lengths, small heads in groups of three.
        dict(name="prompt_ragged", kind="prompt", seqs=29, len_lo=1, len_hi=2500, heads=24, kv_heads=8, dim=64,
             type="f16"),
        # A batch of ordinary prompts.
        dict(name="prompt_batch", kind="prompt", seqs=8, len_lo=1000, len_hi=4099, heads=32, kv_heads=8, dim=128,
             type="bf16"),
        # One long prompt: the matrix rate counts.
        dict(name="prompt_long", kind="prompt", seqs=1, len_lo=12001, len_hi=12001, heads=32, kv_heads=4, dim=128,
             type="bf16"),
        # A step of a few requests, one token each: latency.
        dict(name="pages_step", kind="pages", seqs=48, add_hi=1, held_hi=2000, page=64, part=0.9, ended=0.1, short=0),
        # Many prompts let in at once while others run on; the pool does not
        # last for all of them.
        dict(name="pages_prompts", kind="pages", seqs=2000, add_hi=700, held_hi=9000, page=64, part=0.3, ended=0.05,
             short=100),
        # Two prompts read beside the single tokens of running requests.
        dict(name="append_mixed", kind="append", seqs=40, prompts=2, len_lo=100, len_hi=900, held_hi=3000, kv_heads=8,
             dim=128, group=64, page=64, type="bf16"),
        # Long prompts of small models' heads, few channels to a scale.
        dict(name="append_prompts", kind="append", seqs=12, prompts=12, len_lo=1500, len_hi=9000, held_hi=0,
             kv_heads=8, dim=64, group=32, page=128, type="f16"),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "project", "prompt", "prompt", "pages", "append"])
    case = dict(kind=kind)
    if kind in ("norm", "project"):
        case.update(type=rng.choice(["bf16", "f16"]), residual=rng.random() < 0.6, gain=rng.random() < 0.7,
                    cols=_log(rng, 64, 16384))
        if kind == "norm":
            case["tokens"] = _log(rng, 1, max(1, min(16384, 8192 * 8192 // case["cols"])))
            return case
        case.update(tokens=_log(rng, 1, 4096), outputs=_log(rng, 64, 8192), out=rng.choice([case["type"], "f32"]))
        return case
    if kind == "pages":
        case.update(seqs=_log(rng, 2, 2000), add_hi=_log(rng, 1, 700), held_hi=_log(rng, 1, 9000),
                    page=rng.choice([32, 64, 96, 128, 256]), part=round(rng.uniform(0.1, 1.0), 3),
                    ended=round(rng.uniform(0.0, 0.4), 3), short=rng.choice([0, 0, _log(rng, 1, 100)]))
        return case
    case.update(kv_heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128]), type=rng.choice(["bf16", "f16"]))
    if kind == "prompt":
        case["heads"] = case["kv_heads"] * rng.choice([1, 2, 3, 4, 5, 7, 8])
        case["len_hi"] = _log(rng, 1, 12000)
        case["len_lo"] = rng.randint(1, case["len_hi"])
        # (the plain form computes all sequences at the longest one's length)
        room = 32 * 12001 ** 2 // (case["len_hi"] ** 2 * case["heads"])
        case["seqs"] = _log(rng, 1, max(1, min(64, room)))
        return case
    case.update(group=rng.choice([g for g in (32, 64, 128) if g <= case["dim"]]), page=rng.choice([32, 64, 128, 256]),
                len_hi=_log(rng, 1, 9000), held_hi=_log(rng, 1, 4000))
    case["len_lo"] = rng.randint(1, case["len_hi"])
    case["prompts"] = _log(rng, 1, max(1, min(64, 12 * 9000 // case["len_hi"])))
    case["seqs"] = case["prompts"] + rng.choice([0, _log(rng, 1, 64)])
    return case


def _between(lo, hi, i):
    """The i-th of a ragged run of whole numbers of [lo, hi], the largest among them."""
    return hi - int((hi - lo + 1) * ((0.618 * i) % 1.0)) if hi > lo else hi


def _lengths(case):
    """Tokens of each packed sequence: prompts, then single tokens."""
    prompts = [_between(case["len_lo"], case["len_hi"], b) for b in range(case.get("prompts", case["seqs"]))]
    return prompts + [1] * (case["seqs"] - len(prompts))


def _held(case):
    """Tokens that each sequence's cache holds already: none before a prompt."""
    return [0 if b < case["prompts"] else _between(1, max(1, case["held_hi"]), b) for b in range(case["seqs"])]


def _turn(case):
    """Of each sequence of a step's bookkeeping: tokens held, tokens to add, whether it ended.  Those that ended get
    nothing in the same step; a prompt begins an empty sequence."""
    held, add, ended = [], [], []
    for b in range(case["seqs"]):
        u = (0.7548776662 * (b + 1)) % 1.0
        prompt = case["add_hi"] > 1 and (0.5698402909 * (b + 1)) % 1.0 < 0.5
        gone = u >= 1.0 - case["ended"]
        held.append(0 if prompt and not gone else _between(1, case["held_hi"], b))
        ended.append(gone)
        add.append(0 if gone or u >= case["part"] else _between(1, case["add_hi"], b + 3) if prompt else 1)
    return held, add, ended


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    kind = case["kind"]
    if kind in ("norm", "project"):
        t, k = case["tokens"], case["cols"]
        moved = t * k * 2 * (3 if case["residual"] else 1) + (4 * k if case["gain"] else 0)
        if kind == "norm":  # the values that the 8 bits stand for, and their scales
            return {"bytes": moved + t * k * 4 + 4 * t, "flops": 6 * t * k}
        n = case["outputs"]
        return {"bytes": moved + n * k + 4 * n + t * n * size[case["out"]], "flops": 2 * t * k * n}
    if kind == "prompt":
        tokens = sum(_lengths(case))
        pairs = sum(n * (n + 1) // 2 for n in _lengths(case))
        return {"bytes": 2 * 2 * tokens * (case["heads"] + case["kv_heads"]) * case["dim"],
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    if kind == "pages":
        held, add, ended = _turn(case)
        back = sum(-(-n // case["page"]) for n, e in zip(held, ended) if e)
        new = sum(-(-(n + a) // case["page"]) - -(-n // case["page"]) for n, a in zip(held, add))
        return {"bytes": case["seqs"] * (8 + 1 + 4 + 4) + sum(add) * 8 + 8 * (back + new), "flops": sum(add)}
    tokens, d = sum(_lengths(case)), case["dim"]
    token = d + 8 * (d // case["group"])  # K and V codes and scales of one token and head
    return {"bytes": tokens * case["kv_heads"] * (2 * d * 2 + token + 8 + 2 * d * 4) + 8 * tokens,
            "flops": 8 * tokens * case["kv_heads"] * d}


# ----------------------------------------------------------------- the inputs

def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pack_rows(w):
    """int8 [n, k] as the operands of matrix instructions: tiles of 16 rows by
    64 columns [n/16][k/64][4][16][16], both padded with zeros (k to 128)."""
    n, k = w.shape
    w = torch.nn.functional.pad(w, (0, -k % 128, 0, -n % 16))
    return w.view(w.shape[0] // 16, 16, w.shape[1] // 64, 4, 16).permute(0, 2, 3, 1, 4).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    state = {"case": case}
    if kind in ("norm", "project"):
        t, k, type_ = case["tokens"], case["cols"], DTYPES[case["type"]]
        # Activations with a few large channels, as models' residual streams have.
        channel = torch.exp(0.7 * _normal(gen, 1, k))
        state["x"] = (_normal(gen, t, k) * channel).to(type_)
        state["residual"] = (_normal(gen, t, k) * channel * 3.0).to(type_) if case["residual"] else None
        state["gain"] = 1.0 + 0.3 * _normal(gen, k) if case["gain"] else None
        if kind == "project":
            n = case["outputs"]
            state["w"] = (_normal(gen, n, k) * 36.0).round().clamp(-127, 127).to(torch.int8)
            state["packed"] = _pack_rows(state["w"])
            state["scale"] = torch.rand(n, device="cuda", generator=gen) * 2e-3 + 1e-4
        return state
    if kind == "prompt":
        type_, lengths = DTYPES[case["type"]], _lengths(case)
        t, h, hk, d = sum(lengths), case["heads"], case["kv_heads"], case["dim"]
        # One projection's output holds queries, keys and values side by side;
        # larger queries than unit ones: attention that picks tokens out.
        qkv = _normal(gen, t, h + 2 * hk, d)
        qkv[:, :h] *= 1.5
        state["qkv"] = qkv.to(type_)
        state["offsets"] = _ints([0] + torch.tensor(lengths).cumsum(0).tolist())
        return state
    if kind == "pages":
        held, add, ended = _turn(case)
        page = case["page"]
        counts = [-(-n // page) for n in held]
        back = sum(c for c, e in zip(counts, ended) if e)
        want = sum(-(-(n + a) // page) - c for n, a, c in zip(held, add, counts))
        free = max(0, want - back - case["short"]) if case["short"] else want + 5
        pages = sum(counts) + free
        order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
        table = torch.full((case["seqs"], -(-(case["held_hi"] + case["add_hi"]) // page)), -1, dtype=torch.int32,
                           device="cuda")
        at = torch.tensor(counts, device="cuda").view(-1, 1)
        inside = torch.arange(table.shape[1], device="cuda") < at
        table[inside] = order[:sum(counts)]
        stack = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        stack[:free] = order[sum(counts):]
        state.update(table=table, stack=stack, count=_ints([free]), held=_ints(held), add=_ints(add),
                     ended=torch.tensor(ended, device="cuda"), tokens=sum(add),
                     released=torch.zeros(case["seqs"], dtype=torch.int32, device="cuda"),
                     after=torch.zeros(case["seqs"], dtype=torch.int32, device="cuda"), left=_ints([0, 0]))
        return state
    type_, lengths, held, page = DTYPES[case["type"]], _lengths(case), _held(case), case["page"]
    t, h, d, group = sum(lengths), case["kv_heads"], case["dim"], case["group"]
    counts = [-(-(n + a) // page) for n, a in zip(held, lengths)]
    pages = sum(counts)
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.full((case["seqs"], max(counts)), -1, dtype=torch.int32, device="cuda")
    inside = torch.arange(max(counts), device="cuda") < torch.tensor(counts, device="cuda").view(-1, 1)
    table[inside] = order
    words = lambda *shape: torch.randint(-2 ** 31, 2 ** 31 - 1, shape, dtype=torch.int32, device="cuda", generator=gen)  # noqa: E731
    par = (pages, h, d // group, page, 2)
    state["cache"] = {"k": words(pages, h, page, 4, d // 32), "v": words(pages, h, page // 32, 4, 16, d // 16),
                      "k_par": _normal(gen, *par).half(), "v_par": _normal(gen, *par).half(),
                      "pos": torch.zeros((pages, h, page), dtype=torch.int32, device="cuda"),
                      "acc": torch.rand((pages, h, page), device="cuda", generator=gen), "page_table": table}
    n, first = torch.tensor(lengths, device="cuda"), torch.tensor(held, device="cuda")
    state["seq"] = torch.arange(case["seqs"], device="cuda").repeat_interleave(n).to(torch.int32)
    within = torch.arange(t, device="cuda") - (n.cumsum(0) - n).repeat_interleave(n)
    state["slot"] = (first.repeat_interleave(n) + within).to(torch.int32)
    # Keys' channels are of unequal size; both come from one projection's output.
    both = _normal(gen, t, 2 * h, d) * torch.exp(0.4 * _normal(gen, 1, 2 * h, d))
    state["kv"] = both.to(type_)
    return state


# ------------------------------------------------------------ the plain forms

def _plain_norm(s):
    """The sum in its type, codes and scales of its normed rows, as fp32."""
    x, type_ = s["x"], s["x"].dtype
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(type_)
    f = h.float()
    t = f if s["gain"] is None else f * s["gain"]
    top = t.abs().amax(-1, keepdim=True)
    codes = torch.where(top > 0, (t * 127.0 / top).round(), torch.zeros_like(t))
    root = (f.square().mean(-1, keepdim=True) + EPS).sqrt()
    return h, codes, top / (root * 127.0)


def _plain_project(s):
    h, codes, scale = _plain_norm(s)
    y = (codes @ s["w"].float().t()) * scale * s["scale"]
    y = y.to(DTYPES[s["case"]["out"]])
    return [y] if s["residual"] is None else [h, y]


def _plain_prompt(s):
    case, qkv = s["case"], s["qkv"]
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    begin, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    longest = case["len_hi"]
    at = torch.arange(longest, device=qkv.device)
    there = at < (end - begin).view(-1, 1)
    rows = torch.where(there, begin.view(-1, 1) + at, torch.zeros_like(at))
    padded = qkv[rows].float().transpose(1, 2)  # [seqs, heads, tokens, dim]
    q = padded[:, :h].reshape(-1, hk, h // hk * longest, d)
    k, v = padded[:, h:h + hk], padded[:, h + hk:]
    logits = (q @ k.transpose(-1, -2)).view(-1, h, longest, longest)
    logits *= 1.0 / math.sqrt(d)
    logits.masked_fill_(at.view(1, -1) > at.view(-1, 1), -math.inf)
    logits -= logits.amax(-1, keepdim=True)
    p = torch.exp(logits)
    del logits
    p /= p.sum(-1, keepdim=True)
    o = (p.view(-1, hk, h // hk * longest, longest) @ v).view(-1, h, longest, d)
    out = torch.empty(qkv.shape[0], h, d, dtype=qkv.dtype, device=qkv.device)
    out[rows[there]] = o.transpose(1, 2)[there].to(qkv.dtype)
    return out


def _plain_pages(s):
    page, table, stack = s["case"]["page"], s["table"], s["stack"]
    column = torch.arange(table.shape[1], device=table.device)
    count = s["count"].long()
    # pages of those that ended, in order, behind the free ones
    gone = torch.where(s["ended"], (s["held"] + page - 1) // page, torch.zeros_like(s["held"])).long()
    to = count + (gone.cumsum(0) - gone).view(-1, 1) + column
    inside = column < gone.view(-1, 1)
    stack[to[inside]] = table[inside]
    count = count + gone.sum()
    held = torch.where(s["ended"], torch.zeros_like(s["held"]), s["held"]).long()
    # pages for the new tokens, in order, from the last free one on
    add = s["add"].long()
    have = (held + page - 1) // page
    need = torch.where(add > 0, (held + add + page - 1) // page - have, torch.zeros_like(have))
    upto = need.cumsum(0)
    fits = (need == 0) | (upto <= count)
    take = torch.where(fits, need, torch.zeros_like(need))
    inside = (column >= have.view(-1, 1)) & (column < (have + take).view(-1, 1))
    which = count - 1 - ((upto - need).view(-1, 1) + column - have.view(-1, 1))
    table[inside] = stack[which[inside]]
    count = count - take.sum()
    offsets = torch.nn.functional.pad(add.cumsum(0), (1, 0))
    order = torch.arange(add.shape[0], device=table.device).repeat_interleave(add, output_size=s["tokens"])
    slot = held[order] + torch.arange(s["tokens"], device=table.device) - offsets[order]
    seq = torch.where(fits[order], order, torch.full_like(order, -1))
    slot = torch.where(fits[order], slot, torch.full_like(slot, -1))
    length = held + torch.where(fits, add, torch.zeros_like(add))
    small = lambda x: x.to(torch.int32)  # noqa: E731
    return {"table": table, "stack": stack, "count": small(count), "length": small(length), "offsets": small(offsets),
            "seq": small(seq), "slot": small(slot)}


# A word of the cache holds 8 codes of 4 bits; element e of the word is at nibble e/2 + 4 (e%2).
_NIBBLE = [4 * (e // 2 + 4 * (e % 2)) for e in range(8)]


def _quantise(x, group):
    """Codes of x [..., dim] and the (scale, minimum) [..., dim/group, 2] of
    each group of channels, in 16 bits."""
    g = x.float().clamp(-65504.0, 65504.0).unflatten(-1, (-1, group))
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    base = low.half()
    scale = ((high - low) / 15.0).half()
    code = ((g - base.float()) / scale.float()).round().clamp(0, 15)
    code = torch.where(scale == 0, torch.zeros_like(code), code)
    return code.flatten(-2).to(torch.int32), torch.cat([scale, base], -1)


def _plain_append(s):
    case, cache = s["case"], s["cache"]
    h, d, group, page = case["kv_heads"], case["dim"], case["group"], case["page"]
    shift = torch.tensor(_NIBBLE, dtype=torch.int32, device="cuda")
    slot = s["slot"].long()
    at, place = cache["page_table"][s["seq"].long(), slot // page].long(), slot % page
    kc, kp = _quantise(s["kv"][:, :h], group)
    vc, vp = _quantise(s["kv"][:, h:], group)
    cache["k"][at, :, place] = (kc.view(-1, h, d // 32, 4, 8).transpose(2, 3) << shift).sum(-1, dtype=torch.int32)
    cache["k_par"][at, :, :, place] = kp
    cache["v_par"][at, :, :, place] = vp
    cache["pos"][at, :, place] = s["slot"].view(-1, 1)
    cache["acc"][at, :, place] = 0.0
    # V's words hold 8 tokens of one channel: the new tokens' bits of them
    block, inside = place // 32, place % 32
    bits = shift[4 * (inside // 16) + inside % 4].view(-1, 1, 1)
    head = torch.arange(h, device="cuda").view(1, h)
    index = (at.view(-1, 1), head, block.view(-1, 1), (inside // 4 % 4).view(-1, 1))
    codes = vc.view(-1, h, d // 16, 16).transpose(2, 3)  # [tokens, heads, 16, dim/16]
    word = torch.zeros_like(cache["v"])
    word.index_put_(index, codes << bits.view(-1, 1, 1, 1), accumulate=True)
    mask = torch.zeros_like(cache["v"])
    mask.index_put_(index, (15 << bits.view(-1, 1, 1, 1)).expand_as(codes), accumulate=True)
    cache["v"].bitwise_and_(~mask).bitwise_or_(word)

    def values(codes, par):
        g = codes.unflatten(-1, (-1, group)).float()
        return (g * par[..., :1].float() + par[..., 1:].float()).flatten(-2)

    return {"k": values(kc, kp), "v": values(vc, vp), "pos": cache["pos"], "acc": cache["acc"]}


# ------------------------------------------------------------------- one pass

def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        if kind == "norm":
            h, codes, scale = _plain_norm(state)
            return [scale, codes * scale] if state["residual"] is None else [scale, codes * scale, h]
        if kind == "project":
            return _plain_project(state)
        return {"prompt": _plain_prompt, "pages": _plain_pages, "append": _plain_append}[kind](state)
    from paper_2302_11665_amd import ops
    if kind == "norm":
        codes, h, held = ops.norm_i8(state["x"], state["residual"], state["gain"], eps=EPS, held=True)
        scale = codes.scale.view(-1, 1)
        return [scale, held] if state["residual"] is None else [scale, held, h]
    if kind == "project":
        codes, h = ops.norm_i8(state["x"], state["residual"], state["gain"], eps=EPS)
        w = ops.PackedWeight(state["packed"], state["scale"], case["outputs"], case["cols"])
        y = ops.linear_i8(codes, w, dtype=DTYPES[case["out"]])
        return [y] if state["residual"] is None else [h, y]
    if kind == "prompt":
        h, hk = case["heads"], case["kv_heads"]
        qkv = state["qkv"]
        return ops.attention_prompt(qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:], state["offsets"])
    if kind == "pages":
        pool = ops.PagePool(state["stack"], state["count"])
        left = state["left"]
        ops.pages_release(pool, state["table"], case["page"], state["held"], state["ended"],
                          new_length=state["released"], new_count=left[:1])
        pool = ops.PagePool(state["stack"], left[:1])
        plan = ops.pages_reserve(pool, state["table"], case["page"], state["released"], state["add"], state["tokens"],
                                 new_length=state["after"], new_count=left[1:])
        return {"table": state["table"], "stack": state["stack"], "count": left[1:], "length": state["after"],
                "offsets": plan.offsets, "seq": plan.seq, "slot": plan.slot}
    c, h = state["cache"], case["kv_heads"]
    cache = ops.Cache(k=c["k"], v=c["v"], k_par=c["k_par"], v_par=c["v_par"], pos=c["pos"], acc=c["acc"],
                      page_table=c["page_table"])
    k, v = ops.cache_append_packed(cache, state["kv"][:, :h], state["kv"][:, h:], state["seq"], state["slot"],
                                   held=True)
    return {"k": k, "v": v, "pos": c["pos"], "acc": c["acc"]}


# ------------------------------------------------- the definitions, in 64 bits

def exact(case, seed):
    kind = case["kind"]
    if kind == "pages":
        return None  # whole numbers
    s = prepare(case, seed)
    if kind in ("norm", "project"):
        x = s["x"].double()
        if s["residual"] is not None:  # the sum is kept in its type, and the norm is that of what is kept
            x = (x + s["residual"].double()).to(s["x"].dtype).double()
        t = x if s["gain"] is None else x * s["gain"].double()[None, :]
        largest = t.abs().max(dim=1, keepdim=True).values
        codes = torch.round(127.0 * t / torch.where(largest == 0, torch.ones_like(largest), largest))
        scale = largest / 127.0 / torch.sqrt((x * x).sum(1, keepdim=True) / x.shape[1] + EPS)
        if kind == "norm":
            return [scale, codes * scale] + ([] if s["residual"] is None else [x])
        y = torch.mm(codes, s["w"].double().t().contiguous()) * scale * s["scale"].double()[None, :]
        return [y] if s["residual"] is None else [x, y]
    if kind == "prompt":
        h, hk, d = case["heads"], case["kv_heads"], case["dim"]
        if case["seqs"] * h > 2000:
            return None
        out = torch.empty(s["qkv"].shape[0], h, d, dtype=torch.float64, device="cuda")
        at = 0
        for n in _lengths(case):
            x = s["qkv"][at:at + n].double()
            future = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
            for j in range(h):
                g = j // (h // hk)
                a = torch.mm(x[:, j].contiguous(), x[:, h + g].t().contiguous()) / math.sqrt(d)
                p = torch.softmax(a.masked_fill_(future, -math.inf), dim=-1)
                out[at:at + n, j] = torch.mm(p, x[:, h + hk + g].contiguous())
            at += n
        return out
    h, d, group = case["kv_heads"], case["dim"], case["group"]

    def held(x):
        """The values as 4 bits hold them."""
        g = x.double().reshape(x.shape[0], h, d // group, group)
        low, high = g.min(-1).values, g.max(-1).values
        base, scale = low.to(torch.float16).double(), ((high - low) / 15.0).to(torch.float16).double()
        code = torch.round((g - base[..., None]) / torch.where(scale == 0, torch.ones_like(scale), scale)[..., None])
        code = torch.where((scale == 0)[..., None], torch.zeros_like(code), code.clamp(0, 15))
        return (code * scale[..., None] + base[..., None]).reshape(x.shape)

    return {"k": held(s["kv"][:, :h]), "v": held(s["kv"][:, h:]), "pos": None, "acc": None}
