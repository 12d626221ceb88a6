"""Plain definitions of the operators that take prompts in (numpy, from the
formulas; nothing of the package)."""
from __future__ import annotations

import numpy as np


def norm_rows(h, gain, eps):
    """Codes, scales of rows h [rows, columns] (float64 values of 16 bits).  With
    a gain (fp32), h gain and 127 h gain are rounded to fp32 and the quotient too,
    as the operator states."""
    rms = np.sqrt((h * h).mean(1) + eps)
    with np.errstate(all="ignore"):
        t = h if gain is None else (h.astype(np.float32) * gain[None, :].astype(np.float32)).astype(np.float64)
        top = np.abs(t).max(1)
        fine = np.isfinite(top)
        safe = np.where(fine & (top > 0), top, 1.0)[:, None]
        if gain is None:
            q = 127.0 * np.where(fine[:, None], t, 0.0) / safe
        else:
            prod = np.where(fine[:, None], t, 0.0).astype(np.float32) * np.float32(127.0)
            q = (prod / safe.astype(np.float32)).astype(np.float32).astype(np.float64)
        scale = np.where(fine, np.where(top > 0, top / (127.0 * rms), 0.0), np.nan)
    return np.where((fine & (top > 0))[:, None], np.rint(q), 0.0).astype(np.int64), scale


def attend_causal(q, k, v, scale):
    """Of one head of one sequence: outputs, weights and logits in float64."""
    n = len(q)
    a = (q @ k.T) * scale
    seen = np.arange(n)[None, :] <= np.arange(n)[:, None]
    w = np.where(seen, np.exp(np.where(seen, a, 0.0) - np.where(seen, a, -np.inf).max(1, keepdims=True)), 0.0)
    p = w / w.sum(1, keepdims=True)
    return p @ v, p, np.where(seen, a, 0.0)


def reserve(stack, count, table, page, length, add, n_tokens):
    """Sequence by sequence; returns the new count, lengths, offsets, sequences
    and slots of the rows, and writes the table."""
    seqs, max_pages = table.shape
    length, free = [min(max(int(n), 0), max_pages * page) for n in length], min(max(int(count), 0), len(stack))
    new, seq, slot, offsets = list(length), [-1] * n_tokens, [-1] * n_tokens, [0]
    needed = taken = at = 0
    for b in range(seqs):
        more, n = max(int(add[b]), 0), length[b]
        have, need = -(-n // page), 0
        granted = more == 0 or (n + more <= max_pages * page and at + more <= n_tokens)
        if more and granted:
            need = -(-(n + more) // page) - have
            needed += need
            granted = need == 0 or needed <= free
        if more and granted:
            for i in range(need):
                table[b, have + i] = stack[free - 1 - (needed - need + i)]
            taken = max(taken, needed if need else 0)
            new[b] = n + more
            for i in range(more):
                seq[at + i], slot[at + i] = b, n + i
        at += more
        offsets.append(min(at, n_tokens))
    return free - taken, new, offsets, seq, slot


def release(stack, count, table, page, length, which):
    """Returns the new count and lengths, and writes the stack."""
    count, new = int(count), list(length)
    for b in np.nonzero(which)[0]:
        for i in range(-(-int(length[b]) // page)):
            stack[count] = table[b, i]
            count += 1
        new[b] = 0
    return count, new
