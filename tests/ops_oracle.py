"""Plain 64-bit definitions of the operators of a served model's step (numpy,
from the formulas; nothing of the package), and the storage of the 4-bit cache
written out element by element."""
from __future__ import annotations

import numpy as np


def quantise_rows(x):
    """Codes and scales of rows of float64 values; a row that is not finite has codes 0 and scale NaN."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(axis=1)
    fine = np.isfinite(top)
    safe = np.where(fine & (top > 0), top, 1.0)
    codes = np.where((fine & (top > 0))[:, None], np.rint(127.0 * np.where(fine[:, None], x, 0.0) / safe[:, None]), 0.0)
    return codes.astype(np.int64), np.where(fine, top / 127.0, np.nan)


def tile_index(rows, cols):
    """Byte of row r and column k in the tiles of a matrix of `cols` columns."""
    padded = -(-cols // 128) * 128
    r, k = np.arange(rows)[:, None], np.arange(cols)[None, :]
    return (r // 16) * (padded * 16) + (k // 64) * 1024 + (k // 16 % 4) * 256 + (r % 16) * 16 + k % 16


def nibble(e):
    return 4 * (e // 2 + 4 * (e % 2))


def read_cache(k, v, k_par, v_par, table_row, head, n, page, dim, group):
    """Codes (int) and (scale, minimum) of the first n slots of one sequence and
    head: kc, vc [n, dim], kp, vp [n, dim] pairs spread over the channels."""
    k, v = k.view(np.uint32), v.view(np.uint32)
    kc, vc = np.zeros((n, dim), np.int64), np.zeros((n, dim), np.int64)
    kp, vp = np.zeros((n, dim, 2)), np.zeros((n, dim, 2))
    ch = np.arange(dim)
    for s in range(n):
        p, at = int(table_row[s // page]), s % page
        w = k[p, head, at, ch // 8 % 4, ch // 32]
        kc[s] = w >> np.array([nibble(e) for e in ch % 8], np.uint32) & 15
        t = at % 32
        e = 4 * (t // 16) + t % 4
        w = v[p, head, at // 32, t // 4 % 4, ch % 16, ch // 16]
        vc[s] = w >> np.uint32(nibble(e)) & 15
        kp[s] = k_par[p, head, ch // group, at].astype(np.float64)
        vp[s] = v_par[p, head, ch // group, at].astype(np.float64)
    return kc, vc, kp, vp


def values(codes, par):
    return codes * par[..., 0] + par[..., 1]


def quantise_token(x, group):
    """Codes, scales and minima of x [..., dim] in float64; fp16 parameters."""
    x = np.clip(np.asarray(x, np.float64), -65504.0, 65504.0)
    g = x.reshape(*x.shape[:-1], -1, group)
    low, high = g.min(-1), g.max(-1)
    with np.errstate(invalid="ignore"):
        m = low.astype(np.float16)
        d = ((high - low) / 15.0).astype(np.float16)
        dd = np.where(d > 0, d, np.float16(1)).astype(np.float64)
        code = np.clip(np.rint((g - m.astype(np.float64)[..., None]) / dd[..., None]), 0, 15)
        code = np.where((d > 0)[..., None], code, 0)
    return np.nan_to_num(code).astype(np.int64).reshape(x.shape), d, m


def attend(q, k, v, seen, scale):
    """Softmax attention of q [rows, dim] over k, v [n, dim]; seen [rows, n].
    Rows that see nothing give 0.  Returns the outputs and the probabilities."""
    o, p = np.zeros((q.shape[0], v.shape[1])), np.zeros((q.shape[0], k.shape[0]))
    for r in range(q.shape[0]):
        idx = np.nonzero(seen[r])[0]
        if len(idx) == 0:
            continue
        a = (k[idx] @ q[r]) * scale
        w = np.exp(a - a.max())
        p[r, idx] = w / w.sum()
        o[r] = p[r, idx] @ v[idx]
    return o, p


def keep_slots(acc, pos, total, keep, recent):
    """Slots that stay, in slot order."""
    n = len(acc)
    if n <= keep:
        return np.arange(n)
    order = sorted(range(n), key=lambda s: ((0, 0.0) if pos[s] >= total - recent else
                                            (2, 0.0) if np.isnan(acc[s]) else (1, -float(acc[s])), s))
    return np.array(sorted(order[:keep]), np.int64)
