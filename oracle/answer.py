"""TEST INFRASTRUCTURE.  Answering, in 64 bits from its definitions: rows of a paged cache and their 8-bit form, attention of one new token over it, beam
search's selection and the reordering behind it.
"""
from __future__ import annotations

import math

import numpy as np


def e4m3_values():
    """The 256 values of e4m3 by their bytes: sign, 4 bits of exponent (bias 7), 3 of fraction; no infinity, NaN where all others are set."""
    out = np.empty(256)
    for b in range(256):
        e, f = b >> 3 & 15, b & 7
        x = np.nan if e == 15 and f == 7 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        out[b] = -x if b & 128 else x
    return out


E4M3 = e4m3_values()


def to_e4m3(x):
    """Bytes of the nearest values, halves to the even fraction; NaN and infinities as NaN.  |x| up to 448."""
    x = np.asarray(x, dtype=np.float64)
    size = E4M3[:127]                                                    # 0 .. 448, rising
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert (a <= 448).all()
    hi = np.clip(np.searchsorted(size, a), 1, 126)
    lo = hi - 1
    up, down = size[hi] - a, a - size[lo]
    b = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    b = np.where(np.isfinite(x), b, 127)
    return (b | np.where(np.signbit(x) & np.isfinite(x), 128, 0)).astype(np.uint8)


def quantise(rows):
    """(bytes, scale) of rows [.., d]."""
    rows = np.asarray(rows, dtype=np.float64)
    top = np.where(np.isfinite(rows), np.abs(rows), 0.0).max(-1)
    scale = np.ones_like(top)
    for i, t in np.ndenumerate(top):
        if t > 0:
            e = math.frexp(t / 448.0)[1]                                 # t / 448 = m 2^e, 1/2 <= m < 1
            if t <= 448.0 * 2.0 ** (e - 1):
                e -= 1
            scale[i] = 2.0 ** max(e, -126)
    return to_e4m3(rows / scale[..., None]), scale


def gather(pool, table, n, slots, slot_first):
    """The first n positions of a sequence, [n, heads, d] (or [n, heads]), from a pool [page, slot, heads, ..] or [page, heads, slot, ..]."""
    rows = []
    for m in range(n):
        p, s = table[m // slots], m % slots
        rows.append(pool[p, s] if slot_first else pool[p, :, s])
    return np.array(rows).reshape((n,) + (pool.shape[2:] if slot_first else (pool.shape[1],) + pool.shape[3:]))


def decode(q, k, v, scale):
    """One sequence: q [heads, group, d_k], k [n, heads, d_k], v [n, heads, d_v].  Returns o and sum_m p_m |v_m| [heads, group, d_v], logits [heads, group, n]."""
    H, G, _ = q.shape
    n = k.shape[0]
    o, size, logits = np.zeros((H, G, v.shape[-1])), np.zeros((H, G, v.shape[-1])), np.zeros((H, G, n))
    with np.errstate(invalid="ignore"):
        for h in range(H):
            for g in range(G):
                z = scale * (k[:, h] @ q[h, g])
                logits[h, g] = z
                if n == 0 or (z == -np.inf).all():
                    continue
                p = np.exp(z - z.max())
                p /= p.sum()
                o[h, g], size[h, g] = p @ v[:, h], p @ np.abs(v[:, h])
    return o, size, logits


def beam_select(logits, scores, finished, end_id, slots):
    """One sentence: logits [beams, vocab], scores [beams].  Returns parents, tokens, scores, finished of the best."""
    offers = []
    for i, z in enumerate(np.asarray(logits, dtype=np.float64)):
        if not np.isfinite(scores[i]):
            continue
        if finished is not None and finished[i]:
            offers.append((-scores[i], i, 0.0, end_id))
            continue
        top = z.max()
        if not np.isfinite(top):
            continue
        logp = (z - top) - np.log(np.exp(z - top).sum())
        order = np.lexsort((np.arange(len(z)), -z))[:slots]
        # (a beam's words are ordered by their logits, which a score far from 0 may leave nothing of in 64 bits of the sum)
        offers += [(-(scores[i] + logp[v]), i, -z[v], int(v)) for v in order if z[v] > -np.inf]
    offers.sort()
    got = [(i, v, -s, int(v == end_id or bool(finished is not None and finished[i]))) for s, i, _, v in offers[:slots]]
    got += [(0, end_id, -np.inf, 1)] * (slots - len(got))
    return tuple(np.array(x) for x in zip(*got))
