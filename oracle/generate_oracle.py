"""Plain statements, in numpy and 64 bits, of what a program that generates text does around the attention: rotary position
embedding, attention of chunks of several sequences, the selection of a beam search step, and the sequences that follow it.
Test infrastructure; shares no code with the product."""
from __future__ import annotations

import numpy as np


def rotate(x, pos, freqs, rotary_dim=128, interleaved=False, scale=1.0):
    """x [T, heads, 128], pos [T] -> the rotated rows; also the sum of magnitudes |a| + |b| of every channel's pair (0 where a channel
    passes through)."""
    y = np.asarray(x, np.float64).copy()
    mag = np.zeros_like(y)
    half = rotary_dim // 2
    for t, p in enumerate(pos):
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            # the angle, reduced in extended precision
            th = float(np.fmod(np.longdouble(int(p)) * np.longdouble(freqs[i]), 2 * np.longdouble(np.pi) + np.longdouble(2.4492935982947064e-16)))
            c, s = scale * np.cos(th), scale * np.sin(th)
            xa, xb = y[t, :, a].copy(), y[t, :, b].copy()
            y[t, :, a], y[t, :, b] = xa * c - xb * s, xb * c + xa * s
            mag[t, :, a] = mag[t, :, b] = np.abs(xa) + np.abs(xb)
    return y, mag


def attend(q, k, v, positions, sm_scale, window=0, n_sink=0):
    """Rows q [R, 128] at the given positions over keys k, v [n, 128] of their sequence: the keys n <= position, or with a window those
    that are sinks or among the newest `window`.  Returns (out [R, 128], lse [R], mass-weighted magnitude sum p |v| [R, 128]); a row
    that sees nothing: 0, -inf, 0."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    out, lse, mag = np.zeros((len(q), k.shape[-1])), np.full(len(q), -np.inf), np.zeros((len(q), k.shape[-1]))
    for i, m in enumerate(positions):
        n = np.arange(min(m + 1, len(k)))
        if window:
            n = n[(n < n_sink) | (n > m - window)]
        if len(n) == 0:
            continue
        z = k[n] @ q[i] * sm_scale
        top = z.max()
        p = np.exp(z - top)
        total = p.sum()
        out[i], lse[i], mag[i] = p @ v[n] / total, top + np.log(total), p @ np.abs(v[n]) / total
    return out, lse, mag


def beam_select(logits, scores, finished, n_beams, k, pad_token=0):
    """Per group the k best continuations as lists of (score, row, token); fewer where there are no more."""
    logits = np.asarray(logits, np.float64)
    picked = []
    for g in range(len(logits) // n_beams):
        cands = []
        for row in range(g * n_beams, (g + 1) * n_beams):
            base = 0.0 if scores is None else float(scores[row])
            if finished is not None and finished[row]:
                cands.append((-base, row, pad_token))
                continue
            x = logits[row]
            top = x.max()
            # (the maximum taken off first: in the sum with a normaliser of 3e38, 64 bits would lose the rest)
            s = base + ((x - top) - np.log(np.exp(x - top).sum())) if np.isfinite(top) else np.full(len(x), -np.inf)
            order = np.argsort(-s, kind="stable")[:k]
            cands += [(-s[t], row, int(t)) for t in order]
        cands.sort()
        picked.append([(-s, row, t) for s, row, t in cands[:k]])
    return picked


def reorder(table, lens, refs, src, dst):
    """The table, lengths and counts afterwards, and whether a request was refused."""
    table, lens, refs = np.array(table), np.array(lens), np.array(refs)
    before_t, before_l = table.copy(), lens.copy()
    seen, bad = set(), False
    for s, d in zip(src, dst):
        if d in seen or not 0 <= d < len(table) or not 0 <= s < len(table):
            bad = True
            if 0 <= d < len(table):
                seen.add(d)
            continue
        seen.add(d)
        for e in before_t[d]:
            if 0 <= e < len(refs):
                refs[e] -= 1
        for e in before_t[s]:
            if 0 <= e < len(refs):
                refs[e] += 1
            bad = bad or e >= len(refs)
        table[d], lens[d] = before_t[s], before_l[s]
    return table, lens, refs, bad
