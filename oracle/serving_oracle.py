"""fp64 numpy statements of the batched decoding calls (exactmoe_serving.h):
the paged append with rotary positions, the attention of one new token per row
over a paged cache, and the processing of logits.  Test infrastructure only;
plain loops over tokens, rows and keys, shared with nothing."""
from __future__ import annotations

import numpy as np


def rotate(x, position, inv_freq, interleaved):
    """One head vector turned by its position's angles."""
    y = np.array(x, np.float64)
    half = len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = np.cos(position * inv_freq[i]), np.sin(position * inv_freq[i])
        y[a], y[b] = x[a] * c - x[b] * s, x[a] * s + x[b] * c
    return y


def slot_of(table, n_pages, page_size, seq, position):
    """(page, slot) of a position, None where there is none."""
    if not 0 <= seq < len(table) or position < 0 or position // page_size >= len(table[seq]):
        return None
    page = int(table[seq][position // page_size])
    return (page, position % page_size) if 0 <= page < n_pages else None


def append(q, k, v, positions, seqs, table, n_pages, page_size, inv_freq, interleaved):
    """(rotated q or None per token, {(page, slot): (rotated k, v)}), before any rounding."""
    q_out, stored = [], {}
    for t, p in enumerate(positions):
        s = int(seqs[t])
        if p < 0 or not 0 <= s < len(table):
            q_out.append(None)
            continue
        q_out.append(np.stack([rotate(h, p, inv_freq, interleaved) for h in q[t]]))
        at = slot_of(table, n_pages, page_size, s, int(p))
        if at is not None:
            stored[at] = (np.stack([rotate(h, p, inv_freq, interleaved) for h in k[t]]),
                          np.array(v[t], np.float64))
    return q_out, stored


def visible(table, n_pages, page_size, seq, length, max_keys, window):
    """The (page, slot) of every key that a row sees."""
    if not 0 <= seq < len(table):
        return []
    n = max(0, min(length, max_keys, len(table[seq]) * page_size))
    at = [slot_of(table, n_pages, page_size, seq, j)
          for j in range(max(0, n - window) if window else 0, n)]
    return [a for a in at if a is not None]


def attend(q, k, v, scale):
    """One row: q [H][D], k and v [keys][Hk][D] -> (out [H][D], lse [H], the scores' sums of
    |scale q k|: their largest per head, and out with |v|: the measures of rounding errors)."""
    H, D = q.shape
    out, size = np.zeros((H, D)), np.zeros((H, D))
    lse, most = np.full(H, -np.inf), np.zeros(H)
    if len(k) == 0:
        return out, lse, most, size
    group = H // k.shape[1]
    for h in range(H):
        kk, vv = k[:, h // group].astype(np.float64), v[:, h // group].astype(np.float64)
        z = scale * (kk @ q[h].astype(np.float64))
        w = np.exp(z - z.max())
        lse[h] = z.max() + np.log(w.sum())
        w /= w.sum()
        out[h], size[h] = w @ vv, w @ np.abs(vv)
        most[h] = abs(scale) * (np.abs(kk) @ np.abs(q[h].astype(np.float64))).max()
    return out, lse, most, size


def process_logits(x, history=(), prompt=0, repetition=1.0, presence=0.0, frequency=0.0,
                   biases=(), mask=None):
    """One row: (logits, next token, magnitude of each entry's intermediate values)."""
    x = np.array(x, np.float64)
    size = np.abs(x)
    V = len(x)
    times = {}
    for i, t in enumerate(history):
        if 0 <= t < V:
            times[t] = times.get(t, 0) + (i >= prompt)
    for t, c in times.items():
        x[t] = x[t] / repetition if x[t] > 0 else x[t] * repetition
        size[t] = max(size[t], abs(x[t]))
        x[t] -= frequency * c
        if c > 0:
            x[t] -= presence
        size[t] += abs(frequency * c) + abs(presence)
    last = {int(i): b for i, b in biases if 0 <= i < V}
    for t, b in last.items():
        x[t] += b
        size[t] += abs(b)
    if mask is not None:
        x[[v for v in range(V) if not (int(mask[v // 32]) >> (v % 32)) & 1]] = -np.inf
    best, token = -np.inf, -1
    for t in range(V):
        if x[t] > best:
            best, token = x[t], t
    return x, token, size
