"""fp64 numpy statements of the calls for drafted tokens (exactmoe_drafts.h):
angles with several axes, the attention of a tree's nodes, the acceptance of
drafts, and the moves of keys and values between positions.  Test infrastructure
only; plain loops, shared with the statements of exactmoe_serving.h where the
header refers to them."""
from __future__ import annotations

import numpy as np

from oracle import serving_oracle as S


def depths(masks):
    """Of each node of a tree: how many nodes before it it sees."""
    return [sum((m >> j) & 1 for j in range(i)) for i, m in enumerate(masks)]


def chain(nodes):
    return [(1 << (i + 1)) - 1 for i in range(nodes)]


def append_axes(q, k, v, positions, angles, axes, seqs, table, n_pages, page_size, inv_freq,
                interleaved):
    """As serving_oracle.append, pair i turned by angles[t][axes[i]] * inv_freq[i]."""
    q_out, stored = [], {}
    for t, p in enumerate(positions):
        s = int(seqs[t])
        if p < 0 or not 0 <= s < len(table):
            q_out.append(None)
            continue
        turn = [angles[t][a] * f if 0 <= a < len(angles[t]) else 0.0 for a, f in zip(axes, inv_freq)]
        q_out.append(np.stack([S.rotate(h, 1, turn, interleaved) for h in q[t]]))
        at = S.slot_of(table, n_pages, page_size, s, int(p))
        if at is not None:
            stored[at] = (np.stack([S.rotate(h, 1, turn, interleaved) for h in k[t]]),
                          np.array(v[t], np.float64))
    return q_out, stored


def node_keys(masks, i, table, n_pages, page_size, seq, n, max_keys, window):
    """[((page, slot), |distance|)] of every key that node i of a tree behind n keys sees."""
    if not 0 <= seq < len(table) or n < 0:
        return []
    depth = depths(masks)
    out = []
    for j in range(max(0, n + depth[i] - window + 1) if window else 0, min(n, max_keys)):
        at = S.slot_of(table, n_pages, page_size, seq, j)
        if at is not None:
            out.append((at, abs(n + depth[i] - j)))
    for j in range(len(masks)):
        if not (masks[i] >> j) & 1 or n + j >= max_keys:
            continue
        if window and depth[j] <= depth[i] - window:
            continue
        at = S.slot_of(table, n_pages, page_size, seq, n + j)
        if at is not None:
            out.append((at, abs(depth[i] - depth[j])))
    return out


def attend(q, k, v, distance, scale, cap=0.0, slopes=None):
    """One node: q [H][D], k and v [keys][Hk][D], distance [keys] -> (out [H][D], lse [H], and the
    measures of rounding errors: the largest sum of |scale q k|, the largest score and bias of a
    key, per head, and out with |v|)."""
    H, D = q.shape
    out, size = np.zeros((H, D)), np.zeros((H, D))
    lse, most, shaped = np.full(H, -np.inf), np.zeros(H), np.zeros(H)
    if len(k) == 0:
        return out, lse, most, shaped, size
    group = H // k.shape[1]
    for h in range(H):
        kk, vv = k[:, h // group].astype(np.float64), v[:, h // group].astype(np.float64)
        x = scale * (kk @ q[h].astype(np.float64))
        if cap:
            x = cap * np.tanh(x / cap)
        bias = (0.0 if slopes is None else float(slopes[h])) * np.asarray(distance, np.float64)
        z = x - bias
        w = np.exp(z - z.max())
        lse[h] = z.max() + np.log(w.sum())
        w /= w.sum()
        out[h], size[h] = w @ vv, w @ np.abs(vv)
        most[h] = abs(scale) * (np.abs(kk) @ np.abs(q[h].astype(np.float64))).max()
        shaped[h] = (np.abs(x) + np.abs(bias)).max()
    return out, lse, most, shaped, size


def accept(tokens, chosen, masks):
    """The accepted nodes of one tree and the tokens chosen after them."""
    path, made = [], []
    node = 0 if len(tokens) else None
    while node is not None:
        path.append(node)
        made.append(int(chosen[node]))
        after = None
        for c in range(len(tokens) - 1, 0, -1):
            before = [j for j in range(c) if (masks[c] >> j) & 1]
            if before and before[-1] == node and tokens[c] == chosen[node] and chosen[node] >= 0:
                after = c
        node = after
    return path, made


def compact(pages, table, n_pages, page_size, lengths, paths, accepted, seqs):
    """pages [page][slot]..: a copy of them after the moves of every tree."""
    out = pages.copy()
    for n, path, m, s in zip(lengths, paths, accepted, seqs):
        if not 0 <= s < len(table) or n < 0:
            continue
        for i in range(min(m, len(path))):
            if path[i] <= i:
                continue
            a = S.slot_of(table, n_pages, page_size, s, n + int(path[i]))
            b = S.slot_of(table, n_pages, page_size, s, n + i)
            if a is not None and b is not None:
                out[b] = pages[a]
    return out


def fork(pages, table, n_pages, page_size, parents, lengths, fresh):
    """(new table, a copy of the pages after the copies)."""
    out, rows = pages.copy(), np.full((len(parents), table.shape[1]), -1, np.int64)
    for f, (p, n) in enumerate(zip(parents, lengths)):
        if not 0 <= p < len(table) or n < 0:
            continue
        n = min(n, table.shape[1] * page_size)
        for c in range(-(-n // page_size)):
            page = int(table[p][c])
            part = min(page_size, n - c * page_size)
            if part < page_size and 0 <= page < n_pages and 0 <= fresh[f] < n_pages:
                out[fresh[f], :part] = pages[page, :part]
                page = fresh[f]
            rows[f, c] = page
    return rows, out
