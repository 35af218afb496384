"""GPU parity of the calls for drafted tokens (exactmoe_drafts.h) against their
fp64 oracle (oracle/drafts_oracle.py).

Tolerances, from the operations alone (u = 2^-24): those of tests/test_gpu_serving.py
for rotations and for the attention; and for the tree attention's shaped scores
  cap         x / cap, tanh and the product: a few roundings each, 16 u |x|;
  bias        its slope and that of log2 e, the distance, their product with the
              score's added: 6 u (|x| + |bias|) of a score's terms.
Moves and the acceptance are exact.
"""
import math

import numpy as np
import pytest
import torch

from oracle import drafts_oracle as O
from oracle import serving_oracle as S
from paper_2608_15383_amd import api
from paper_2608_15383_amd._lib import EMOE_EINVAL, ExactMoEError
from tests.test_gpu_serving import HALF, TYPES, U, Cache, check, f64, gpu, ids, table_for

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3")]


def random_tree(rng, nodes, reach=8):
    """Masks of a tree: every node sees itself and its parent's."""
    masks = []
    for i in range(nodes):
        p = int(rng.integers(max(0, i - reach), i)) if i else -1
        masks.append((1 << i) | (masks[p] if p >= 0 else 0))
    return masks


def bits64(masks):
    return gpu(np.array([m & (2 ** 64 - 1) for m in masks], np.uint64).view(np.int64))


# ---------------------------------------------------------------- append
def run_axes(kind, cache_kind, tokens, heads, hk, d, page, rotary, inter, n_axes, seed, axes="mixed",
             in_place=False):
    rng = np.random.default_rng(seed)
    seqs = rng.integers(0, 4, tokens)
    base = rng.integers(0, 5 * page, 4)
    pos = base[seqs] + np.array([np.sum(seqs[:i] == s) for i, s in enumerate(seqs)])
    table, pages = table_for(rng, base + tokens, page)
    c = Cache(cache_kind, pages, page, hk, d, seed)
    if tokens > 4:
        seqs[1], pos[2], seqs[3] = -1, -5, 4                       # padding tokens
        table[seqs[4], pos[4] // page] = rng.choice([-1, pages])   # no page there
    angles = rng.integers(-50, 5000, (tokens, n_axes))
    if axes == "mixed":
        axis = rng.integers(0, n_axes, rotary // 2)
        axis[0] = -1 if rotary else 0
        axis[-1] = n_axes
    else:
        axis = np.zeros(rotary // 2, int)
    wide = torch.randn(tokens, (heads + 2 * hk) * d + 8, device="cuda:0").to(TYPES[kind])
    q, k, v = (x.unflatten(1, (-1, d)) for x in
               wide[:, :-8].split([heads * d, hk * d, hk * d], 1))
    freq = api.rope_frequencies(rotary)
    q0, k0, v0 = f64(q), f64(k), f64(v)
    q_out = torch.full((tokens, heads, d), 7.0, device="cuda:0", dtype=TYPES[kind])
    want_q, stored = O.append_axes(q0, k0, v0, pos, angles, axis, seqs, table, pages, page, f64(freq),
                                   inter)
    kb, vb = c.bits("k").clone(), c.bits("v").clone()
    stretched = ids(np.concatenate([angles, angles[:, :1]], 1))[:, :n_axes]   # a stride of its own
    api.paged_append_axes(c.kv, q, k, v, ids(pos), stretched, ids(axis) if axes == "mixed" else None,
                          ids(table), freq, seqs=ids(seqs), q_out=None if in_place else q_out,
                          interleaved=inter)
    torch.cuda.synchronize()
    got_q = f64(q if in_place else q_out)
    rel, tiny = HALF[kind]
    noise = lambda x: 4 * U * 2 * np.abs(x).max(-1, keepdims=True)
    for t in range(tokens):
        if want_q[t] is None:
            assert np.array_equal(got_q[t], q0[t] if in_place else np.full((heads, d), 7.0)), t
        else:
            check(got_q[t], want_q[t], rel * np.abs(want_q[t]) + noise(q0[t]) * (1 + rel) + tiny, t)
    rel, tiny = HALF[cache_kind]
    ks = np.ones(hk) if c.ks is None else f64(c.ks)
    vs = np.ones(hk) if c.vs is None else f64(c.vs)
    gk, gv = f64(c.k.float()), f64(c.v.float())
    for (p, s), (kk, vv) in stored.items():
        kk, vv = kk / ks[:, None], vv / vs[:, None]
        near = noise(kk) + 2 * U * np.abs(kk)
        limit = 448.0 if cache_kind == "e4m3" else np.inf
        kk, vv = np.clip(kk, -limit, limit), np.clip(vv, -limit, limit)
        check(gk[p, s], kk, rel * np.abs(kk) + (1 + rel) * near + tiny, f"k {p} {s}")
        check(gv[p, s], vv, rel * np.abs(vv) + 2 * U * np.abs(vv) + tiny, f"v {p} {s}")
    keep = np.ones((pages, page), bool)
    for p, s in stored:
        keep[p, s] = False
    at = gpu(np.flatnonzero(keep))
    for now, was in ((c.bits("k"), kb), (c.bits("v"), vb)):
        assert torch.equal(now.reshape(pages * page, -1)[at], was.reshape(pages * page, -1)[at])


@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("d,rotary,inter,n_axes", [(64, 64, False, 3), (64, 32, True, 2),
                                                   (128, 128, False, 1), (128, 128, True, 4),
                                                   (256, 176, False, 3), (256, 16, True, 1)])
def test_axes(kind, cache_kind, d, rotary, inter, n_axes):
    run_axes(kind, cache_kind, 11, 5, 5, d, 8, rotary, inter, n_axes, seed=d + rotary)


@pytest.mark.parametrize("tokens,opts", [(1, {}), (2, dict(axes=None)), (70, dict(in_place=True)),
                                         (300, dict(axes=None))])
def test_axes_sizes(tokens, opts):
    run_axes("bf16", "bf16", tokens, 4, 2, 128, 16, 128, False, 3, seed=tokens, **opts)


def test_axes_of_positions_are_the_plain_append():
    """One axis whose angles are the positions: the bits of paged_append."""
    for kind, cache_kind in KINDS:
        caches, outs = [], []
        x = torch.randn(3, 9, 4, 128, device="cuda:0").to(TYPES[kind])
        pos = ids(np.arange(100, 109))
        for axes in (False, True):
            c = Cache(cache_kind, 8, 16, 4, 128, 3)
            c.k.view(torch.uint8).zero_(), c.v.view(torch.uint8).zero_()
            q = torch.empty_like(x[0])
            args = (x[0], x[1], x[2], pos)
            rest = (ids(np.arange(8)[None].repeat(9, 0)), api.rope_frequencies(128))
            if axes:
                api.paged_append_axes(c.kv, *args, pos[:, None], None, *rest, q_out=q,
                                      seqs=ids([0] * 9))
            else:
                api.paged_append(c.kv, *args, *rest, q_out=q, seqs=ids([0] * 9))
            caches.append(c), outs.append(q)
        assert torch.equal(*outs)
        for which in "kv":
            assert torch.equal(caches[0].bits(which), caches[1].bits(which))
            assert caches[0].bits(which).any()


# ---------------------------------------------------------------- tree attention
def run_tree(kind, cache_kind, lengths, nodes, heads, hk, d, page, seed, window=0, cap=0.0,
             slopes=False, seqs=None, max_keys=None, max_nodes=None, holes=0, scale=None,
             slots_inside=False, gap=0, uniform=False, masks=None, ws=None, spare_rows=2, poison=None):
    """poison(cache, slot): changes what lies there, once all is stored."""
    rng = np.random.default_rng(seed)
    trees = len(lengths)
    seqs = np.arange(trees) if seqs is None else np.asarray(seqs)
    n_seqs = max(1, int(seqs.max()) + 1)
    room = [max([n + t for n, t, s in zip(lengths, nodes, seqs) if s == i] + [0]) for i in range(n_seqs)]
    table, pages = table_for(rng, room, page)
    c = Cache(cache_kind, pages, page, hk, d, seed, slots_inside, gap)
    for _ in range(holes):
        table[rng.integers(0, n_seqs), rng.integers(0, table.shape[1])] = rng.choice([-1, pages, 1 << 30])
    max_keys = max(max(n + t for n, t in zip(lengths, nodes)), 0) if max_keys is None else max_keys
    given = masks is not None
    if masks is None:
        masks = [O.chain(t) if uniform else random_tree(rng, t) for t in nodes]
    at = [[O.node_keys(m, i, table, pages, page, int(s), n, max_keys, window) for i in range(len(m))]
          for m, s, n in zip(masks, seqs, lengths)]
    stored = c.fill(sorted({x for tree in at for node in tree for x, _ in node}))
    if poison:
        poison(c, stored)
    rows = sum(nodes)
    total = rows if uniform else rows + spare_rows                  # rows of no tree at the end
    wide = torch.randn(total, heads * d + 8, device="cuda:0").to(TYPES[kind])
    q = wide[:, :-8].unflatten(1, (heads, d))
    out = torch.full((total + 1, heads * d + 16), 7.0, device="cuda:0", dtype=TYPES[kind])
    o = out[:total, :heads * d].unflatten(1, (heads, d))
    lse = torch.full((total + 1, heads), 7.0, device="cuda:0")
    most = max(nodes) if max_nodes is None else max_nodes
    slope = gpu((2.0 ** -np.arange(1, heads + 1)).astype(np.float32)) if slopes else None
    if ws is None:
        ws = torch.full((api.paged_tree_attention_workspace_bytes(c.kv, trees, heads, max_keys, most),),
                        255, dtype=torch.uint8, device="cuda:0")
    flat = [m for t in masks for m in t] + [0] * (total - rows)
    starts = ids(np.concatenate([[0], np.cumsum(nodes)]))
    call = lambda: api.paged_tree_attention(
        c.kv, q, ids(table), ids(lengths), o, ws, max_keys, most,
        tree=None if uniform and not given else bits64(flat), starts=None if uniform else starts,
        seqs=ids(seqs), scale=scale, cap=cap, slopes=slope, window=window, lse=lse[:total])
    call()
    torch.cuda.synchronize()
    got, z = f64(o), f64(lse)
    assert bool((out[rows:] == 7).all()) and bool((out[:, heads * d:] == 7).all())
    assert bool((lse[rows:] == 7).all())
    sc = 1 / math.sqrt(d) if scale is None else scale
    rel, tiny = HALF[kind]
    sl = None if slope is None else f64(slope)
    r = 0
    for g in range(trees):
        for i in range(nodes[g]):
            n = len(at[g][i])
            k = np.stack([stored[x][0] for x, _ in at[g][i]]) if n else np.zeros((0, hk, d))
            v = np.stack([stored[x][1] for x, _ in at[g][i]]) if n else np.zeros((0, hk, d))
            with np.errstate(all="ignore"):
                want, want_lse, size_z, shaped, size = O.attend(f64(q)[r], k, v,
                                                                [y for _, y in at[g][i]], sc, cap, sl)
            # An infinity among the values makes its dimension infinite or NaN: two halves of a weight
            # multiply it.
            lost = ~np.isfinite(want) & ~np.isfinite(got[r])
            got[r][lost] = want[lost]
            dz = 2 * (d + 4) * U * size_z + 22 * U * shaped * bool(cap or slopes)
            bound = (2 * dz[:, None] + 2.0 ** -15 + 4 * (n + 64) * U) * size
            check(got[r], want, bound * (1 + rel) + rel * np.abs(want) + tiny,
                  f"tree {g} node {i} of {n} keys")
            limit = dz + (n + 64) * U + 4 * U * np.where(n, np.abs(want_lse), 0) + 2.0 ** -20
            check(z[r], want_lse, limit, f"lse {g} {i}")
            r += 1
    first = o.clone()
    call()
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), o.view(torch.int16))   # equal calls, equal bits
    return got


EDGES = [0, 1, 2, 15, 31, 32, 33, 63, 65, 127, 129, 255, 257, -3]


@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [8, 16, 256])
def test_tree_lengths(kind, cache_kind, d, page):
    rng = np.random.default_rng(d + page)
    nodes = rng.integers(0, 14, len(EDGES)).tolist()
    nodes[0], nodes[1], nodes[2] = 1, 13, 0
    run_tree(kind, cache_kind, EDGES, nodes, 4, 2, d, page, seed=d + page)


@pytest.mark.parametrize("nodes", [1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 63, 64])
@pytest.mark.parametrize("cache_kind", ["bf16", "e4m3"])
def test_tree_nodes(nodes, cache_kind):
    run_tree("bf16", cache_kind, [100, 40, 0], [nodes, 1, nodes], 4, 2, 128, 16, seed=nodes)


@pytest.mark.parametrize("heads,hk", [(1, 1), (16, 16), (3, 3), (5, 1), (16, 1), (17, 1), (40, 1),
                                      (28, 4), (21, 3), (64, 2)])
@pytest.mark.parametrize("kind,cache_kind,d", [("bf16", "bf16", 128), ("fp16", "fp16", 64),
                                               ("bf16", "e4m3", 256)])
def test_tree_head_layouts(heads, hk, kind, cache_kind, d):
    run_tree(kind, cache_kind, [1, 70, 301, 0], [7, 3, 9, 2], heads, hk, d, 16, seed=heads)


def test_tree_of_more_lines_than_workgroups():
    run_tree("bf16", "bf16", [33, 0, 70], [2, 1, 3], 1200, 600, 64, 8, seed=1)


@pytest.mark.parametrize("lengths,nodes,heads,hk,d,page", [
    ([5000], [7], 8, 2, 128, 16), ([4096, 1, 4097], [4, 4, 9], 4, 4, 64, 64),
    ([12011], [3], 4, 1, 256, 128), ([5000, 40, 7, 1200], [16, 1, 5, 8], 12, 2, 128, 8),
    ([1] * 40 + [3001], [2] * 41, 4, 4, 64, 16), ([700] * 33, [2] * 33, 8, 8, 128, 32),
    ([20000], [2], 2, 1, 64, 1024), ([3000, 2500, 1, 3100], [33, 60, 3, 20], 4, 1, 128, 16),
    ([2000, 5, 900], [64, 30, 64], 2, 1, 256, 16), ([300] * 70, [3] * 70, 2, 2, 64, 16),
    ([900, 1000], [40, 50], 8, 2, 64, 32)])
@pytest.mark.parametrize("kind,cache_kind", [("bf16", "bf16"), ("fp16", "e4m3"), ("fp16", "fp16")])
def test_tree_long_and_ragged(lengths, nodes, heads, hk, d, page, kind, cache_kind):
    run_tree(kind, cache_kind, lengths, nodes, heads, hk, d, page, seed=len(lengths))


@pytest.mark.parametrize("window", [1, 2, 7, 32, 100, 1000, (1 << 31) - 1])
@pytest.mark.parametrize("page,d", [(8, 64), (64, 128)])
def test_tree_window(window, page, d):
    run_tree("bf16", "bf16", [0, 1, 31, 100, 133, 2000, 1025], [9, 2, 3, 17, 1, 20, 5], 4, 2, d, page,
             seed=window % 97, window=window)


@pytest.mark.parametrize("cap,slopes,window", [(30.0, False, 0), (0.0, True, 0), (5.0, True, 50),
                                               (0.5, False, 7), (1e4, True, 0), (2.0 ** -60, False, 0),
                                               (2.0 ** 60, False, 0)])
@pytest.mark.parametrize("kind,cache_kind,d", [("bf16", "bf16", 128), ("fp16", "fp16", 64),
                                               ("fp16", "e4m3", 256)])
def test_tree_shaped_scores(cap, slopes, window, kind, cache_kind, d):
    run_tree(kind, cache_kind, [0, 70, 333, 1500], [9, 5, 20, 3], 6, 2, d, 16, seed=4, window=window,
             cap=cap, slopes=slopes, scale=1.0 if cap else None)


@pytest.mark.parametrize("page", [8, 16, 128])
@pytest.mark.parametrize("cache_kind", ["fp16", "e4m3"])
def test_tree_missing_pages(page, cache_kind):
    run_tree("fp16", cache_kind, [300, 33, 1, 900, 64, 8], [6, 9, 20, 3, 1, 8], 4, 2, 64, page,
             seed=page, holes=9)


@pytest.mark.parametrize("slots_inside,gap", [(True, 0), (False, 64), (True, 16)])
def test_tree_layouts(slots_inside, gap):
    for kind in ("bf16", "e4m3"):
        run_tree("bf16", kind, [70, 0, 200], [5, 9, 2], 4, 2, 128, 16, seed=gap,
                 slots_inside=slots_inside, gap=gap)


@pytest.mark.parametrize("nodes", [1, 6, 64])
def test_tree_chains_without_starts(nodes):
    run_tree("bf16", "bf16", [70, 0, 200], [nodes] * 3, 4, 2, 64, 16, seed=1, uniform=True)


def test_tree_masks_of_any_kind():
    """Masks that see later nodes (a block seen whole), not themselves, nothing at all, bits past
    the tree."""
    masks = [[0b1111] * 4, [0, 0b1, 0b10, ~0], [0], [0, 0], [1 << 63, 2 ** 64 - 1]]
    for lengths in ([50, 3, 0, 0, 7], [0, 0, 0, 31, 32]):
        for more in ({}, dict(window=2), dict(slopes=True)):
            run_tree("bf16", "bf16", lengths, [4, 4, 1, 2, 2], 4, 2, 64, 8, seed=2, masks=masks, **more)


def test_tree_sequences_and_padding():
    """Several trees of one sequence, trees of no sequence, more trees than sequences."""
    run_tree("bf16", "bf16", [20, 50, 20, 7, 30], [4, 3, 5, 6, 2], 4, 2, 64, 16, seed=3,
             seqs=[0, 2, 0, -1, 1 << 20][:4] + [1])
    c = Cache("bf16", 4, 8, 1, 64, 0)
    q = torch.randn(3, 2, 64, device="cuda:0").to(torch.bfloat16)
    ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, 3, 2, 5000, 1), dtype=torch.uint8,
                     device="cuda:0")
    for table in (np.full((3, 400), -1), np.full((3, 400), 4), np.zeros((3, 0)), np.zeros((0, 400))):
        out, lse = torch.full_like(q, 7), torch.full((3, 2), 7.0, device="cuda:0")
        api.paged_tree_attention(c.kv, q, gpu(table.astype(np.int32)), ids([4999, 0, 40]), out, ws,
                                 5000, 1, lse=lse)
        torch.cuda.synchronize()
        assert not out.any() and bool((lse == -math.inf).all())


def test_tree_cuts_to_max_keys_and_table():
    for max_keys in (64, 66, 0, 5, 1 << 30):
        run_tree("bf16", "bf16", [100, 64, 62, 10], [5, 6, 7, 3], 4, 2, 64, 16, seed=4, max_keys=max_keys)


def test_tree_bounds_its_starts():
    """Starts that point outside the rows, go backwards or hold more nodes than max_nodes: what
    belongs to no tree stays."""
    c = Cache("bf16", 8, 16, 2, 64, 5)
    c.fill([(p, s) for p in range(8) for s in range(16)])
    q = torch.randn(12, 4, 64, device="cuda:0").to(torch.bfloat16)
    table = ids([[0, 1, 2], [3, 4, 5]])
    ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, 2, 4, 48, 4), dtype=torch.uint8,
                     device="cuda:0")

    def run(starts):
        out = torch.full_like(q, 7)
        api.paged_tree_attention(c.kv, q, table, ids([20, 9]), out, ws, 48, 4, starts=ids(starts))
        torch.cuda.synchronize()
        return out

    good = run([3, 7, 11])
    for starts, rows in (([3, 9, 13], [0, 0, 0, 1, 1, 1, 1, 0, 0, 0, 0, 0]),
                         ([3, -5, 2 ** 31 - 1], [0] * 12), ([-2 ** 31, 12, 2 ** 31 - 1], [0] * 12),
                         ([3, 7, 7], [0, 0, 0, 1, 1, 1, 1, 0, 0, 0, 0, 0])):
        got = run(starts)
        for r, there in enumerate(rows):
            want = good[r] if there else torch.full_like(good[r], 7)
            if there or starts != [3, 9, 13]:
                assert torch.equal(got[r], want), (starts, r)


@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("d,heads", [(64, 2), (128, 8), (256, 4)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_tree_unseen_values_have_no_effect(kind, cache_kind, d, heads, value):
    """A node of NaN or infinities: nodes that do not see it do not notice; likewise keys before
    the window of some nodes only."""
    if cache_kind == "e4m3" and value == math.inf:
        pytest.skip("the type has no infinity")
    n, page = 45, 16
    masks = [0b1, 0b11, 0b101, 0b1011, 0b10101, 0b100001, 0b1100001]
    for window in (0, 40):
        def outputs(bad_nodes, bad_keys):
            c = Cache(cache_kind, 5, page, 1, d, 9)
            c.fill([(p, s) for p in range(4) for s in range(page)])
            for at in [n + b for b in bad_nodes] + bad_keys:
                for t in (c.k, c.v):
                    bits = torch.tensor(value).to(t.dtype)
                    t.view(torch.uint8 if cache_kind == "e4m3" else torch.int16)[at // page, at % page] = \
                        bits.view(torch.uint8 if cache_kind == "e4m3" else torch.int16).item()
            q = torch.randn(7, heads, d, device="cuda:0",
                            generator=torch.Generator("cuda:0").manual_seed(3)).to(TYPES[kind])
            out = torch.empty_like(q)
            ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, 1, heads, n + 7, 7),
                             dtype=torch.uint8, device="cuda:0")
            api.paged_tree_attention(c.kv, q, ids([[0, 1, 2, 3]]), ids([n]), out, ws, n + 7, 7,
                                     tree=bits64(masks), starts=ids([0, 7]), window=window)
            torch.cuda.synchronize()
            return f64(out)

        good = outputs([], [])
        for bad in ([1], [2, 3], [6]):
            got = outputs(bad, [])
            for i, m in enumerate(masks):
                if any((m >> b) & 1 for b in bad):
                    assert not np.isfinite(got[i]).any()
                else:
                    assert np.array_equal(got[i], good[i]), (window, bad, i)
        if window:
            got = outputs([], [n - window + 1])      # inside the windows of depths 0 only
            for i, depth in enumerate(O.depths(masks)):
                assert np.isfinite(got[i]).all() == (depth > 0)
                assert depth == 0 or np.array_equal(got[i], good[i])


def test_tree_infinite_value_in_one_dimension():
    """Its own dimension is infinite or NaN for those that see it, the others are as without it."""
    for kind in ("bf16", "fp16"):
        def poison(c, stored):
            (p, s) = sorted(stored)[20]
            c.v[p, s, 0, 5] = math.inf
            stored[p, s][1][0, 5] = math.inf
        got = run_tree(kind, kind, [37], [6], 2, 1, 64, 8, seed=6, poison=poison)
        assert np.isinf(got[:, :, 5]).any()


def test_tree_offsets_past_32_bits():
    """A pool above 8 GiB: pages at its two ends."""
    page, hk, d, pages = 64, 8, 256, 18000
    kv = torch.empty(2, pages, page, hk, d, device="cuda:0", dtype=torch.bfloat16)
    small = torch.randn(2, 4, page, hk, d, device="cuda:0").to(torch.bfloat16)
    at = [0, pages - 1, 17000, 8192]
    kv[:, at] = small
    q = torch.randn(5, 8, d, device="cuda:0").to(torch.bfloat16)
    outs = []
    for t, table in ((kv, at), (small, [0, 1, 2, 3])):
        c = api.PagedKV(t[0], t[1])
        out = torch.empty_like(q)
        ws = torch.empty(api.paged_tree_attention_workspace_bytes(c, 1, 8, 256, 5), dtype=torch.uint8,
                         device="cuda:0")
        api.paged_tree_attention(c, q, ids([table]), ids([250]), out, ws, 256, 5)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs)


def test_tree_many_small_trees():
    """More trees than a wavefront's lanes, many of them empty."""
    rng = np.random.default_rng(0)
    run_tree("bf16", "bf16", rng.integers(0, 400, 150).tolist(), rng.integers(0, 4, 150).tolist(), 2, 1,
             64, 16, seed=5)
    run_tree("bf16", "bf16", rng.integers(0, 40, 700).tolist(), rng.integers(0, 3, 700).tolist(), 2, 2,
             64, 8, seed=6, max_nodes=64)


@pytest.mark.parametrize("lengths,hk", [([3, 2, 1, 0] * 80 + [2500, 900], 2), ([40] * 599 + [700], 1),
                                        ([2000] * 90, 2), ([500] * 150 + [1, 0], 2), ([1001] * 64, 4)])
def test_tree_many_trees_cut(lengths, hk):
    """Long keys cut over workers, and more trees than a wavefront's lanes, or than there are workers."""
    rng = np.random.default_rng(len(lengths))
    run_tree("bf16", "bf16", lengths, rng.integers(0, 3, len(lengths)).tolist(), 2 * hk, hk, 64, 16, seed=8,
             max_nodes=2)


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("kind,cache_kind,d", [("bf16", "bf16", 128), ("fp16", "e4m3", 64)])
def test_tree_outputs_for_every_cu(kind, cache_kind, d, slopes):
    """Some 300 outputs of up to 500 keys: whole, with a bias by distance cut."""
    rng = np.random.default_rng(2)
    lengths, nodes = rng.integers(0, 480, 38), rng.integers(1, 18, 38)
    lengths[3], nodes[3] = 480, 17
    run_tree(kind, cache_kind, lengths.tolist(), nodes.tolist(), 16, 8, d, 16, seed=9, slopes=slopes)


def test_tree_more_trees_than_a_launch():
    """Seven trees over and over: each as often as it comes gives the same bits."""
    n, times = 7, 10001
    c = Cache("bf16", 40, 8, 1, 64, 1)
    c.fill([(p, s) for p in range(40) for s in range(8)])
    table = ids(np.arange(35).reshape(7, 5))
    lengths, seqs = [0, 7, 31, 38, 8, 20, 33], list(range(n))
    q = torch.randn(n, 2, 64, device="cuda:0").to(torch.bfloat16)
    outs = []
    for k in (1, times):
        ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, n * k, 2, 40, 1), dtype=torch.uint8,
                         device="cuda:0")
        out = torch.empty(n * k, 2, 64, device="cuda:0", dtype=torch.bfloat16)
        api.paged_tree_attention(c.kv, q.repeat(k, 1, 1), table, ids(lengths * k), out, ws, 40, 1,
                                 seqs=ids(seqs * k))
        outs.append(out.view(torch.int16).unflatten(0, (k, n)))
    torch.cuda.synchronize()
    assert outs[0].any() and bool((outs[1] == outs[0]).all())


@pytest.mark.parametrize("kind,cache_kind,d,heads", [("fp16", "fp16", 64, 1), ("fp16", "fp16", 128, 8),
                                                     ("fp16", "e4m3", 256, 1), ("bf16", "bf16", 128, 8)])
def test_tree_of_small_weights(kind, cache_kind, d, heads):
    """Values of 0 where the weights are large, large ones where they are small: a bias of half of
    the distance leaves weights from 1 to e^-41."""
    def poison(c, stored):                       # one page: a slot is its position
        for p, s in stored:
            x = 384.0 if s < 62 else 0.0
            c.v[p, s] = torch.tensor(x).to(c.v.dtype)
            stored[p, s][1][:] = x if c.vs is None else x * f64(c.vs)[:, None]

    run_tree(kind, cache_kind, [80], [3], heads, 1, d, 128, seed=11, slopes=True, poison=poison, scale=0.05)


def test_tree_workspace_and_graphs():
    """One workspace for calls of different sizes, eager and in two captured graphs, replayed in turn
    with other work between; a stream of its own; two streams with a workspace each."""
    c = Cache("bf16", 600, 16, 2, 64, 4)
    c.fill([(p, s) for p in range(600) for s in range(16)])
    rng = np.random.default_rng(3)
    calls = []
    for trees, nodes, longest in ((3, 9, 1500), (40, 2, 900), (1, 40, 2900)):
        table = ids(rng.integers(0, 600, (trees, -(-longest // 16) + 4)))
        q = torch.randn(trees * nodes, 4, 64, device="cuda:0").to(torch.bfloat16)
        calls.append((q, table, ids(rng.integers(0, longest, trees)), longest + nodes, nodes))
    need = max(api.paged_tree_attention_workspace_bytes(c.kv, t[1].shape[0], 4, t[3], t[4]) for t in calls)
    spaces = [torch.full((need,), 255, dtype=torch.uint8, device="cuda:0") for _ in range(2)]

    def run(i, out, ws=0):
        q, table, lengths, keys, nodes = calls[i]
        api.paged_tree_attention(c.kv, q, table, lengths, out, spaces[ws], keys, nodes)

    want, outs, graphs = [torch.empty_like(t[0]) for t in calls], [torch.empty_like(t[0]) for t in calls], []
    for i in range(3):
        run(i, want[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(i, outs[i])
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1):
            outs[i].fill_(7)
            graphs[i].replay()
            if turn % 2:
                run(2, outs[2])
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i])
    # Other lengths in place: the graph takes them.
    calls[0][2].copy_(ids([1, 700, 3]))
    graphs[0].replay()
    run(0, want[0])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i, s in enumerate(streams):
        outs[i].fill_(7)
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                run(i, outs[i], i)
    torch.cuda.synchronize()
    for i in (0, 1):
        assert torch.equal(outs[i], want[i])


def test_tree_nothing():
    c = Cache("bf16", 1, 8, 1, 64, 2)
    e = torch.empty(0, 1, 64, device="cuda:0", dtype=torch.bfloat16)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    api.paged_tree_attention(c.kv, e, ids([[0]]), ids([]), e, ws, 8, 3)
    one = torch.full((4, 1, 64), 7.0, device="cuda:0", dtype=torch.bfloat16)
    api.paged_tree_attention(c.kv, one, ids([[0]]), ids([3, 3]), one, ws, 8, 3, starts=ids([0, 0, 0]))
    torch.cuda.synchronize()
    assert bool((one == 7).all())


# ---------------------------------------------------------------- acceptance
def run_accept(nodes, seed, agree=0.7, uniform=False, alphabet=5, with_tree=True):
    rng = np.random.default_rng(seed)
    trees, most = len(nodes), max(max(nodes), 1)
    masks = [random_tree(rng, t) if with_tree else O.chain(t) for t in nodes]
    tokens = [rng.integers(0, alphabet, t) for t in nodes]
    chosen = [rng.integers(-1, alphabet, t) for t in nodes]
    for t, x, m in zip(tokens, chosen, masks):
        for i in range(1, len(t)):
            before = m[i] & ((1 << i) - 1)
            if before and rng.random() < agree:
                x[before.bit_length() - 1] = t[i]
    lengths = rng.integers(0, 1000, trees)
    flat = lambda xs: ids(np.concatenate([np.asarray(x, np.int64) for x in xs] + [[7] * (not uniform)]))
    new = lambda *shape: torch.full(shape, 77, dtype=torch.int32, device="cuda:0")
    path, made = new(trees, most + 3)[:, :most], new(trees, most)
    accepted, after = new(trees), new(trees)
    api.accept_drafts(flat(tokens), flat(chosen), ids(lengths), path, accepted, made, after,
                      tree=bits64([x for m in masks for x in m] + [0] * (not uniform)) if with_tree else None,
                      starts=None if uniform else ids(np.concatenate([[0], np.cumsum(nodes)])))
    torch.cuda.synchronize()
    some = 0
    for g in range(trees):
        want, tok = O.accept(tokens[g], chosen[g], masks[g])
        some = max(some, len(want))
        pad = [-1] * (most - len(want))
        assert path[g].tolist() == want + pad and made[g].tolist() == tok + pad
        assert int(accepted[g]) == len(want) and int(after[g]) == lengths[g] + len(want)
    return some


def test_accept():
    assert run_accept([26], 1) > 1
    assert run_accept([0, 1, 2, 64, 63, 33, 0, 7], 2) > 2
    assert run_accept(np.random.default_rng(0).integers(0, 65, 500).tolist(), 3) > 5
    assert run_accept([64] * 9, 4, agree=1.0, alphabet=2) > 5
    assert run_accept([17] * 5, 5, uniform=True) > 1
    assert run_accept([64] * 5, 6, uniform=True, agree=1.0, with_tree=False) == 64
    assert run_accept([9, 3], 7, agree=0.0, alphabet=50304) == 1


def test_accept_takes_the_first_of_equal_children_and_no_missing_choice():
    tree = bits64([0b1, 0b11, 0b101, 0b1011, 0b10101])
    for chosen, want in (([5, 9, 8, 0, 0], [0, 1]), ([5, 6, 8, 0, 0], [0, 1, 3]), ([-1, 6, 6, 0, 0], [0]),
                         ([4, 6, 6, 0, 0], [0])):
        path, acc, n = ids([[0] * 5]), ids([0]), ids([10])
        api.accept_drafts(ids([1, 5, 5, 6, 6]), ids(chosen), n, path, acc, new_lengths=n, tree=tree)
        assert path.tolist() == [want + [-1] * (5 - len(want))]
        assert acc.tolist() == [len(want)] and n.tolist() == [10 + len(want)]


# ---------------------------------------------------------------- moves
def layers_of(kind, n, pages, page, hk, d, seed, slots_inside=False, gap=0):
    out = [Cache(kind, pages, page, hk, d, seed, slots_inside, gap) for _ in range(n)]
    rng = torch.Generator("cuda:0").manual_seed(seed)
    for c in out:
        for which in "kv":
            b = c.bits(which)
            b.copy_(torch.randint(0, 100, b.shape, device="cuda:0", generator=rng).to(b.dtype))
    return out


def whole(c, which):
    """The pages with what lies between their heads and slots."""
    t = c.k if which == "k" else c.v
    base = t._base if t._base is not None else t
    while base._base is not None:
        base = base._base
    return base.view(torch.uint8)


@pytest.mark.parametrize("kind,hk,d,page,slots_inside,gap", [
    ("bf16", 2, 128, 16, False, 0), ("e4m3", 3, 64, 8, False, 0), ("fp16", 1, 256, 32, False, 16),
    ("bf16", 4, 64, 16, True, 0), ("e4m3", 2, 256, 64, True, 32)])
@pytest.mark.parametrize("layers,trees,nodes", [(1, 1, 5), (3, 7, 64), (2, 40, 20), (70, 2, 9)])
def test_compact(kind, hk, d, page, slots_inside, gap, layers, trees, nodes):
    rng = np.random.default_rng(trees + nodes)
    lengths = rng.integers(0, 70, trees)
    lengths[0] = 0
    table, pages = table_for(rng, lengths + nodes, page)
    seqs = rng.permutation(trees)
    table = table[np.argsort(seqs)]
    accepted = rng.integers(0, nodes + 1, trees)
    path = np.stack([np.sort(rng.permutation(nodes)) for _ in range(trees)])
    for g in range(trees):
        keep = np.sort(rng.permutation(nodes)[:accepted[g]])
        path[g] = -1
        path[g, :len(keep)] = keep
    if trees > 4:
        seqs[1], lengths[2], seqs[3] = -1, -7, trees           # skipped
        accepted[4] = nodes + 50                               # cut
        table[seqs[5], table.shape[1] // 2] = -1               # a page that is missing
        path[6] = rng.permutation(nodes)                       # in any order
    cs = layers_of(kind, layers, pages, page, hk, d, 1, slots_inside, gap)
    before = [[c.bits(w).cpu().numpy().copy() for w in "kv"] for c in cs]
    wholes = [[whole(c, w).clone() for w in "kv"] for c in cs]
    api.paged_compact([c.kv for c in cs], ids(table), ids(lengths), ids(path), ids(accepted), seqs=ids(seqs))
    torch.cuda.synchronize()
    changed = 0
    for c, old, gaps in zip(cs, before, wholes):
        for w, x, gap_bytes in zip("kv", old, gaps):
            want = O.compact(x, table, pages, page, lengths, path, accepted, seqs)
            assert np.array_equal(c.bits(w).cpu().numpy(), want)
            changed += not np.array_equal(want, x)
            if gap:   # what lies between the heads stays
                c.bits(w).copy_(gpu(x))
                assert torch.equal(whole(c, w), gap_bytes)
    assert changed


def test_compact_without_seqs_is_by_row():
    cs = layers_of("bf16", 2, 6, 8, 2, 64, 3)
    old = [c.bits("v").clone() for c in cs]
    api.paged_compact(tuple(c.kv for c in cs), ids([[0, 1], [2, 3], [4, 5]]), ids([0, 5]),
                      ids([[0, 3, 7], [2, 4, 9]]), ids([3, 2]))
    torch.cuda.synchronize()
    for c, o in zip(cs, old):
        want = o.clone()
        want[0, 1], want[0, 2] = o[0, 3], o[0, 7]
        want[2, 5], want[2, 6] = o[2, 7], o[3, 1]
        assert torch.equal(c.bits("v"), want)


@pytest.mark.parametrize("kind,hk,d,page,slots_inside,gap", [
    ("bf16", 2, 128, 16, False, 0), ("e4m3", 3, 64, 8, False, 0), ("fp16", 1, 256, 32, False, 16),
    ("bf16", 5, 64, 128, True, 0), ("e4m3", 2, 256, 64, True, 32)])
@pytest.mark.parametrize("layers,parents,forks,with_fresh", [(1, 1, 3, True), (3, 9, 30, True),
                                                             (2, 5, 8, False), (70, 2, 3, True)])
def test_fork(kind, hk, d, page, slots_inside, gap, layers, parents, forks, with_fresh):
    rng = np.random.default_rng(parents + forks)
    have = rng.integers(1, 5 * page, parents)
    have[0] = 2 * page + 3
    table, used = table_for(rng, have, page, spare=0)
    pages = used + forks
    of = rng.integers(0, parents, forks)
    of[0] = 0
    lengths = have[of].copy()
    lengths[-1] = max(1, lengths[-1] // 2)
    fresh = used + rng.permutation(forks)
    if forks > 20:
        of[1], of[2], lengths[3], lengths[4] = -1, parents, -4, 0
        lengths[5], fresh[6], fresh[7] = 2 * page, -1, pages
        lengths[8] = 1 << 30
        table[1, 0] = -1
    cs = layers_of(kind, layers, pages, page, hk, d, 2, slots_inside, gap)
    before = [[c.bits(w).cpu().numpy().copy() for w in "kv"] for c in cs]
    new = torch.full((forks, table.shape[1] + 3), 77, dtype=torch.int32, device="cuda:0")
    api.paged_fork([c.kv for c in cs], ids(table), ids(of), ids(lengths),
                   ids(fresh) if with_fresh else None, new[:, :table.shape[1]])
    torch.cuda.synchronize()
    gone = fresh if with_fresh else np.full(forks, -1)
    for c, old in zip(cs, before):
        for w, x in zip("kv", old):
            rows, want = O.fork(x, table, pages, page, of, lengths, gone)
            assert np.array_equal(c.bits(w).cpu().numpy(), want)
            assert np.array_equal(want, x) == (not with_fresh)
    assert np.array_equal(new[:, :-3].cpu().numpy(), rows) and bool((new[:, -3:] == 77).all())


# ---------------------------------------------------------------- a run of them together
class Model:
    """One attention layer and an argmax over a small vocabulary, enough to decode with: token ids
    to queries, keys and values by a table, outputs to logits by another."""

    def __init__(self, heads, hk, d, vocab, seed, dtype=torch.bfloat16):
        g = torch.Generator("cuda:0").manual_seed(seed)
        r = lambda *s: torch.randn(*s, device="cuda:0", generator=g)
        self.heads, self.hk, self.d, self.dtype = heads, hk, d, dtype
        self.qkv = r(2, vocab, (heads + 2 * hk), d)      # a table for each of two layers
        self.head = r(heads * d, vocab)

    def parts(self, tokens, layer):
        x = self.qkv[layer][tokens.long()].to(self.dtype)
        return x.split([self.heads, self.hk, self.hk], 1)


def step_by_step(m, prompt, steps, cache, table, freq, window):
    """Greedy decoding, a token at a time, two layers' outputs added."""
    tokens = list(prompt)
    kvs = [c.kv for c in cache]
    ws = torch.zeros(api.paged_attention_workspace_bytes(kvs[0], 1, m.heads, 512), dtype=torch.uint8,
                     device="cuda:0")
    scores = []
    for p in range(len(prompt) + steps - 1):
        t = ids([tokens[p]])
        total = 0
        for layer, kv in enumerate(kvs):
            q, k, v = (x.contiguous() for x in m.parts(t, layer))
            api.paged_append(kv, q, k, v, ids([p]), table, freq)
            out = torch.empty_like(q)
            api.paged_attention(kv, q, table, ids([p + 1]), out, ws, 512, window=window)
            total = total + out.float()
        if p >= len(prompt) - 1:
            logits = total.flatten(1) @ m.head
            tokens.append(int(logits.argmax()))
            scores.append(logits.topk(2).values[0])
    return tokens[len(prompt):], scores


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("captured", [False, True])
def test_drafted_decoding_gives_the_greedy_tokens(window, captured):
    """Trees of drafts, some of them the tokens that greedy decoding gives: append, attend, choose,
    accept, compact, for three sequences of which one was forked from another; the accepted tokens
    are greedy decoding's, and so are the caches' keys and values, bit by bit."""
    m = Model(4, 2, 64, 50, 1)
    freq = api.rope_frequencies(64)
    steps, T, page = 24, 11, 8
    prompts = [[3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13], [7] * 20, None]
    prompts[2] = prompts[0]
    want, caches = [], []
    for p in prompts:
        c = [Cache("bf16", 12, page, 2, 64, 0) for _ in range(2)]
        tok, scores = step_by_step(m, p, steps, c, ids(np.arange(12)[None]), freq, window)
        # Greedy decoding is well defined here: no two logits within reach of the roundings.
        assert min(float(s[0] - s[1]) for s in scores) > 1e-2
        want.append(tok), caches.append(c)

    kvs = [Cache("bf16", 40, page, 2, 64, 0) for _ in range(2)]
    views = [c.kv for c in kvs]
    rng = np.random.default_rng(0)
    pool = rng.permutation(40)
    old = np.full((2, 12), -1)
    old[0, :2], old[1, :3] = pool[:2], pool[2:5]
    ws = torch.zeros(api.paged_attention_workspace_bytes(views[0], 64, 4, 512), dtype=torch.uint8,
                     device="cuda:0")
    for s, p in enumerate(prompts[:2]):                      # all but the prompt's last token
        n = len(p) - 1
        for layer, kv in enumerate(views):
            q, k, v = (x.contiguous() for x in m.parts(ids(p[:n]), layer))
            api.paged_append(kv, q, k, v, ids(np.arange(n)), ids(old), freq, seqs=ids([s] * n))
    new = torch.empty(3, 12, dtype=torch.int32, device="cuda:0")
    n0 = [len(p) - 1 for p in prompts]
    api.paged_fork(views, ids(old), ids([0, 1, 0]), ids(n0), ids([-1, -1, pool[5]]), new)
    table = new.cpu().numpy()
    at = 6
    for s in range(3):                                       # room for what comes
        for col in range(-(-n0[s] // page), 12):
            if at < 40:
                table[s, col] = pool[at]
                at += 1
    assert at <= 40
    table = ids(table)
    lengths = ids(n0)
    tokens = torch.zeros(3 * T, dtype=torch.int32, device="cuda:0")
    tree, depth = torch.zeros(3 * T, dtype=torch.int64, device="cuda:0"), ids([0] * (3 * T))
    seqs = ids(np.repeat(np.arange(3), T))
    slot = ids(np.tile(np.arange(T), 3))
    tws = torch.empty(api.paged_tree_attention_workspace_bytes(views[0], 3, 4, 128, T), dtype=torch.uint8,
                      device="cuda:0")
    lws = torch.zeros(api.process_logits_workspace_bytes(3 * T, 50), dtype=torch.uint8, device="cuda:0")
    path, made = ids(np.zeros((3, T))), ids(np.zeros((3, T)))
    accepted, after, chosen = ids([0] * 3), ids([0] * 3), ids([0] * (3 * T))

    def step():
        base = lengths.repeat_interleave(T)
        total = 0
        for layer, kv in enumerate(views):
            q, k, v = (x.contiguous() for x in m.parts(tokens, layer))
            api.paged_append_axes(kv, q, k, v, base + slot, (base + depth)[:, None].contiguous(), None,
                                  table, freq, seqs=seqs)
            out = torch.empty_like(q)
            api.paged_tree_attention(kv, q, table, lengths, out, tws, 128, T, tree=tree, window=window)
            total = total + out.float()
        logits = total.flatten(1) @ m.head
        api.process_logits(logits, workspace=lws, next_token=chosen)
        api.accept_drafts(tokens, chosen, lengths, path, accepted, made, after, tree=tree)
        api.paged_compact(views, table, lengths, path, accepted)
        lengths.copy_(after)

    last = [p[-1] for p in prompts]
    got = [[], [], []]
    graph = None
    rounds = 0
    while min(len(x) for x in got) < steps - T:
        host_tokens, host_masks = [], []
        for s in range(3):
            masks = random_tree(rng, T, reach=4)
            parents = [(mm & ((1 << i) - 1)).bit_length() - 1 for i, mm in enumerate(masks)]
            depths = O.depths(masks)
            t = [last[s]]
            for i in range(1, T):   # the greedy token of its depth, or any
                k = len(got[s]) + depths[i] - 1
                t.append(want[s][k] if k < steps and rng.random() < 0.6 else int(rng.integers(0, 50)))
            host_tokens += t
            host_masks += masks
            assert parents[0] == -1
        tokens.copy_(ids(host_tokens)), tree.copy_(bits64(host_masks))
        depth.copy_(ids([d for s in range(3) for d in O.depths(host_masks[s * T:s * T + T])]))
        if captured and graph is None:
            saved = [t.clone() for c in kvs for t in (c.bits("k"), c.bits("v"))]
            n_saved = lengths.clone()
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                step()
            torch.cuda.current_stream().wait_stream(stream)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for t, o in zip([t for c in kvs for t in (c.bits("k"), c.bits("v"))], saved):
                t.copy_(o)
            lengths.copy_(n_saved)
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        for s in range(3):
            count = int(accepted[s])
            assert count >= 1
            new_tokens = made[s].tolist()[:count]
            assert new_tokens == want[s][len(got[s]):len(got[s]) + count], (s, rounds)
            got[s] += new_tokens
            last[s] = new_tokens[-1]
        rounds += 1
    assert rounds < max(len(x) for x in got)     # drafts were accepted
    tab = table.cpu().numpy()
    for s in range(3):
        n = int(lengths[s])
        assert n == n0[s] + len(got[s])
        for c, ref in zip(kvs, caches[s]):
            for which in "kv":
                for p in range(n):
                    assert torch.equal(c.bits(which)[tab[s, p // page], p % page],
                                       ref.bits(which)[p // page, p % page]), (s, p)


def test_binding_checks_tensors():
    c = Cache("bf16", 4, 8, 2, 64, 0)
    q = torch.randn(6, 4, 64, device="cuda:0").to(torch.bfloat16)
    out, ws = torch.empty_like(q), torch.empty(1 << 22, dtype=torch.uint8, device="cuda:0")
    table, n, mask = ids([[0, 1], [2, 3]]), ids([3, 4]), bits64([1] * 6)
    good = dict(kv=c.kv, q=q, page_table=table, lengths=n, out=out, workspace=ws, max_keys=16, max_nodes=3,
                tree=mask)
    api.paged_tree_attention(**good)
    for bad in (dict(tree=mask.int()), dict(tree=mask[:5]), dict(starts=ids([0, 3])), dict(q=q.float()),
                dict(lengths=n.long()), dict(lengths=n.cpu()), dict(out=out[:5]), dict(workspace=ws[:8]),
                dict(workspace=None), dict(max_nodes=65), dict(max_nodes=4), dict(max_nodes="x"),
                dict(cap=-1.0), dict(cap=math.nan), dict(cap="x"), dict(slopes=torch.ones(3, device="cuda:0")),
                dict(lse=torch.ones(6, 3, device="cuda:0")), dict(window=1 << 40), dict(seqs=ids([0])),
                dict(page_table=table.t())):
        with pytest.raises(ExactMoEError) as e:
            api.paged_tree_attention(**{**good, **bad})
        assert e.value.status in (EMOE_EINVAL, -2), bad
    k = torch.randn(6, 2, 64, device="cuda:0").to(torch.bfloat16)
    for angles, axes in ((ids([0] * 6), None), (ids([[0]] * 5), None), (ids([[0]] * 6).long(), None),
                         (ids([[0]] * 6), ids([0] * 31))):
        with pytest.raises(ExactMoEError):
            api.paged_append_axes(c.kv, q, k, k, ids([0] * 6), angles, axes, table, api.rope_frequencies(64))
    path, acc = ids([[0] * 3] * 2), ids([0, 0])
    for bad in (dict(chosen=ids([0] * 5)), dict(path=path[0]), dict(accepted=ids([0])), dict(tree=mask.int()),
                dict(new_lengths=acc, lengths=None), dict(tokens=torch.zeros(6, dtype=torch.int32))):
        with pytest.raises(ExactMoEError):
            api.accept_drafts(**{**dict(tokens=ids([0] * 6), chosen=ids([0] * 6), lengths=n, path=path,
                                        accepted=acc), **bad})
    other = Cache("bf16", 4, 16, 2, 64, 0)
    for kvs in ([], [c.kv, other.kv], [c.kv, c.kv], [c.kv, None], [c.kv, 3]):
        with pytest.raises(ExactMoEError):
            api.paged_compact(kvs, table, n, path, acc)
        with pytest.raises(ExactMoEError):
            api.paged_fork(kvs, table, n, n, None, torch.empty_like(table))
    with pytest.raises(ExactMoEError):
        api.paged_fork([c.kv], table, n, n, None, table)
    with pytest.raises(ExactMoEError):
        api.paged_fork([c.kv], table, n, n, None, torch.empty_like(table)[:, :1])
