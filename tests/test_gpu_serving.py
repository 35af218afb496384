"""GPU parity of the batched decoding calls (exactmoe_serving.h) against their
fp64 oracle (oracle/serving_oracle.py).

Tolerances, from the operations alone (u = 2^-24, the rounding of an fp32
operation; half(t) = finfo(t).eps / 2, that of storing a 16-bit value):
  rotation    a c - b s: cosine and sine rounded to fp32, two products and a
              sum: 4 u (|a| + |b|), then the store;
  attention   a score of D products, summed in an order of the kernel's own and
              scaled: 2 (D + 4) u * (largest sum of |scale q k|) =: dz.  Weights
              are off by 2 dz + 2^-15 relatively (both exponents, exp itself,
              the two 16-bit halves: 2^-16), sums of n terms by 2 n u more:
              (2 dz + 2^-15 + 4 (n + 64) u) * sum w |v|, then the store;
  log-sum-exp dz + (n + 64) u + 4 u |lse| + 2^-20 (exp2, log2 and their bases);
  logits      at most six operations, each u of its intermediate values, the store.
"""
import math
import threading

import numpy as np
import pytest
import torch

from oracle import serving_oracle as S
from paper_2608_15383_amd import api
from paper_2608_15383_amd._lib import EMOE_EINVAL, EMOE_SERVING_TICKET_BYTES, ExactMoEError

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32,
         "e4m3": torch.float8_e4m3fn}
# Largest relative rounding of a store and half of the smallest step.
HALF = {"bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25), "f32": (0.0, 0.0),
        "e4m3": (2.0 ** -4, 2.0 ** -10)}


def gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else torch.tensor(a)
    return t.to("cuda:0") if dtype is None else t.to("cuda:0").to(dtype)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def ids(a):
    return gpu(np.asarray(a, np.int32))


def check(got, want, bound, label):
    bad = ~(np.abs(got - want) <= bound)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    bad &= ~same
    assert not bad.any(), (label, int(bad.sum()), got[bad][:4], want[bad][:4],
                           np.broadcast_to(bound, got.shape)[bad][:4])


class Cache:
    """A paged cache whose every slot starts as NaN."""

    def __init__(self, kind, pages, page, hk, d, seed, slots_inside=False, gap=0):
        self.kind, self.page, self.hk, self.d, self.pages = kind, page, hk, d, pages
        dt = TYPES[kind]
        shape = (pages, hk, page, d + gap) if slots_inside else (pages, page, hk, d + gap)
        raw = [torch.full(shape, math.nan, device="cuda:0").to(dt) for _ in range(2)]
        view = [r[..., :d].permute(0, 2, 1, 3) if slots_inside else r[..., :d] for r in raw]
        self.k, self.v = view
        self.rng = np.random.default_rng(seed)
        self.ks = self.vs = None
        if kind == "e4m3":
            self.ks, self.vs = (gpu((0.01 + 0.05 * self.rng.random(hk)).astype(np.float32))
                                for _ in range(2))
        self.kv = api.PagedKV(self.k, self.v, self.ks, self.vs)

    def bits(self, which):
        t = self.k if which == "k" else self.v
        return t.view(torch.uint8 if self.kind == "e4m3" else torch.int16)

    def fill(self, slots):
        """Random keys and values in these (page, slot); returns {slot: (k, v)} as stored, scaled."""
        if not slots:
            return {}
        p, s = (torch.tensor([x[i] for x in slots], device="cuda:0") for i in (0, 1))
        out = []
        for which, scale in (("k", self.ks), ("v", self.vs)):
            x = gpu(self.rng.standard_normal((len(slots), self.hk, self.d)).astype(np.float32))
            x = x if scale is None else x / scale[:, None]
            x = x.to(TYPES[self.kind])
            self.bits(which)[p, s] = x.view(self.bits(which).dtype)
            x = f64(x.float())
            out.append(x if scale is None else x * f64(scale)[:, None])
        return {at: (out[0][i], out[1][i]) for i, at in enumerate(slots)}


def table_for(rng, lengths, page, spare=2):
    """Shuffled pages for sequences of these lengths; -1 behind their ends."""
    need = [-(-max(n, 0) // page) for n in lengths]
    pool = rng.permutation(sum(need) + spare)
    table = np.full((len(lengths), max(1, max(need))), -1, np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = pool[at:at + n]
        at += n
    return table, sum(need) + spare


# ---------------------------------------------------------------- append
def run_append(kind, cache_kind, tokens, heads, hk, d, page, rotary, inter, seed, lengths=None,
               slots_inside=False, gap=0, with_q=True, in_place=False):
    rng = np.random.default_rng(seed)
    seqs = rng.integers(0, 4, tokens)
    base = rng.integers(0, 5 * page, 4) if lengths is None else np.asarray(lengths)
    nth = np.array([np.sum(seqs[:i] == s) for i, s in enumerate(seqs)])
    pos = base[seqs] + nth
    table, pages = table_for(rng, base + tokens, page)
    c = Cache(cache_kind, pages, page, hk, d, seed, slots_inside, gap)
    if tokens > 4:
        seqs[1], pos[2], seqs[3] = -1, -5, 4                       # padding tokens
        table[seqs[4], pos[4] // page] = rng.choice([-1, pages])   # no page there
    wide = torch.randn(tokens, (heads + 2 * hk) * d + 8, device="cuda:0").to(TYPES[kind])
    q, k, v = (x.unflatten(1, (-1, d)) for x in
               wide[:, :-8].split([heads * d, hk * d, hk * d], 1))
    freq = api.rope_frequencies(rotary) if rotary else None
    q0, k0, v0 = f64(q), f64(k), f64(v)
    q_out = torch.full((tokens + 2, heads, d), 7.0, device="cuda:0", dtype=TYPES[kind])
    want_q, stored = S.append(q0, k0, v0, pos, seqs, table, pages, page,
                              [] if freq is None else f64(freq), inter)
    kb, vb = c.bits("k").clone(), c.bits("v").clone()
    api.paged_append(c.kv, q if with_q else None, k, v, ids(pos), ids(table), freq, seqs=ids(seqs),
                     q_out=None if in_place or not with_q else q_out[:tokens], interleaved=inter)
    torch.cuda.synchronize()
    got_q = f64(q if in_place else q_out)
    rel, tiny = HALF[kind]
    noise = lambda x: 4 * U * 2 * np.abs(x).max(-1, keepdims=True)
    for t in range(tokens):
        if not with_q:
            break
        if want_q[t] is None:
            assert np.array_equal(got_q[t], q0[t] if in_place else np.full((heads, d), 7.0)), t
        else:
            check(got_q[t], want_q[t], rel * np.abs(want_q[t]) + noise(q0[t]) * (1 + rel) + tiny,
                  f"q {t}")
    if not in_place:
        assert np.all(got_q[tokens:] == 7.0)
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
        if cache_kind == kind:
            assert np.array_equal(gv[p, s], vv)                    # copied, not computed
    # Every other slot keeps its bytes.
    keep = np.ones((pages, page), bool)
    for p, s in stored:
        keep[p, s] = False
    at = gpu(np.flatnonzero(keep))
    for now, was in ((c.bits("k"), kb), (c.bits("v"), vb)):
        assert torch.equal(now.reshape(pages * page, -1)[at], was.reshape(pages * page, -1)[at])
    return len(stored)


@pytest.mark.parametrize("kind,cache_kind", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"),
                                             ("fp16", "e4m3")])
@pytest.mark.parametrize("d,rotary,inter", [(64, 64, False), (64, 32, True), (128, 128, False),
                                            (128, 128, True), (128, 32, False), (128, 0, False),
                                            (256, 256, False), (256, 16, True), (256, 176, False)])
def test_append(kind, cache_kind, d, rotary, inter):
    # Three tokens are padding, one or more have no page.
    n = run_append(kind, cache_kind, 11, 5, 5, d, 8, rotary, inter, seed=d + rotary)
    assert 3 <= n <= 7


@pytest.mark.parametrize("tokens,heads,hk,page,opts", [
    (1, 16, 16, 16, {}), (2, 8, 1, 1024, {}), (3, 3, 3, 32, dict(slots_inside=True)),
    (64, 7, 7, 16, dict(gap=16)), (129, 4, 2, 8, dict(slots_inside=True, gap=64)),
    (300, 6, 3, 64, {}), (12, 4, 2, 16, dict(with_q=False)), (13, 4, 2, 16, dict(in_place=True)),
])
def test_append_sizes_and_layouts(tokens, heads, hk, page, opts):
    for kind, cache_kind in (("bf16", "bf16"), ("fp16", "e4m3")):
        n = run_append(kind, cache_kind, tokens, heads, hk, 128, page, 128, False, seed=tokens, **opts)
        assert n == tokens if tokens <= 4 else n > 0


def test_append_far_positions():
    """Angles in fp64: a position near 2^21 of a window whose earlier pages were given back."""
    for inter in (False, True):
        table = np.full((2, (1 << 21) // 16 + 2), -1, np.int32)
        pos = np.array([(1 << 21) - 1, 1 << 21, 999_999, 1 << 22])   # the last: past the table
        seqs = np.array([0, 0, 1, 1])
        for i, (s, p) in enumerate(zip(seqs[:3], pos[:3])):
            table[s, p // 16] = i
        c = Cache("fp16", 3, 16, 2, 128, 1)
        q, k, v = (torch.randn(4, 2, 128, device="cuda:0").half() for _ in range(3))
        freq = api.rope_frequencies(128)
        q_out = torch.empty_like(q)
        want, stored = S.append(f64(q), f64(k), f64(v), pos, seqs, table, 3, 16, f64(freq), inter)
        api.paged_append(c.kv, q, k, v, ids(pos), ids(table), freq, seqs=ids(seqs), q_out=q_out,
                         interleaved=inter)
        # The angle itself: a product of fp64, off by 2^-53 of 2^22.
        slack = 2.0 ** -29 + 8 * U
        for t in range(4):
            check(f64(q_out)[t], want[t], 2.0 ** -11 * np.abs(want[t]) + slack * np.abs(f64(q)[t]).max(),
                  t)
        assert len(stored) == 3
        for (p, s), (kk, _) in stored.items():
            check(f64(c.k)[p, s], kk, 2.0 ** -11 * np.abs(kk) + slack * 5, (p, s))


def test_append_saturates_and_keeps_nan():
    c = Cache("e4m3", 1, 8, 1, 64, 2)
    k = torch.zeros(1, 1, 64, device="cuda:0", dtype=torch.bfloat16)
    k[0, 0, :6] = torch.tensor([1e6, -1e6, math.nan, math.inf, -math.inf, 0.0])
    c.ks.fill_(1.0), c.vs.fill_(0.5)
    api.paged_append(c.kv, None, k, k, ids([3]), ids([[0]]), None)
    for got in (f64(c.k.float())[0, 3, 0, :6], f64(c.v.float())[0, 3, 0, :6]):
        assert np.array_equal(got, [448, -448, math.nan, 448, -448, 0], equal_nan=True)
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    every = every[torch.isfinite(every)].to("cuda:0")              # the type's own values
    for part in every.split(64):
        k[0, 0, :] = 0
        k[0, 0, :len(part)] = part.to(torch.bfloat16)
        c.vs.fill_(1.0)
        api.paged_append(c.kv, None, k, k, ids([0]), ids([[0]]), None)
        assert torch.equal(c.k.float()[0, 0, 0], k[0, 0].float())
        assert torch.equal(c.v.float()[0, 0, 0], k[0, 0].float())


def test_append_ties_to_even_in_8_bits():
    c = Cache("e4m3", 1, 8, 1, 64, 2)
    c.ks.fill_(1.0), c.vs.fill_(1.0)
    k = torch.zeros(1, 1, 64, device="cuda:0", dtype=torch.float16)
    x = [17.0, 19.0, 21.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 440.0, 456.0]
    k[0, 0, :len(x)] = torch.tensor(x)
    api.paged_append(c.kv, None, k, k, ids([0]), ids([[0]]), None)
    want = [16.0, 20.0, 20.0, 1.0, 1.25, 0.0, 2.0 ** -8, 0.0, 448.0, 448.0]
    assert f64(c.v.float())[0, 0, 0, :len(x)].tolist() == want


def test_append_more_tokens_than_one_launch():
    """All but a few of 2^24 + 5 tokens are padding; the others are what a call of them alone gives."""
    n, d = (1 << 24) + 5, 64
    at = torch.tensor([0, (1 << 22) - 1, 1 << 22, n - 1], device="cuda:0")
    k = torch.empty(n, 1, d, device="cuda:0", dtype=torch.bfloat16)
    v = torch.empty_like(k)
    k[at], v[at] = (torch.randn(4, 1, d, device="cuda:0").to(k.dtype) for _ in "kv")
    seqs = torch.full((n,), -1, dtype=torch.int32, device="cuda:0")
    positions = torch.zeros_like(seqs)
    seqs[at] = 0
    positions[at] = ids([3, 4, 5, 7])
    caches = []
    for pick in (slice(None), at):
        pages = torch.zeros(2, 1, 8, 1, d, device="cuda:0", dtype=k.dtype)
        api.paged_append(api.PagedKV(pages[0], pages[1]), None, k[pick], v[pick], positions[pick],
                         ids([[0]]), api.rope_frequencies(d), seqs=seqs[pick])
        caches.append(pages)
    assert torch.equal(*caches)
    assert all(bool(caches[0][:, 0, slot].any()) == (slot in (3, 4, 5, 7)) for slot in range(8))


def test_append_nothing():
    c = Cache("bf16", 1, 8, 1, 64, 2)
    e = torch.empty(0, 1, 64, device="cuda:0", dtype=torch.bfloat16)
    api.paged_append(c.kv, e, e, e, ids([]), ids([[0]]), api.rope_frequencies(64))
    one = torch.ones(1, 1, 64, device="cuda:0", dtype=torch.bfloat16)
    api.paged_append(c.kv, None, one, one, ids([0]), gpu(np.zeros((0, 4), np.int32)), None)
    torch.cuda.synchronize()
    assert torch.isnan(c.k).all()


# ---------------------------------------------------------------- attention
def run_attention(kind, cache_kind, lengths, heads, hk, d, page, seed, window=0, seqs=None,
                  max_keys=None, holes=0, scale=None, with_lse=True, slots_inside=False, gap=0,
                  ws=None, stream=None):
    rng = np.random.default_rng(seed)
    rows = len(lengths)
    seqs = np.arange(rows) if seqs is None else np.asarray(seqs)
    n_seqs = max(1, int(seqs.max()) + 1)
    room = [max([n for n, s in zip(lengths, seqs) if s == i] + [0]) for i in range(n_seqs)]
    table, pages = table_for(rng, room, page)
    c = Cache(cache_kind, pages, page, hk, d, seed, slots_inside, gap)
    for _ in range(holes):
        table[rng.integers(0, n_seqs), rng.integers(0, table.shape[1])] = rng.choice([-1, pages, 1 << 30])
    max_keys = max(max(lengths), 0) if max_keys is None else max_keys
    at = [S.visible(table, pages, page, int(s), n, max_keys, window) for s, n in zip(seqs, lengths)]
    # The window's rows leave what lies before it as NaN.
    stored = c.fill(sorted(set().union(*map(set, at))))
    wide = torch.randn(rows, heads * d + 8, device="cuda:0").to(TYPES[kind])
    q = wide[:, :-8].unflatten(1, (heads, d))
    out = torch.full((rows + 1, heads * d + 16), 7.0, device="cuda:0", dtype=TYPES[kind])
    o = out[:rows, :heads * d].unflatten(1, (heads, d))
    lse = torch.full((rows + 1, heads), 7.0, device="cuda:0") if with_lse else None
    if ws is None:
        ws = torch.zeros(api.paged_attention_workspace_bytes(c.kv, rows, heads, max_keys),
                         dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    call = lambda: api.paged_attention(c.kv, q, ids(table), ids(lengths), o, ws, max_keys,
                                       seqs=ids(seqs), scale=scale, window=window,
                                       lse=None if lse is None else lse[:rows], stream=stream)
    call()
    torch.cuda.synchronize()
    assert not ws[:EMOE_SERVING_TICKET_BYTES].any()
    got, z = f64(o), None if lse is None else f64(lse)
    assert bool((out[rows:] == 7).all()) and bool((out[:, heads * d:] == 7).all())
    assert lse is None or bool((lse[rows:] == 7).all())
    sc = 1 / math.sqrt(d) if scale is None else scale
    rel, tiny = HALF[kind]
    for r in range(rows):
        n = len(at[r])
        k = np.stack([stored[x][0] for x in at[r]]) if n else np.zeros((0, hk, d))
        v = np.stack([stored[x][1] for x in at[r]]) if n else np.zeros((0, hk, d))
        want, want_lse, most, size = S.attend(f64(q)[r], k, v, sc)
        dz = 2 * (d + 4) * U * most
        bound = (2 * dz[:, None] + 2.0 ** -15 + 4 * (n + 64) * U) * size
        check(got[r], want, bound * (1 + rel) + rel * np.abs(want) + tiny, f"row {r} of {n} keys")
        if z is not None:
            limit = dz + (n + 64) * U + 4 * U * np.where(n, np.abs(want_lse), 0) + 2.0 ** -20
            check(z[r], want_lse, limit, f"lse {r}")
    first = o.clone()
    call()
    torch.cuda.synchronize()
    # Equal calls, equal bits (of NaN too: some 8-bit values lie past the largest one).
    assert torch.equal(first.view(torch.int16), o.view(torch.int16))
    return got


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, -3]


@pytest.mark.parametrize("kind,cache_kind", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"),
                                             ("fp16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [8, 16, 32, 256])
def test_attention_lengths(kind, cache_kind, d, page):
    run_attention(kind, cache_kind, EDGES, 4, 2, d, page, seed=d + page)


@pytest.mark.parametrize("heads,hk", [(1, 1), (16, 16), (3, 3), (5, 1), (16, 1), (17, 1), (40, 1),
                                      (28, 4), (21, 3), (64, 2)])
@pytest.mark.parametrize("cache_kind", ["bf16", "e4m3"])
def test_attention_head_layouts(heads, hk, cache_kind):
    run_attention("bf16", cache_kind, [1, 70, 300, 0, 513], heads, hk, 128, 16, seed=heads)


def test_attention_of_more_lines_than_workgroups():
    run_attention("bf16", "bf16", [33, 0, 70], 1200, 600, 64, 8, seed=1)


@pytest.mark.parametrize("lengths,heads,hk,d,page", [
    ([5000], 8, 2, 128, 16), ([4096, 1, 4097], 4, 4, 64, 64), ([20011], 4, 1, 256, 128),
    ([9000, 40, 7, 1200], 12, 2, 128, 8), ([1] * 40 + [3000], 4, 4, 64, 16),
    ([700] * 33, 8, 8, 128, 32), ([33000], 2, 1, 64, 1024)])
@pytest.mark.parametrize("kind,cache_kind", [("bf16", "bf16"), ("fp16", "e4m3")])
def test_attention_long_and_ragged(lengths, heads, hk, d, page, kind, cache_kind):
    run_attention(kind, cache_kind, lengths, heads, hk, d, page, seed=len(lengths))


def ragged(rows, longest):
    return np.random.default_rng(rows).integers(0, longest + 1, rows).tolist()


@pytest.mark.parametrize("lengths,heads,hk,d", [
    ([8000], 8, 1, 128), ([3000, 2500, 1, 3100], 32, 4, 128), ([8000], 16, 1, 64),     # long joins
    ([300], 16, 16, 128), ([900] * 47, 4, 4, 64), (ragged(200, 400), 2, 1, 128),      # an output a workgroup
    (ragged(32, 900), 8, 8, 128), (ragged(64, 400), 8, 8, 64), ([130] * 64, 8, 8, 64),  # a row a worker
    (ragged(31, 900), 8, 8, 128), ([600] * 16, 4, 4, 256), (ragged(16, 1100), 4, 4, 256),
    (ragged(90, 300), 16, 8, 64), (ragged(130, 200), 8, 8, 128), (ragged(300, 64), 4, 4, 256),  # one wavefront
    (ragged(1100, 40), 2, 2, 64), ([64, 1, 33], 40, 2, 128), ([65, 700], 48, 2, 64)])
@pytest.mark.parametrize("kind,cache_kind", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3")])
def test_attention_cuts(lengths, heads, hk, d, kind, cache_kind):
    """Rows whole, in parts of their own and in equal runs, with four and with eight wavefronts."""
    run_attention(kind, cache_kind, lengths, heads, hk, d, 16, seed=len(lengths) + d)


@pytest.mark.parametrize("window", [1, 7, 32, 100, 1000, 1 << 30])
@pytest.mark.parametrize("page", [8, 64])
def test_attention_window(window, page):
    run_attention("bf16", "bf16", [0, 1, 31, 100, 133, 2000, 1025], 4, 2, 128, page, seed=window % 97,
                  window=window)


@pytest.mark.parametrize("page", [8, 16, 32, 128])
@pytest.mark.parametrize("cache_kind", ["fp16", "e4m3"])
def test_attention_missing_pages(page, cache_kind):
    run_attention("fp16", cache_kind, [300, 33, 1, 900, 64, 8], 4, 2, 64, page, seed=page, holes=9)


def test_attention_rows_without_any_page():
    c = Cache("bf16", 3, 16, 2, 64, 0)
    q = torch.randn(3, 4, 64, device="cuda:0").to(torch.bfloat16)
    out, lse = torch.full_like(q, 7), torch.full((3, 4), 7.0, device="cuda:0")
    ws = torch.zeros(api.paged_attention_workspace_bytes(c.kv, 3, 4, 5000), dtype=torch.uint8,
                     device="cuda:0")
    for table in (np.full((3, 400), -1), np.full((3, 400), 3), np.zeros((3, 0)), np.zeros((0, 400))):
        out.fill_(7), lse.fill_(7)
        api.paged_attention(c.kv, q, gpu(table.astype(np.int32)), ids([5000, 1, 40]), out, ws, 5000,
                            lse=lse)
        torch.cuda.synchronize()
        assert not out.any() and bool((lse == -math.inf).all())


def test_attention_many_rows_of_one_sequence():
    """A prompt's rows: each sees its own positions; padding rows between them see none."""
    run_attention("bf16", "bf16", list(range(1, 70)) + [5, 6, 200], 4, 2, 128, 16, seed=3,
                  seqs=[0] * 69 + [-1, 7, 2])


def test_attention_cuts_lengths_to_max_keys_and_table():
    run_attention("bf16", "bf16", [100, 64, 65, 10], 4, 2, 64, 16, seed=4, max_keys=64)
    run_attention("bf16", "bf16", [100, 64], 4, 2, 64, 16, seed=4, max_keys=0)
    run_attention("bf16", "bf16", [100, 64, 3], 4, 2, 64, 16, seed=4, max_keys=1 << 20)
    c = Cache("bf16", 4, 8, 1, 64, 0)
    c.fill([(p, s) for p in range(4) for s in range(8)])
    q = torch.randn(2, 1, 64, device="cuda:0").to(torch.bfloat16)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws = torch.zeros(api.paged_attention_workspace_bytes(c.kv, 2, 1, 1 << 30), dtype=torch.uint8,
                     device="cuda:0")
    t = ids([[0, 1, 2], [3, 2, 1]])
    api.paged_attention(c.kv, q, t, ids([24, 24]), a, ws, 1 << 30)
    api.paged_attention(c.kv, q, t, ids([(1 << 31) - 1, 25]), b, ws, 1 << 30)
    assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 4.0])
def test_attention_scale(scale):
    """Scores up to about +-200 at scale 4: the running maximum moves far."""
    run_attention("bf16", "bf16", [700, 5, 64], 4, 4, 128, 16, seed=9, scale=scale)


@pytest.mark.parametrize("slots_inside,gap", [(True, 0), (False, 16), (True, 64)])
def test_attention_layouts(slots_inside, gap):
    for cache_kind in ("bf16", "e4m3"):
        run_attention("bf16", cache_kind, [77, 300, 16], 6, 3, 64, 16, seed=5,
                      slots_inside=slots_inside, gap=gap, with_lse=False)


def test_attention_without_a_finite_score():
    """As the formula has it: NaN and +inf scores make NaN, keys of -inf scores weigh nothing."""
    c = Cache("fp16", 2, 8, 1, 64, 0)
    c.fill([(0, s) for s in range(8)])
    q = torch.zeros(1, 1, 64, device="cuda:0", dtype=torch.float16)
    q[0, 0, 0] = 1.0
    out, lse = torch.empty_like(q), torch.empty(1, 1, device="cuda:0")
    ws = torch.zeros(api.paged_attention_workspace_bytes(c.kv, 1, 1, 8), dtype=torch.uint8, device="cuda:0")
    c.k[0, :, 0, :] = 0
    c.k[0, 2, 0, 0] = -math.inf
    api.paged_attention(c.kv, q, ids([[0]]), ids([8]), out, ws, 8, lse=lse)
    rest = f64(c.v)[0, [0, 1, 3, 4, 5, 6, 7], 0]
    check(f64(out)[0, 0], rest.mean(0), 2.0 ** -11 * np.abs(rest.mean(0)) + 2.0 ** -14, "-inf")
    assert abs(float(lse) - math.log(7)) < 1e-5
    for bad in (math.inf, math.nan):
        c.k[0, 2, 0, 0] = bad
        api.paged_attention(c.kv, q, ids([[0]]), ids([8]), out, ws, 8, lse=lse)
        assert torch.isnan(out).all()


@pytest.mark.parametrize("n,at", [(6, 2), (128, 127), (700, 300), (3000, 5), (3000, 2999)])
def test_attention_of_infinite_values(n, at):
    """An infinite value that the row sees leaves nothing finite in its own dimension, and
    everything as it is in the others, however the row is split."""
    c = Cache("bf16", 400, 8, 1, 64, 0)
    c.fill([(p, s) for p in range(400) for s in range(8)])
    q = torch.randn(1, 2, 64, device="cuda:0").to(torch.bfloat16)
    out, ok = torch.empty_like(q), torch.empty_like(q)
    ws = torch.zeros(api.paged_attention_workspace_bytes(c.kv, 1, 2, n), dtype=torch.uint8, device="cuda:0")
    args = (q, ids(np.arange(400)[None]), ids([n]))
    api.paged_attention(c.kv, *args, ok, ws, n)
    c.v[at // 8, at % 8, 0, 3], c.v[at // 8, at % 8, 0, 40] = math.inf, -math.inf
    api.paged_attention(c.kv, *args, out, ws, n)
    got = f64(out)[0]
    assert not np.isfinite(got[:, [3, 40]]).any()
    assert np.array_equal(np.delete(got, [3, 40], 1), np.delete(f64(ok)[0], [3, 40], 1))


@pytest.mark.parametrize("rows,longest", [(1025, 40), (1100, 300), (2050, 1)])
def test_attention_more_rows_than_one_launch(rows, longest):
    rng = np.random.default_rng(rows)
    run_attention("bf16", "bf16", rng.integers(0, longest + 1, rows).tolist(), 2, 1, 64, 16, seed=rows)


@pytest.mark.parametrize("n", [5, 128, 3000])
def test_attention_of_nan(n):
    """A query of NaN has NaN outputs, however its row is split; its neighbours do not notice."""
    c = Cache("bf16", 400, 8, 1, 64, 0)
    c.fill([(p, s) for p in range(400) for s in range(8)])
    q = torch.randn(3, 2, 64, device="cuda:0").to(torch.bfloat16)
    out, lse, ok = torch.empty_like(q), torch.empty(3, 2, device="cuda:0"), torch.empty_like(q)
    ws = torch.zeros(api.paged_attention_workspace_bytes(c.kv, 3, 2, n), dtype=torch.uint8, device="cuda:0")
    args = (gpu(np.tile(np.arange(400, dtype=np.int32), (3, 1))), ids([n] * 3))
    api.paged_attention(c.kv, q, *args, ok, ws, n)
    q[1, 0] = math.nan
    api.paged_attention(c.kv, q, *args, out, ws, n, lse=lse)
    assert torch.isnan(out[1, 0]).all() and torch.isnan(lse[1, 0])
    ok[1, 0] = 0
    out[1, 0] = 0
    assert torch.equal(out, ok)


def test_attention_offsets_past_32_bits():
    """A pool above 8 GiB: the pages at its two ends."""
    page, hk, d = 64, 8, 128
    pages = (1 << 33) // (page * hk * d * 2) + 3
    k = torch.empty(pages, page, hk, d, device="cuda:0", dtype=torch.bfloat16)
    v = torch.empty_like(k)
    use = [pages - 1, 0, pages - 2, 1]
    rng = np.random.default_rng(6)
    for t in (k, v):
        t[use] = gpu(rng.standard_normal((4, page, hk, d)).astype(np.float32), torch.bfloat16)
    kv = api.PagedKV(k, v)
    new = torch.randn(1, hk, d, device="cuda:0").to(torch.bfloat16)
    api.paged_append(kv, None, new, new, ids([64 + 63]), ids([[0, pages - 2]]), None)
    assert torch.equal(k[pages - 2, 63], new[0]) and torch.equal(v[pages - 2, 63], new[0])
    q = torch.randn(1, 8, d, device="cuda:0").to(torch.bfloat16)
    out = torch.empty_like(q)
    ws = torch.zeros(api.paged_attention_workspace_bytes(kv, 1, 8, 256), dtype=torch.uint8, device="cuda:0")
    api.paged_attention(kv, q, ids([use]), ids([250]), out, ws, 256)
    kk, vv = (f64(t[use]).reshape(-1, hk, d)[:250] for t in (k, v))
    want, _, most, size = S.attend(f64(q)[0], kk, vv, d ** -0.5)
    bound = (4 * (d + 4) * U * most[:, None] + 2.0 ** -15 + 4 * 314 * U) * size
    check(f64(out)[0], want, bound * 1.01 + 2.0 ** -8 * np.abs(want), "far pages")


# ---------------------------------------------------------------- logits
def logits_case(kind, rows, vocab, width, seed, biases=0, mask=None, alone=True, stride=0):
    """Random inputs of process_logits as (device arguments, per-row oracle arguments)."""
    rng = np.random.default_rng(seed)
    x = torch.randn(rows, vocab + stride, device="cuda:0").mul(4).to(TYPES[kind])[:, :vocab]
    dev, rows_of = dict(logits=x), [dict(x=f64(x)[r]) for r in range(rows)]
    if width:
        h = (rng.zipf(1.3, (rows, width)) * 31 % (vocab + 3)) - 2    # a few outside
        n, p = rng.integers(-1, width + 2, rows), rng.integers(-1, width + 2, rows)
        f = [(1 + rng.random(rows)).astype(np.float32), rng.random(rows).astype(np.float32),
             rng.normal(0, 0.5, rows).astype(np.float32)]
        f[0][0], f[1][0], f[2][0] = 1.0, 0.0, 0.0                    # a row without penalties
        dev |= dict(history=ids(h), history_lengths=ids(n), prompt_lengths=ids(p),
                    repetition=gpu(f[0]), presence=gpu(f[1]), frequency=gpu(f[2]))
        for r, a in enumerate(rows_of):
            a |= dict(history=h[r, :max(0, min(width, n[r]))].tolist(), prompt=p[r],
                      repetition=float(f[0][r]), presence=float(f[1][r]), frequency=float(f[2][r]))
    if biases:
        i = rng.integers(-2, vocab + 2, (rows, biases))
        b = rng.normal(0, 3, (rows, biases)).astype(np.float32)
        n = rng.integers(-1, biases + 2, rows)
        dev |= dict(bias_ids=ids(i), bias_values=gpu(b), bias_counts=ids(n))
        for r, a in enumerate(rows_of):
            m = max(0, min(biases, n[r]))
            a["biases"] = list(zip(i[r, :m].tolist(), b[r, :m].astype(np.float64)))
    if mask is not None:
        words = -(-vocab // 32)
        m = rng.integers(0, 2 ** 32, (max(rows, 3), words), dtype=np.uint32)
        m[-1] = 0
        dev["mask"] = gpu(m.view(np.int32))
        which = np.arange(rows)
        if mask == "rows":
            which = rng.integers(-1, len(m) + 1, rows)
            which[0] = len(m) - 1                                    # nothing allowed
            dev["mask_rows"] = ids(which)
        for r, a in enumerate(rows_of):
            if 0 <= which[r] < len(m):
                a["mask"] = m[which[r]].tolist()
    return dev, rows_of


def check_logits(kind, got, token, rows_of):
    rel, tiny = HALF[kind]
    for r, a in enumerate(rows_of):
        want, t, size = S.process_logits(**a)
        finite = np.isfinite(want)
        check(got[r], want, 6 * U * size * (1 + rel) + np.where(finite, rel * np.abs(want), 0) + tiny, r)
        if token is None:
            continue
        if t < 0:
            assert token[r] == -1
        else:
            # The same token, unless two are as near as the roundings.
            assert token[r] == t or want[token[r]] >= want[t] - 12 * U * max(size[t], size[token[r]]) > -np.inf
            if want[token[r]] == want[t]:
                assert token[r] == t


def run_logits(kind, rows, vocab, width, seed, in_place=False, token=True, **kw):
    dev, rows_of = logits_case(kind, rows, vocab, width, seed, **kw)
    out = dev["logits"] if in_place else torch.full((rows + 1, vocab + 3), 7.0, device="cuda:0",
                                                    dtype=TYPES[kind])[:, :vocab]
    nt = torch.full((rows + 1,), 77, dtype=torch.int32, device="cuda:0") if token else None
    ws = torch.zeros(api.process_logits_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda:0")
    api.process_logits(out=None if in_place else out[:rows], workspace=ws if token else None,
                       next_token=None if nt is None else nt[:rows], **dev)
    torch.cuda.synchronize()
    assert not ws.any()
    if not in_place:
        assert bool((out[rows:] == 7).all())
        whole = out._base if out._base is not None else out
        assert bool((whole[:, vocab:] == 7).all())
    assert nt is None or int(nt[rows]) == 77
    check_logits(kind, f64(out[:rows]), None if nt is None else nt.tolist(), rows_of)


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 33, 1000, 1023, 1025, 4097, 9999])
def test_logits(kind, vocab):
    run_logits(kind, 5, vocab, 50, seed=vocab, biases=9, mask="rows")


@pytest.mark.parametrize("kind", ["f32", "bf16", "fp16"])
@pytest.mark.parametrize("opts", [dict(width=0), dict(width=1), dict(width=3001),
                                  dict(width=6143), dict(width=6144, biases=3),
                                  dict(width=0, biases=300), dict(width=0, mask="own"),
                                  dict(width=40, in_place=True, biases=3, mask="own"),
                                  dict(width=40, token=False), dict(width=40, stride=5)])
def test_logits_parts(kind, opts):
    run_logits(kind, 4, 3001, seed=opts["width"] + 1, **opts)


@pytest.mark.parametrize("kind,rows,vocab", [("f32", 200, 12001), ("bf16", 150, 32771),
                                             ("fp16", 1, 50304), ("fp16", 90, 50021),
                                             ("f32", 3, 200001)])
def test_logits_large(kind, rows, vocab):
    run_logits(kind, rows, vocab, 300, seed=rows, biases=20, mask="rows")


def test_logits_more_rows_than_one_launch():
    rows, vocab = 4096 + 300, 1500
    x = torch.randn(rows, vocab, device="cuda:0")
    nt = torch.empty(rows, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(api.process_logits_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda:0")
    out = torch.empty_like(x)
    api.process_logits(x, out, ws, next_token=nt)
    assert torch.equal(out, x) and torch.equal(nt.long(), x.argmax(1))


def test_logits_of_two_streams_at_once():
    """Calls with their own workspaces, each with more rows of two chunks than the device holds
    workgroups: a row's workgroups wait for none that has no place yet."""
    rows, vocab = 4096, 8000
    jobs = []
    for i in range(2):
        x = torch.randn(rows, vocab, device="cuda:0")
        nt = torch.empty(rows, dtype=torch.int32, device="cuda:0")
        ws = torch.zeros(api.process_logits_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda:0")
        jobs.append((x, torch.empty_like(x), ws, nt, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for turn in range(3):
        for x, out, ws, nt, stream in jobs:
            api.process_logits(x, out, ws, next_token=nt, stream=stream)
        torch.cuda.synchronize()
        for x, out, ws, nt, _ in jobs:
            assert torch.equal(out, x) and torch.equal(nt.long(), x.argmax(1)) and not ws.any()
            nt.fill_(-7)
            out.zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("rows,vocab", [(1, 1 << 30), (5, (1 << 29) + 1)])
def test_logits_offsets_past_32_bits(rows, vocab):
    x = torch.zeros(rows, vocab, device="cuda:0", dtype=torch.bfloat16)
    at = [(vocab - 1 - 12345 * r) % vocab for r in range(rows)]
    for r, v in enumerate(at):
        x[r, v] = 2.0 + r
    h = ids([[v, v // 2] for v in at])
    nt = torch.empty(rows, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(api.process_logits_workspace_bytes(rows, vocab), dtype=torch.uint8, device="cuda:0")
    two, quarter = (torch.full((rows,), s, device="cuda:0") for s in (2.0, 0.25))
    api.process_logits(x, workspace=ws, next_token=nt, history=h, repetition=two, presence=quarter)
    assert nt.tolist() == at and not ws.any()
    for r, v in enumerate(at):
        assert float(x[r, v]) == (2 + r) / 2 - 0.25 and float(x[r, v // 2]) == -0.25
    assert sum(int(x[r].count_nonzero()) for r in range(rows)) == 2 * rows


def test_logits_special_values():
    """Ties to the lower id (also -0 with +0), NaN never chosen, infinities as they come."""
    V = 5000
    rows = [torch.full((V,), -1.0) for _ in range(7)]
    rows[0][[4321, 17, 4999]] = 2.0
    rows[1][:] = -math.inf
    rows[2][:] = math.nan
    rows[3][[5, 4000]] = math.inf
    rows[4][:] = math.nan
    rows[4][4998] = -3.0e38
    rows[5][3], rows[5][2000] = -0.0, 0.0
    rows[6][:] = -3.4028234663852886e38                              # the type's lowest value
    x = torch.stack(rows).to("cuda:0")
    nt = torch.empty(7, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(api.process_logits_workspace_bytes(7, V), dtype=torch.uint8, device="cuda:0")
    out = torch.empty_like(x)
    api.process_logits(x, out, ws, next_token=nt)
    assert nt.tolist() == [17, -1, -1, 5, 4998, 3, 0]
    assert torch.equal(out.view(torch.int32), x.view(torch.int32))


def test_logits_choice_comes_before_the_store():
    """Two bf16 neighbours that a penalty makes equal only once they are rounded."""
    x = torch.full((1, 64), -9.0, device="cuda:0").to(torch.bfloat16)
    x[0, 3], x[0, 9] = 4.0, 4.03125
    nt = torch.empty(1, dtype=torch.int32, device="cuda:0")
    ws = torch.zeros(api.process_logits_workspace_bytes(1, 64), dtype=torch.uint8, device="cuda:0")
    out = torch.empty_like(x)
    api.process_logits(x, out, ws, bias_ids=ids([[9]]), bias_values=gpu([[-0.03]]), next_token=nt)
    assert float(out[0, 3]) == float(out[0, 9]) == 4.0 and int(nt) == 9


# ---------------------------------------------------------------- together, streams, graphs
class Step:
    """One layer's part of a decode step over static buffers: append, attend, logits."""

    def __init__(self, seed, rows=5, heads=8, hk=2, d=64, page=16, vocab=2003):
        g = torch.Generator(device="cuda:0").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, device="cuda:0", generator=g)
        rng = np.random.default_rng(seed)
        self.at = rng.integers(0, 900, rows)
        table, pages = table_for(rng, self.at + 1, page)
        self.k, self.v = (rand(pages, page, hk, d).to(torch.bfloat16) for _ in range(2))
        self.kv = api.PagedKV(self.k, self.v)
        self.table, self.pos, self.n = ids(table), ids(self.at), ids(self.at + 1)
        self.q, self.qr = (rand(rows, heads, d).to(torch.bfloat16) for _ in range(2))
        self.new_k, self.new_v = (rand(rows, hk, d).to(torch.bfloat16) for _ in range(2))
        self.freq = api.rope_frequencies(d)
        self.out = torch.empty_like(self.q)
        self.head = rand(heads * d, vocab).to(torch.bfloat16)
        self.x = torch.empty(rows, vocab, device="cuda:0", dtype=torch.bfloat16)
        self.hist = ids(rng.integers(0, vocab, (rows, 64)))
        self.rep = gpu((1 + rng.random(rows)).astype(np.float32))
        self.next = torch.empty(rows, dtype=torch.int32, device="cuda:0")
        zeros = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda:0")
        self.ws = zeros(api.paged_attention_workspace_bytes(self.kv, rows, heads, 1024))
        self.logits_ws = zeros(api.process_logits_workspace_bytes(rows, vocab))

    def run(self, stream=None):
        api.paged_append(self.kv, self.q, self.new_k, self.new_v, self.pos, self.table, self.freq,
                         q_out=self.qr, stream=stream)
        api.paged_attention(self.kv, self.qr, self.table, self.n, self.out, self.ws, 1024, stream=stream)

    def finish(self, stream=None):
        api.process_logits(self.x, self.x, self.logits_ws, history=self.hist, repetition=self.rep,
                           next_token=self.next, stream=stream)

    def all(self):
        self.run()
        torch.mm(self.out.flatten(1), self.head, out=self.x)
        self.finish()
        return self.out.clone(), self.x.clone(), self.next.clone()


def test_step_against_the_oracle():
    s = Step(11)
    k0, v0 = f64(s.k), f64(s.v)
    out, x, token = s.all()
    torch.cuda.synchronize()
    table, freq = s.table.cpu().numpy(), f64(s.freq)
    hist, rep = s.hist.tolist(), s.rep.tolist()
    raw = f64(torch.mm(out.flatten(1), s.head))
    for r, p in enumerate(s.at):
        q = np.stack([S.rotate(h, p, freq, False) for h in f64(s.q)[r]])
        at = S.visible(table, len(k0), 16, r, p + 1, 1024, 0)
        k = np.stack([k0[a] for a in at[:-1]] + [np.stack([S.rotate(h, p, freq, False) for h in f64(s.new_k)[r]])])
        v = np.stack([v0[a] for a in at[:-1]] + [f64(s.new_v)[r]])
        want, _, most, size = S.attend(q, k, v, 64 ** -0.5)
        # Rounded queries and the rounded last key move every score by two halves.
        dz = (2 * 2.0 ** -8 + 2 * 68 * U) * most[:, None]
        check(f64(out)[r], want, (2 * dz + 2.0 ** -15 + 4 * 1088 * U) * size * 1.01 + 2.0 ** -8 * np.abs(want), r)
        want, t, size = S.process_logits(raw[r], hist[r], 0, rep[r])
        check(f64(x)[r], want, 2.0 ** -8 * np.abs(want) + 6 * U * size, r)
        assert int(token[r]) == t or want[int(token[r])] == want[t]


def test_two_graphs_share_a_workspace():
    """Captured calls of different sizes over one workspace of each kind, replayed in turn with
    eager ones."""
    a, b = Step(1), Step(2, rows=9, heads=4, hk=4, vocab=5000)
    for name in ("ws", "logits_ws"):
        larger = max((getattr(a, name), getattr(b, name)), key=lambda t: t.numel())
        setattr(a, name, larger), setattr(b, name, larger)
    want = [[t.clone() for t in s.all()[:2:2]] + [s.next.clone()] for s in (a, b)]
    raw = [torch.mm(s.out.flatten(1), s.head) for s in (a, b)]
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                s.run()
                s.finish()
        graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(4):
        for i, s in enumerate((a, b)):
            s.out.fill_(7), s.x.copy_(raw[i]), s.next.fill_(-5)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(s.out, want[i][0]) and torch.equal(s.next, want[i][-1]), (turn, i)
        assert not a.ws[:EMOE_SERVING_TICKET_BYTES].any() and not a.logits_ws.any()
        a.all()


def test_two_streams_with_their_own_workspaces():
    steps = [Step(3 + i) for i in range(2)]
    want = [s.all() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for turn in range(3):
        for s, st in zip(steps, streams):
            s.run(stream=st)
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            assert torch.equal(s.out, w[0])


def test_two_threads_call_at_once():
    """Each with tensors, workspaces and a stream of its own."""
    steps = [Step(7 + i) for i in range(4)]
    want = [[t.clone() for t in s.all()] for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]

    def work(i):
        for _ in range(50):
            steps[i].run(stream=streams[i])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert torch.equal(s.out, w[0])


def test_binding_checks_tensors():
    c = Cache("bf16", 2, 16, 2, 64, 0)
    q = torch.zeros(2, 4, 64, device="cuda:0", dtype=torch.bfloat16)
    k = torch.zeros(2, 2, 64, device="cuda:0", dtype=torch.bfloat16)
    t, p = ids([[0], [1]]), ids([0, 0])
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda:0")
    ok = dict(kv=c.kv, q=q, page_table=t, lengths=p, out=torch.zeros_like(q), workspace=ws, max_keys=16)
    api.paged_attention(**ok)
    bad = [dict(q=q.half()), dict(q=q.cpu()), dict(q=q[:, :, :32]), dict(out=q[:1]),
           dict(out=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(lengths=p.long()),
           dict(lengths=p[:1]), dict(page_table=t.float()), dict(page_table=t[0]),
           dict(workspace=ws[:100]), dict(workspace=ws.cpu()), dict(lse=torch.zeros(2, 4)),
           dict(lse=torch.zeros(2, 5, device="cuda:0")), dict(seqs=p.cpu())]
    for change in bad:
        with pytest.raises(ExactMoEError) as e:
            api.paged_attention(**{**ok, **change})
        assert e.value.status == EMOE_EINVAL, change
    ok = dict(kv=c.kv, q=q, k=k, v=k, positions=p, page_table=t, inv_freq=api.rope_frequencies(64))
    api.paged_append(**ok)
    for change in (dict(k=k.half()), dict(v=k[:1]), dict(v=k[:, :1]), dict(positions=p.float()),
                   dict(inv_freq=torch.zeros(32, device="cuda:0")), dict(q_out=q.float()),
                   dict(interleaved=np.zeros(2))):
        with pytest.raises(ExactMoEError):
            api.paged_append(**{**ok, **change})
    x = torch.zeros(2, 100, device="cuda:0")
    for change in (dict(out=x.half()), dict(out=x[:, :99]), dict(history=p), dict(presence=p),
                   dict(mask=ids(np.zeros((2, 3)))), dict(next_token=p.long()),
                   dict(bias_ids=ids(np.zeros((2, 2))), bias_values=torch.zeros(2, 3, device="cuda:0"))):
        with pytest.raises(ExactMoEError):
            api.process_logits(**{**dict(logits=x, workspace=ws), **change})
    for kp, vp, more in ((c.k, c.v.half(), ()), (c.k, c.v[:1], ()), (c.k.float(), c.v.float(), ()),
                         (c.k, c.v, (torch.ones(2, device="cuda:0"),) * 2), (c.k[0], c.v[0], ())):
        with pytest.raises(ExactMoEError):
            api.PagedKV(kp, vp, *more)
