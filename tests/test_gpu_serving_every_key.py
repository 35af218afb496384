"""The paged attention sees every key of a row once and no other, at lengths where one
tile more or less is far below what rounding allows random values.

Equal weights: queries of 0 over any keys make every weight the same power of two, and
values of 0 and 1 say which tile of 32 keys a key is of: in even key heads tile t has
its ones in dimension t % d, in odd ones in dimension t // ceil(tiles / d).  All sums are
whole numbers below 2^24, so the output is their exact quotient but for two fp32
roundings and the store, and a tile lost, doubled or taken for another one changes a
dimension by 1 part in 33 or more.  The log-sum-exp is the logarithm of the number of
keys: log2 to an ulp below 2^-19, two fp32 roundings; one key of 131,072 is 2^-17.

Needles: keys of +-1 and a query that equals one of them at a scale of 1 leave all
other keys together a weight below 2^-20, which is checked; the output is that key's
value.  Weights are known to 2^-15, sums (of one weight) to 2^-18.
"""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_serving import HALF, TYPES, U, check, f64, ids, ragged
from tests.test_gpu_serving_weights import attend, shuffled_cache

pytestmark = pytest.mark.gpu

TILE = 32
KINDS = [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "e4m3"), ("fp16", "e4m3")]
# lengths, heads, key heads, dimensions, page, window
CASES = [
    ([131_072], 32, 8, 128, 64, 0), ([131_072], 2, 1, 64, 1024, 0), ([70_001], 4, 4, 256, 16, 0),
    ([33_000, 5, 20_011, 1], 8, 2, 128, 8, 0), ([9000, 9000], 40, 2, 64, 32, 0),
    (ragged(32, 2000), 32, 8, 128, 16, 0), (ragged(31, 900), 8, 8, 64, 64, 0),
    (ragged(16, 3000), 8, 4, 256, 128, 0), (ragged(47, 6000), 16, 4, 64, 16, 1024),
    (ragged(90, 4000), 8, 8, 128, 32, 0), (ragged(300, 60), 8, 8, 128, 8, 0),
    (ragged(1100, 300), 8, 4, 64, 16, 0), ([40_000] * 3, 8, 2, 128, 64, 30_007)]


def one_sequence(kind, cache_kind, k, v, page):
    one = torch.ones(k.shape[1], device="cuda:0") if cache_kind == "e4m3" else None
    return shuffled_cache(cache_kind, k, v, page, one, one, seed=k.shape[0])


def spans(lengths, window):
    return [(max(0, n - window) if window else 0, n) for n in lengths]


@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("lengths,heads,hk,d,page,window", CASES)
def test_equal_weights(kind, cache_kind, lengths, heads, hk, d, page, window):
    n, rows, group = max(lengths), len(lengths), heads // hk
    tile = torch.arange(n, device="cuda:0") // TILE
    tiles = -(-n // TILE)
    dims = [tile % d, tile // -(-tiles // d)]
    v = torch.zeros(n, hk, d, device="cuda:0")
    for g in range(hk):
        v[torch.arange(n, device="cuda:0"), g, dims[g % 2]] = 1.0
    kv, table = one_sequence(kind, cache_kind, torch.randn(n, hk, d, device="cuda:0"), v, page)
    q = torch.zeros(rows, heads, d, device="cuda:0", dtype=TYPES[kind])
    got, lse = attend(kv, table, q, lengths, seqs=ids([0] * rows), scale=1.0, window=window)
    rel, tiny = HALF[kind]
    where = [x.cpu().numpy() for x in dims]
    for r, (first, last) in enumerate(spans(lengths, window)):
        keys = last - first
        for g in range(hk):
            count = np.bincount(where[g % 2][first:last], minlength=d)
            want = np.broadcast_to(count / max(1, keys), (group, d))
            bound = (rel + 3 * U) * want + tiny
            check(got[r, g * group:(g + 1) * group], want, bound, ("row", r, "key head", g))
            # A whole tile less would show.
            full = count[count >= TILE]
            if kind == "fp16" or keys > 64 * TILE:
                assert (TILE / np.maximum(full, 1) * 0.9 > 2 * (rel + 3 * U)).all()
        want_lse = math.log(keys) if keys else -math.inf
        check(lse[r], want_lse, 2.0 ** -18, ("lse", r))


def needles(first, last, count, seed):
    """Positions in [first, last): its ends, both sides of tiles, pages and runs, and others."""
    edges = [first, first + 1, last - 1, last - 2]
    for at in (8, 32, 64, 128, 256, 1024, 2048, (first + last) // 2 // TILE * TILE):
        edges += [at - 1, at, last // at * at - 1, last // at * at] if at else []
    rng = np.random.default_rng(seed)
    edges = [p for p in dict.fromkeys(edges) if first <= p < last]
    rng.shuffle(edges)
    return (edges + rng.integers(first, last, count).tolist())[:count]


@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("lengths,heads,hk,d,page,window", CASES)
def test_needles(kind, cache_kind, lengths, heads, hk, d, page, window):
    lengths = [max(1, x) for x in lengths]
    n, rows, group = max(lengths), len(lengths), heads // hk
    gen = torch.Generator(device="cuda:0").manual_seed(n)
    k = torch.randint(0, 2, (n, hk, d), device="cuda:0", generator=gen, dtype=torch.int8).float() * 2 - 1
    v = torch.randn(n, hk, d, device="cuda:0", generator=gen).to(TYPES[cache_kind]).float()
    kv, table = one_sequence(kind, cache_kind, k, v, page)
    at = torch.tensor([needles(first, last, heads, r) for r, (first, last) in
                       enumerate(spans(lengths, window))], device="cuda:0")        # [rows][heads]
    head = torch.arange(heads, device="cuda:0") // group
    q = k[at, head]
    # The scores are whole numbers: exact in fp32, by any library's product.
    others, spread = torch.zeros(rows, heads, device="cuda:0"), torch.arange(n, device="cuda:0")
    span = torch.tensor(spans(lengths, window), device="cuda:0")
    seen = (spread >= span[:, :1]) & (spread < span[:, 1:])                        # [rows][n]
    for h in range(heads):
        z = torch.mm(q[:, h], k[:, h // group].t().contiguous()) - d               # [rows][n], 0 at the needle
        w = torch.exp(z.double()) * seen
        w[torch.arange(rows, device="cuda:0"), at[:, h]] = 0
        others[:, h] = w.sum(1)
    assert float(others.max()) < 2.0 ** -20
    got, lse = attend(kv, table, q.to(TYPES[kind]), lengths, seqs=ids([0] * rows), scale=1.0, window=window)
    want = f64(v[at, head])
    rel, tiny = HALF[kind]
    bound = (2.0 ** -15 + 2.0 ** -18) * np.abs(want) + 2.0 ** -20 * 2 * float(v.abs().max())
    check(got, want, bound * (1 + rel) + rel * np.abs(want) + tiny, "values")
    check(lse, float(d), 2.0 ** -20 + 4 * U * d + 2.0 ** -18, "lse")
