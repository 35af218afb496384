"""The paged attention's softmax weights, small ones among them, against 64 bits.

Scores here are single products or small whole numbers, so that what remains is,
with u = 2^-24 (the rounding of an fp32 operation):
  scores      the scale, its log2 e and a key scale: 4 u |z| =: dz;
  weights     2 dz + 2^-15 of each (both exponents, exp2 itself, its two 16-bit halves);
  sums        no more than 1,024 additions one after another, of the products and of the
              weights: a wavefront takes at most 4 tiles of 32 keys of these rows (256
              workgroups of 4 wavefronts at 256 dimensions, else of 8), with 6 products per
              key at most (two halves in up to three turns); then the wavefronts' and the
              workgroups' parts are joined;
  the store   half a step.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_15383_amd import api
from tests.test_gpu_serving import HALF, TYPES, U, check, f64, gpu, ids, ragged, run_attention

pytestmark = pytest.mark.gpu

SUMS = 2 * 1024 * U
KINDS = [("fp16", "fp16"), ("fp16", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")]


def shuffled_cache(cache_kind, k, v, page, ks=None, vs=None, seed=0):
    """A cache that holds k and v [keys][kv heads][dim] as one sequence, NaN elsewhere."""
    n, hk, d = k.shape
    need = -(-n // page)
    table = np.random.default_rng(seed).permutation(need + 2)[:need].astype(np.int32)
    pages = []
    for x in (k, v):
        whole = torch.full((need * page, hk, d), math.nan, device="cuda:0")
        whole[:n] = x
        raw = torch.full((need + 2, page, hk, d), math.nan, device="cuda:0").to(TYPES[cache_kind])
        bits = torch.uint8 if cache_kind == "e4m3" else torch.int16
        raw.view(bits)[gpu(table).long()] = whole.to(raw.dtype).view(bits).view(need, page, hk, d)
        pages.append(raw)
    return api.PagedKV(*pages, ks, vs), gpu(table[None])


def attend(kv, table, q, lengths, max_keys=None, seqs=None, scale=1.0, window=0):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda:0")
    max_keys = max(lengths) if max_keys is None else max_keys
    ws = torch.zeros(api.paged_attention_workspace_bytes(kv, *q.shape[:2], max_keys), dtype=torch.uint8,
                     device="cuda:0")
    api.paged_attention(kv, q, table, ids(lengths), out, ws, max_keys, seqs=seqs, scale=scale,
                        window=window, lse=lse)
    torch.cuda.synchronize()
    return f64(out), f64(lse)


def check_weights(kind, got, lse, z, v):
    """One row: z [heads][keys], v [keys][dim] (of one key head)."""
    rel, tiny = HALF[kind]
    for h in range(len(z)):
        w = np.exp(z[h] - z[h].max())
        want_lse = z[h].max() + math.log(w.sum())
        w /= w.sum()
        want, size = w @ v, w @ np.abs(v)
        dz = 4 * U * np.abs(z[h]).max()
        bound = (2 * dz + 2.0 ** -15 + SUMS) * size
        check(got[h], want, bound * (1 + rel) + rel * np.abs(want) + tiny, ("head", h))
        check(lse[h:h + 1], want_lse, dz + SUMS + 4 * U * abs(want_lse) + 2.0 ** -18, ("lse", h))


def sinks(n, where):
    return {"first": [0], "last": [n - 1], "tiles": list(range(5, n, 32)),
            "some": np.random.default_rng(n).integers(0, n, 7).tolist()}[where]


@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("n,d,where,size", [
    (131_073, 128, "first", 1.0), (131_073, 64, "last", 1.0), (120_000, 256, "some", 1.0),
    (4096, 128, "tiles", 256.0), (500, 64, "tiles", 256.0), (64, 128, "last", 256.0),
    (33, 256, "first", 256.0)])
def test_weights_far_below_the_largest(kind, cache_kind, n, d, where, size):
    """Keys of value 0 draw nearly all of the weight; the others, up to 30 nats below them, are all
    that the output is made of.  A second head sees no difference, a third the reverse."""
    for gap in (0.0, 9.0, 12.0, 14.0, 16.0, 17.0, 17.375, 18.0, 22.0, 30.0):
        at = sinks(n, where)
        k, v = torch.zeros(n, 1, d, device="cuda:0"), torch.empty(n, 1, d, device="cuda:0")
        k[at, 0, 0] = 1.0
        # Values that the types hold, with as many bits as they have.
        step = {"fp16": 1 + 2.0 ** -10, "bf16": 1 + 2.0 ** -7, "e4m3": 1.125}[cache_kind]
        v[:] = size * torch.tensor([1.0, step, -1.0, 0.5 * step], device="cuda:0").repeat(d // 4)
        v[at] = 0.0
        one = torch.ones(1, device="cuda:0") if cache_kind == "e4m3" else None
        kv, table = shuffled_cache(cache_kind, k, v, 64, one, one)
        q = torch.zeros(1, 3, d, device="cuda:0")
        q[0, 0, 0], q[0, 2, 0] = gap, -gap
        q = q.to(TYPES[kind])
        got, lse = attend(kv, table, q, [n])
        z = f64(q)[0] @ f64(k)[:, 0].T
        check_weights(kind, got[0], lse[0], z, f64(v)[:, 0])


@pytest.mark.parametrize("cache_kind", ["fp16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("scale", [1.0, 4.0, -0.3, 0.0])
def test_scores_far_apart(cache_kind, d, scale):
    """Random scores of up to +-200: large and small weights in one tile, in tiles that a row, a
    window or a missing page cuts, and a maximum that moves far."""
    for lengths, more in (([700, 5, 64, 0, 3001], {}), (ragged(70, 500), dict(holes=30)),
                          ([1000, 33, 2050], dict(window=300)), (ragged(300, 64), {})):
        run_attention("fp16", cache_kind, lengths, 4, 2, d, 16, seed=d, scale=scale, **more)


@pytest.mark.parametrize("gap", [33.0, 38.0, 43.0, 60.0])
def test_weights_of_large_values(gap):
    """fp16 weights of 2^-47 to 2^-86 of the largest, times the type's largest values: what of them
    still shows in fp16."""
    n, d = 131_073, 64
    k, v = torch.zeros(n, 1, d, device="cuda:0"), torch.full((n, 1, d), 65504.0, device="cuda:0")
    k[1000, 0, 0], v[1000] = 1.0, 0.0
    v[2000:, 0, 1] = -60000.0
    kv, table = shuffled_cache("fp16", k, v, 32)
    q = torch.zeros(1, 2, d, device="cuda:0").half()
    q[0, 0, 0], q[0, 1, 0] = gap, 5.0
    got, lse = attend(kv, table, q, [n])
    check_weights("fp16", got[0], lse[0], f64(q)[0] @ f64(k)[:, 0].T, f64(v)[:, 0])
    # 131,072 times 65,504 times e^-gap reaches half of the smallest value up to 40.2 nats.
    assert got[0].any(1).tolist() == [gap < 40.2, True]


@pytest.mark.parametrize("cache_kind", ["fp16", "e4m3"])
def test_one_key_gives_back_its_value(cache_kind):
    """Every finite value of the type, its subnormal ones too, as the only key of a row."""
    if cache_kind == "fp16":
        v = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.float16)
    else:
        v = torch.arange(256, dtype=torch.uint8).repeat(4).view(torch.float8_e4m3fn)
    v = v.reshape(-1, 1, 1, 64).to("cuda:0")
    rows = v.shape[0]
    pages = torch.zeros(rows, 8, 1, 64, device="cuda:0", dtype=v.dtype)
    pages.view(torch.uint8)[:, :1] = v.view(torch.uint8)
    kv = api.PagedKV(torch.zeros_like(pages), pages)
    q = torch.randn(rows, 2, 64, device="cuda:0").half()
    got, lse = attend(kv, ids(np.arange(rows)[:, None]), q, [1] * rows)
    want = np.repeat(f64(v.float())[:, 0], 2, 1)
    finite = np.isfinite(want)
    assert np.array_equal(got[finite], want[finite]) and not np.isfinite(got[~finite]).any()
    assert not lse.any()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_subnormal_keys_count(d):
    """fp16 keys of 2^-20 under large queries: scores of several nats."""
    k = torch.zeros(40, 1, d, device="cuda:0")
    k[7], k[20] = 2.0 ** -20, -(2.0 ** -24)
    v = torch.zeros_like(k)
    v[7], v[20], v[33] = 1.0, 2.0, -1.5
    kv, table = shuffled_cache("fp16", k, v, 8)
    q = torch.full((1, 2, d), 30000.0 * 64 / d, device="cuda:0").half()
    got, lse = attend(kv, table, q, [40])
    check_weights("fp16", got[0], lse[0], f64(q)[0] @ f64(k)[:, 0].T, f64(v)[:, 0])
