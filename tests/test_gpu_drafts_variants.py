"""The tree attention's kernels at both numbers of columns (query heads of a key head, of
all nodes that a tree may have): up to 16, or 32 of 64 dimensions, wavefronts take keys
of their own, with more they share them.  Against the same oracle and with the same
tolerances as in tests/test_gpu_drafts.py.
"""
import math

import numpy as np
import pytest
import torch

from oracle import drafts_oracle as O
from paper_2608_15383_amd import api
from tests.test_gpu_drafts import KINDS, bits64, run_tree
from tests.test_gpu_serving import Cache, ids

pytestmark = pytest.mark.gpu

# Three query heads to a key head: 15, 30 and 60 columns.  30 are the second tile of the
# first kernel at 64 dimensions.
COLUMNS = [(d, most) for d in (64, 128, 256) for most in (5, 20)] + [(64, 10)]


def cut(most, nodes):
    return [min(n, most) for n in nodes]


@pytest.mark.parametrize("cap,slopes,window", [(30.0, False, 0), (0.0, True, 0), (5.0, True, 50),
                                               (0.5, False, 7)])
@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("d,most", COLUMNS)
def test_shaped_scores(cap, slopes, window, kind, cache_kind, d, most):
    run_tree(kind, cache_kind, [0, 70, 333, 1500], cut(most, [9, 5, 20, 3]), 6, 2, d, 16, seed=4,
             window=window, cap=cap, slopes=slopes, scale=1.0 if cap else None)


@pytest.mark.parametrize("window", [1, 7, 33, 100, 601, 1000, 2500, (1 << 31) - 1])
@pytest.mark.parametrize("d,most", COLUMNS)
def test_windows(window, d, most):
    """Among them such as have their keys cut over workers from a first key that no unit begins with."""
    lengths = [0, 1, 31, 133, 2000, 1025, 3333, 2999]
    run_tree("bf16", "e4m3" if window == 601 else "bf16", lengths, cut(most, [9, 2, 3, 1, 20, 5, 4, 2]), 6, 2,
             d, 64, seed=window % 97, window=window)


@pytest.mark.parametrize("page", [8, 128])
@pytest.mark.parametrize("kind,cache_kind", KINDS)
@pytest.mark.parametrize("d,most", COLUMNS)
def test_missing_pages(page, kind, cache_kind, d, most):
    run_tree(kind, cache_kind, [300, 33, 1, 900, 64, 8], cut(most, [6, 9, 20, 3, 1, 8]), 6, 2, d, page,
             seed=page, holes=9)


@pytest.mark.parametrize("slots_inside,gap", [(True, 0), (False, 64), (True, 16)])
@pytest.mark.parametrize("cache_kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,most", COLUMNS)
def test_layouts(slots_inside, gap, cache_kind, d, most):
    run_tree("bf16", cache_kind, [70, 0, 200, 1200], cut(most, [5, 20, 2, 9]), 6, 2, d, 16, seed=gap,
             slots_inside=slots_inside, gap=gap)


@pytest.mark.parametrize("at", [5, 70, 103])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("d,most", COLUMNS)
def test_infinite_value_in_one_dimension(at, kind, d, most):
    """Of a key that all nodes see, whose tile has nothing masked, or of a node: its own dimension
    is infinite or NaN for those that see it, the others are as without it."""
    def poison(c, stored):                       # one page: a slot is its position
        c.v[:, at, 0, 5] = math.inf
        for (p, s), (_, v) in stored.items():
            if s == at:
                v[0, 5] = math.inf

    got = run_tree(kind, kind, [100], [most], 3, 1, d, 128, seed=6, poison=poison)
    assert np.isinf(got[:, :, 5]).any() and np.isfinite(got[:, :, 6:]).all()


@pytest.mark.parametrize("most", [4, 40])
def test_rows_of_no_tree_stay(most):
    """starts that hold more nodes than max_nodes: the first max_nodes count, the rows behind them and
    those before the first tree are not written."""
    c = Cache("bf16", 8, 16, 2, 64, 5)
    c.fill([(p, s) for p in range(8) for s in range(16)])
    rows = 3 * most + 5
    q = torch.randn(rows, 4, 64, device="cuda:0").to(torch.bfloat16)
    table = ids([[0, 1, 2], [3, 4, 5]])
    ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, 2, 4, 48, most), dtype=torch.uint8,
                     device="cuda:0")

    def run(starts):
        out, lse = torch.full_like(q, 7), torch.full((rows, 4), 7.0, device="cuda:0")
        api.paged_tree_attention(c.kv, q, table, ids([20, 9]), out, ws, 48, most, starts=ids(starts), lse=lse)
        torch.cuda.synchronize()
        return out, lse

    second = most + 5
    for starts in ([3, second, second + most], [3, second, rows]):
        out, lse = run(starts)
        alone = [run([3, 3 + most, 3 + most]), run([second, second, second + most])]
        for r in range(rows):
            tree = 0 if 3 <= r < 3 + most else 1 if second <= r < second + most else None
            for got, a, b in zip((out, lse), *alone):
                want = torch.full_like(got[r], 7) if tree is None else (a, b)[tree][r]
                assert torch.equal(got[r], want), (starts, r)
                assert tree is None or bool((want != 7).any())


@pytest.mark.parametrize("most", [3, 30])
def test_trees_of_no_sequence(most):
    """Sequences at or above n_seqs, and below 0, between others: no keys, whatever lies behind the table."""
    rng = np.random.default_rng(most)
    c = Cache("bf16", 12, 16, 2, 64, 5)
    c.fill([(p, s) for p in range(12) for s in range(16)])
    tables = ids(rng.permutation(12).reshape(4, 3))          # the call has the first two of them
    nodes = [most, 2, 1, most, 3, 2]
    seqs = [1, 2, 1 << 20, 0, -1, 3]
    starts = np.concatenate([[0], np.cumsum(nodes)])
    rows = int(starts[-1])
    q = torch.randn(rows, 4, 64, device="cuda:0").to(torch.bfloat16)
    mask = bits64([m for n in nodes for m in O.chain(n)])

    def run(seqs):
        out, lse = torch.full_like(q, 7), torch.full((rows, 4), 7.0, device="cuda:0")
        ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, 6, 4, 48, most), dtype=torch.uint8,
                         device="cuda:0")
        api.paged_tree_attention(c.kv, q, tables[:2], ids([10, 3, 0, 17, 9, 5]), out, ws, 48, most, tree=mask,
                                 starts=ids(starts), seqs=ids(seqs), lse=lse)
        torch.cuda.synchronize()
        return out, lse

    (out, lse), (want, want_lse) = run(seqs), run([1, 0, 1, 0, 1, 0])
    for g, s in enumerate(seqs):
        at = slice(int(starts[g]), int(starts[g + 1]))
        if 0 <= s < 2:
            assert torch.equal(out[at], want[at]) and torch.equal(lse[at], want_lse[at])
        else:
            assert not out[at].any() and bool((lse[at] == -math.inf).all())
            assert want[at].any() and bool(want_lse[at].isfinite().all())


@pytest.mark.parametrize("trees", [127, 128])
@pytest.mark.parametrize("most", [1, 30])
def test_long_keys_on_both_sides_of_many_outputs(trees, most):
    """1,016 and 1,024 outputs (a tree and key head each), some of them of thousands of keys."""
    rng = np.random.default_rng(trees)
    lengths = rng.integers(0, 60, trees)
    lengths[[2, 50, trees - 1]] = 5000, 1777, 3200
    nodes = rng.integers(0, 2, trees)
    nodes[[2, 7, trees - 1]] = most, 0, 1
    run_tree("bf16", "bf16", lengths.tolist(), nodes.tolist(), 16, 8, 64, 16, seed=most, max_nodes=most)


@pytest.mark.parametrize("lengths,most,heads,hk,max_keys", [
    ([30] * 127 + [1900], 9, 16, 8, None),               # whole: no keys beyond 2,048
    ([30] * 127 + [1900], 1, 16, 8, 2049),               # cut, and as its bound says
    ([2100] + [5, 40, 0] * 340 + [3001, 70, 2500] * 5, 2, 2, 1, None),   # 1,036 trees: two launches
    ([40, 2500] * 15 + [7], 1, 70, 70, None)])           # 2,170 outputs of many key heads: whole
def test_many_outputs_whole_and_cut(lengths, most, heads, hk, max_keys):
    rng = np.random.default_rng(len(lengths))
    nodes = rng.integers(0, most + 1, len(lengths))
    nodes[[0, -1]] = most
    run_tree("bf16", "bf16", lengths, nodes.tolist(), heads, hk, 64, 16, seed=3, max_nodes=most,
             max_keys=max_keys)


def test_one_launch_and_several_give_the_same_bits():
    """The trees of one launch, over and over: each as often as it comes, in whichever launch."""
    n, times = 1024, 3
    c = Cache("bf16", 400, 16, 1, 64, 1)
    c.fill([(p, s) for p in range(400) for s in range(16)])
    rng = np.random.default_rng(0)
    table = ids(rng.integers(0, 400, (8, 200)))
    lengths, seqs = rng.integers(0, 90, n), rng.integers(0, 8, n)
    lengths[[3, 700]] = 3100, 2500
    q = torch.randn(n, 2, 64, device="cuda:0").to(torch.bfloat16)
    outs = []
    for k in (1, times):
        ws = torch.empty(api.paged_tree_attention_workspace_bytes(c.kv, n * k, 2, 3200, 1), dtype=torch.uint8,
                         device="cuda:0")
        out = torch.empty(n * k, 2, 64, device="cuda:0", dtype=torch.bfloat16)
        api.paged_tree_attention(c.kv, q.repeat(k, 1, 1), table, ids(np.tile(lengths, k)), out, ws, 3200, 1,
                                 seqs=ids(np.tile(seqs, k)))
        outs.append(out.view(torch.int16).unflatten(0, (k, n)))
    torch.cuda.synchronize()
    assert outs[0].any() and bool((outs[1] == outs[0]).all())
