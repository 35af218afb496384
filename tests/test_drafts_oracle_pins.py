"""The drafted-token oracle (oracle/drafts_oracle.py) against closed forms."""
import numpy as np

from oracle import drafts_oracle as O
from oracle import serving_oracle as S


def test_depths_and_chains():
    assert O.chain(4) == [1, 3, 7, 15] and O.depths(O.chain(4)) == [0, 1, 2, 3]
    assert O.depths([0b1, 0b11, 0b101, 0b1011, 0b10101]) == [0, 1, 1, 2, 2]
    assert O.depths([0b110, 0b010, 0b101]) == [0, 0, 1]


def test_axes_turn_pairs_by_their_own_angle():
    q = k = v = np.array([[[1.0, 0.0, 2.0, 0.0]]])
    table = np.array([[0]])
    out, stored = O.append_axes(q, k, v, [0], [[90, 7]], [0, 5], [0], table, 1, 8, [np.pi / 180] * 2,
                                True)
    assert np.allclose(out[0], [[0, 1, 2, 0]]) and np.allclose(stored[0, 0][0], [[0, 1, 2, 0]])
    angles = np.arange(5)
    for inter in (False, True):
        a = O.append_axes(np.ones((5, 1, 8)), np.ones((5, 1, 8)), np.ones((5, 1, 8)), angles,
                          angles[:, None], [0] * 4, [0] * 5, table, 1, 8, [1, .5, .1, .01], inter)
        b = S.append(np.ones((5, 1, 8)), np.ones((5, 1, 8)), np.ones((5, 1, 8)), angles, [0] * 5, table,
                     1, 8, [1, .5, .1, .01], inter)
        assert np.allclose(a[0], b[0])


def test_a_chain_of_one_node_sees_what_a_decode_step_does():
    table = np.array([[3, 1, 0]])
    for n in (0, 5, 16, 20):
        for window in (0, 1, 6):
            got = [at for at, _ in O.node_keys([1], 0, table, 4, 8, 0, n, 100, window)]
            assert got == S.visible(table, 4, 8, 0, n + 1, 100, window)


def test_nodes_see_ancestors_within_the_window():
    table = np.array([[0, 1]])
    masks = [0b1, 0b11, 0b101, 0b1011]
    keys = lambda i, w: [(s, d) for (p, s), d in O.node_keys(masks, i, table, 2, 8, 0, 2, 100, w)]
    assert keys(3, 0) == [(0, 4), (1, 3), (2, 2), (3, 1), (5, 0)]
    assert keys(3, 3) == [(2, 2), (3, 1), (5, 0)]
    assert keys(2, 2) == [(2, 1), (4, 0)]
    assert O.node_keys(masks, 3, table, 2, 8, 0, 2, 4, 0)[-1] == ((0, 3), 1)   # cut
    assert O.node_keys(masks, 0, table, 2, 8, 1, 2, 4, 0) == []
    assert O.node_keys(masks, 0, table, 2, 8, 0, -1, 4, 0) == []


def test_shaped_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 4)), rng.normal(size=(5, 1, 4)), rng.normal(size=(5, 1, 4))
    plain = O.attend(q, k, v, range(5), 0.5)
    assert np.allclose(plain[0], S.attend(q, k, v, 0.5)[0])
    assert np.allclose(O.attend(q, k, v, range(5), 0.5, cap=1e6)[0], plain[0])
    flat = O.attend(q, k, v, range(5), 1e6, cap=1e-9)          # all scores alike
    assert np.allclose(flat[0], v[:, 0].mean(0)) and np.allclose(flat[1], np.log(5))
    near = O.attend(q, k, v, range(5), 0.5, slopes=[1e3, 0.0])  # only the nearest key
    assert np.allclose(near[0][0], v[0, 0]) and np.allclose(near[0][1], plain[0][1])


def test_accept_walks_agreeing_drafts():
    assert O.accept([5, 1, 2, 3], [1, 2, 3, 9], O.chain(4)) == ([0, 1, 2, 3], [1, 2, 3, 9])
    assert O.accept([5, 1, 2, 3], [1, 7, 3, 9], O.chain(4)) == ([0, 1], [1, 7])
    assert O.accept([5, 1, 1, 4], [1, 8, 4, 6], [1, 3, 5, 0b1101]) == ([0, 1], [1, 8])
    assert O.accept([5, 1, 2, 4], [2, 8, 4, 6], [1, 3, 5, 0b1101]) == ([0, 2, 3], [2, 4, 6])
    assert O.accept([5, 0], [-1, 0], O.chain(2)) == ([0], [-1])
    assert O.accept([], [], []) == ([], [])


def test_moves():
    pages = np.arange(4 * 8).reshape(4, 8, 1)
    table = np.array([[2, 0], [1, 3]])
    out = O.compact(pages, table, 4, 8, [6], [[0, 2, 3, -1]], [3], [0])
    assert out[2, 6, 0] == 16 + 6 and out[2, 7, 0] == 0 and out[0, 0, 0] == 1 and out[0, 1, 0] == 1
    rows, out = O.fork(pages, np.array([[2, 0, -1]]), 4, 8, [0, 0, 0, 3], [11, 8, 3, 5], [3, 1, -1, 0])
    assert rows.tolist() == [[2, 3, -1], [2, -1, -1], [2, -1, -1], [-1, -1, -1]]
    assert out[3, :, 0].tolist() == [0, 1, 2, 27, 28, 29, 30, 31] and np.array_equal(out[:3], pages[:3])
