"""Pins of the batched decoding oracle (oracle/serving_oracle.py): closed forms
and the decoder oracle's own rotation."""
import numpy as np

from oracle import serving_oracle as S


def test_rotation_turns_pairs_by_the_position():
    x = np.array([1.0, 0.0, 0.0, 2.0, 5.0])
    y = S.rotate(x, 3, [1.0, 0.5], interleaved=False)      # pairs (0, 2), (1, 3)
    np.testing.assert_allclose(y, [np.cos(3), -2 * np.sin(1.5), np.sin(3), 2 * np.cos(1.5), 5.0])
    y = S.rotate(x, 3, [1.0, 0.5], interleaved=True)       # pairs (0, 1), (2, 3)
    np.testing.assert_allclose(y, [np.cos(3), np.sin(3), -2 * np.sin(1.5), 2 * np.cos(1.5), 5.0])
    assert np.array_equal(S.rotate(x, 0, [1.0, 0.5], False), x)


def test_slots_follow_the_table():
    table = [[4, -1, 2], [9, 0, 1]]
    assert S.slot_of(table, 5, 8, 0, 7) == (4, 7)
    assert S.slot_of(table, 5, 8, 0, 8) is None            # no page
    assert S.slot_of(table, 5, 8, 0, 17) == (2, 1)
    assert S.slot_of(table, 5, 8, 1, 0) is None            # page 9 of 5
    assert S.slot_of(table, 5, 8, 0, 24) is None and S.slot_of(table, 5, 8, 2, 0) is None
    assert S.visible(table, 5, 8, 0, 18, 100, 3) == [(2, 0), (2, 1)]
    assert S.visible(table, 5, 8, 0, 0, 100, 0) == [] and S.visible(table, 5, 8, -1, 4, 9, 0) == []
    assert len(S.visible(table, 5, 8, 0, 50, 7, 0)) == 7


def test_attention_of_equal_and_of_dominant_scores():
    rng = np.random.default_rng(0)
    v = rng.standard_normal((6, 1, 4))
    out, lse, _, _ = S.attend(np.zeros((2, 4)), rng.standard_normal((6, 1, 4)), v, 1.0)
    np.testing.assert_allclose(out, np.repeat(v.mean(0), 2, 0))
    np.testing.assert_allclose(lse, np.log(6))
    k = np.zeros((6, 1, 4))
    k[3, 0, 0] = 1000.0
    out, lse, _, _ = S.attend(np.ones((1, 4)), k, v, 1.0)
    np.testing.assert_allclose(out[0], v[3, 0])
    np.testing.assert_allclose(lse, 1000.0)
    out, lse, _, _ = S.attend(np.ones((1, 4)), k[:0], v[:0], 1.0)
    assert not out.any() and lse[0] == -np.inf


def test_heads_share_the_key_head_of_their_group():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((6, 4)), rng.standard_normal((5, 2, 4)), rng.standard_normal((5, 2, 4))
    out, _, _, _ = S.attend(q, k, v, 0.5)
    for h in range(6):
        one, _, _, _ = S.attend(q[h:h + 1], k[:, h // 3:h // 3 + 1], v[:, h // 3:h // 3 + 1], 0.5)
        np.testing.assert_allclose(out[h], one[0])


def test_logits_by_hand():
    x, t, _ = S.process_logits([2.0, -2.0, 1.0, 0.5, 3.0], history=[0, 1, 2, 2, 9, -1], prompt=2,
                               repetition=2.0, presence=0.25, frequency=0.5,
                               biases=[(3, 9.0), (3, 0.5), (-4, 1.0), (5, 1.0)], mask=[0b01111])
    # 0, 1: prompt only; 2: twice generated; 3: the later bias; 4: not allowed.
    np.testing.assert_allclose(x, [1.0, -4.0, 0.5 - 1.0 - 0.25, 1.0, -np.inf])
    assert t == 0                                            # ties go to the lower id
    assert S.process_logits([1.0, 2.0], mask=[0])[1] == -1
    assert S.process_logits([np.nan, 2.0])[1] == 1
