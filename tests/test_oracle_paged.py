"""Pins of the paged-cache definitions (oracle/paged.py) on cases done by hand, no GPU."""
import numpy as np

import oracle.paged as ref


def test_page_plan_by_hand():
    table = np.full((2, 4), -1, np.int32)
    table[0, :2] = (5, 6)
    table[1, :1] = (7,)
    got = ref.page_plan([7, 2], [3, 1], [(2, 0), (1, 0)], table, np.array([1, 2, 3, 0], np.int32),
                        [4, 6, 0], 4, 6)
    assert got["table"].tolist() == [[5, 6, 1, -1], [7, -1, -1, -1]]
    assert got["pages"].tolist() == [[3, 0], [1, 0]]
    assert got["cursor"].tolist() == [5, 6, 0]
    assert got["starts"].tolist() == [0, 3, 4] and got["totals"].tolist() == [10, 3]
    assert got["slots"].tolist() == [6 * 4 + 3, 4, 5, 7 * 4 + 2, -1, -1]
    assert got["positions"].tolist() == [7, 8, 9, 2, -1, -1]


def test_page_plan_window_by_hand():
    # 21 tokens, window 8: the next query is at 21 and sees 14 .., so entries 0-2 (keys 0-11) are
    # behind it; entry 0 holds the sinks and stays
    table = np.arange(10, 16, dtype=np.int32)[None]
    got = ref.page_plan([21], [1], [(6, 0)], table, np.full(8, -1, np.int32), [0, 0, 0], 4, 1, 8, 2)
    assert got["pages"].tolist() == [[6, 3]]
    assert got["cursor"].tolist() == [0, 2, 0] and got["queue"][:2].tolist() == [11, 12]
    got = ref.page_plan([21], [-1], [(6, 3)], table, got["queue"], got["cursor"], 4, 0, 8, 2)
    assert got["queue"][:6].tolist() == [11, 12, 10, 13, 14, 15] and got["cursor"].tolist() == [0, 6, 0]


def test_norm_rope_quarter_turn():
    x = np.array([[[3.0, 0.0, 4.0, 0.0]]])
    one, zero = np.ones((1, 2)), np.zeros((1, 2))
    assert np.allclose(ref.norm_rope(x, None, zero, one, 0, False), [[[-4, 0, 3, 0]]])
    assert np.allclose(ref.norm_rope(x, None, zero, one, 0, True), [[[0, 3, 0, 4]]])
    assert np.allclose(ref.norm_rope(x, np.full(4, 2.0), one, zero, 0, True),
                       np.array([[[3, 0, 4, 0]]]) / 2.5 * 2)


def test_attention_masks():
    # one head of width 1 and q = 0: the output is the mean of the visible values
    v = np.arange(12.0).reshape(3, 4, 1, 1)
    k, q = np.ones_like(v), np.zeros((2, 1, 1))
    table, starts, totals = np.array([[2, 0, -1]]), [0, 2], [7]
    row = lambda **m: ref.attention(q, k, v, table, starts, totals, **m)[0][:, 0, 0].tolist()  # noqa: E731
    # keys 0-3 are 8 .. 11, keys 4-6 are 0 .. 2; queries at 5 and 6
    assert row() == [39 / 6, 41 / 7]
    assert row(causal=False) == [41 / 7, 41 / 7]
    assert row(window=2) == [0.5, 1.5]
    assert row(window=2, sinks=1) == [9 / 3, 11 / 3]
    got = ref.attention(q, k, v, table, starts, totals, window=1, shared_table=[1], shared_length=3)[0]
    assert got[:, 0, 0].tolist() == [(4 + 5 + 6 + 1) / 4, (4 + 5 + 6 + 2) / 4]
    assert ref.attention(q, k, v, np.array([[-1, -1, -1]]), starts, totals)[0].tolist() == [[[0]], [[0]]]
