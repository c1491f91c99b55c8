"""The 4-bit cache's plain definitions (oracle/cache4.py) on values worked out by hand."""
import numpy as np

import oracle.cache4 as ref


def test_codes_and_scales():
    x = np.zeros((1, 32))
    x[0, :8] = [7, -7, 0.25, 0.75, 5, -2.5, 0.2, -0.0]  # 7 <= 7 * 2^0: scale 1, 0.25 and 0.75 and 5 are ties
    codes, scales = ref.quantise(x)
    assert scales.tolist() == [[127]]
    assert codes[0, :4].tolist() == [0xF7, 0x20, 0xC6, 0x80]  # 6 -6, 0 1, 4 -2, 0 -0
    assert ref.values(codes, scales)[0, :8].tolist() == [6, -6, 0, 1, 4, -2, 0, 0]
    x[0, 0] = 7.0001
    assert ref.quantise(x)[1].tolist() == [[128]]
    assert ref.quantise(np.zeros((1, 32)))[1].tolist() == [[1]]
    assert ref.quantise(np.full((1, 32), 1e300))[1].tolist() == [[252]]
    x[0, 5] = np.inf
    codes, scales = ref.quantise(x)
    assert scales.tolist() == [[255]] and np.isnan(ref.values(codes, scales)).all()


def test_every_element_is_within_one_scale():
    x = np.random.default_rng(0).normal(size=(50, 64)) * 2.0 ** np.arange(-25, 25)[:, None]
    codes, scales = ref.quantise(x)
    off = np.abs(ref.values(codes, scales) - x)
    s = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    assert (off <= s).all() and (np.abs(x).reshape(50, 2, 32).max(-1) > 3.5 * 2.0 ** (scales.astype(float) - 127)).all()


def test_weights_are_probabilities():
    """A step's weights over all keys of a head add up to its query rows; lse is the logarithm of the sum."""
    g = np.random.default_rng(1)
    q, k, v = g.normal(size=(3, 4, 32)), g.normal(size=(2, 8, 2, 32)), g.normal(size=(2, 8, 2, 32))
    table, starts, totals = np.array([[1, 0]]), np.array([0, 3]), np.array([13])
    out, _, _, _, lse = ref.attention(q, k, v, table, starts, totals)
    w, _, terms = ref.key_weights(q, lse, k, table, starts, totals, np.zeros((2, 2, 8)))
    np.testing.assert_allclose(w.sum((0, 2)), [6, 6], rtol=1e-12)  # 3 queries of 2 heads each
    assert terms[1, 0, 0] == 6 and terms[0, 0, 4] == 2 and terms[0, 0, 5] == 0
    s = np.array([k[table[0, j // 8], j % 8, 1] @ q[0, 2] / np.sqrt(32) for j in range(11)])
    p = np.exp(s - lse[0, 2])
    np.testing.assert_allclose(p.sum(), 1, rtol=1e-12)
    np.testing.assert_allclose(out[0, 2], sum(p[j] * v[table[0, j // 8], j % 8, 1] for j in range(11)), rtol=1e-9)


def test_eviction_by_hand():
    """Six tokens on pages 2, 0 (of 4 places): budget 3 keeps the first, the last and the heaviest of the others."""
    part = np.arange(3 * 4).reshape(3, 4, 1, 1)
    weights = np.zeros((3, 1, 4))
    weights[2, 0], weights[0, 0, :2] = [9, 1, 5, 5], [5, 0]
    queue = np.full(4, -1)
    parts, w, queue, totals, pages, cursor, evicted = ref.evict(
        [part], weights, np.array([[2, 0]]), np.array([6]), np.array([[2, 0]]), queue, np.array([0, 3, 0]), 3, 4, 1, 1)
    assert parts[0][2, :, 0, 0].tolist() == [8, 10, 1, 11] and w[2, 0].tolist() == [9, 5, 0, 5]
    assert parts[0][0].tolist() == part[0].tolist() and queue.tolist() == [-1, -1, -1, 0]
    assert (totals.tolist(), pages.tolist(), cursor.tolist(), evicted.tolist()) == ([3], [[1, 0]], [0, 4, 0], [3])
