"""Hand-worked cases of the block-sparse attention's oracle (CPU)."""
import math

import numpy as np

from oracle import block as B


def test_norm_and_rotation_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])                    # mean square 25/4
    y = B.norm_rope(x, None, 1e-30)
    assert np.allclose(y, [[[1.2, 1.6, 0.0, 0.0]]])
    quarter = np.array([[[0.0, 1.0], [1.0, 0.0]]])            # pair 0 by 90 degrees, pair 1 not
    assert np.allclose(B.norm_rope(x, None, 1e-30, quarter), [[[-1.6, 1.2, 0.0, 0.0]]])
    assert np.allclose(B.norm_rope(x, None, 1e-30, quarter, halves=True), [[[0.0, 1.6, 1.2, 0.0]]])
    assert np.allclose(B.norm_rope(x, [2, 1, 1, 1], 1e-30, quarter), [[[-1.6, 2.4, 0.0, 0.0]]])


def test_means_count_the_keys_that_are_there():
    K = np.arange(5.0).reshape(1, 5, 1, 1)
    assert np.allclose(B.block_means(K, [5], 2)[0, 0, :, 0], [0.5, 2.5, 4.0])
    assert np.allclose(B.block_means(K, [3], 2)[0, 0, :, 0], [0.5, 2.0, 0.0])


def test_select_ties_forced_and_empty():
    q = np.ones((1, 1, 2, 1))
    km = np.array([1.0, 3.0, 3.0, 0.0, 3.0]).reshape(1, 1, 5, 1)

    def lists(vis, top_k, first=0, last=0):
        idx, count = B.block_select(q, km, np.array([[vis]]), 2, top_k, first, last, 10)
        return idx[0, 0, 0].tolist(), int(count[0, 0, 0])

    assert lists(10, 2) == ([1, 2], 2)
    assert lists(10, 2, 1) == ([0, 1], 2)
    assert lists(8, 3, 1, 1) == ([0, 1, 3], 3)
    assert lists(3, 3) == ([0, 1, -1], 2)
    assert lists(0, 3, 1, 1) == ([-1, -1, -1], 0)


def test_attend_by_hand():
    Q = np.array([2.0, 0.0]).reshape(1, 1, 2, 1)
    K = np.array([0.0, math.log(3.0) / 2, 5.0]).reshape(1, 3, 1, 1)
    V = np.array([4.0, 8.0, 100.0]).reshape(1, 3, 1, 1)
    O, A, _ = B.block_attend(Q, K, V, np.array([[[[0, 0, 7]]]]), np.array([[[3]]]), np.array([[3]]), 2)
    assert np.allclose(O.ravel(), [7.0, 6.0]) and np.allclose(A, O)
    O, _, _ = B.block_attend(Q, K, V, np.array([[[[0, 1, -1]]]]), np.array([[[2]]]), np.array([[2]]), 2)
    assert np.allclose(O.ravel(), [7.0, 6.0])                  # block 1 is not seen
    O, _, _ = B.block_attend(Q, K, V, np.array([[[[0, 1, -1]]]]), np.array([[[2]]]), np.array([[0]]), 2)
    assert np.array_equal(O.ravel(), [0.0, 0.0])
