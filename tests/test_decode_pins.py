"""The 64-bit forms of the decoding operators against hand-made cases (CPU)."""
import math

import numpy as np
import pytest

from oracle import decode


@pytest.mark.parametrize("u,token", [(0.0, 0), (0.24, 0), (0.25, 1), (0.5, 2), (0.75, 3), (0.99, 3),
                                     (1.0, 3), (-1.0, 0), (math.nan, 0)])
def test_equal_logits_are_drawn_in_index_order(u, token):
    assert decode.sample_row(np.zeros(4, np.float32), u) == (token, 0.25)


def test_filters_cut_the_ranking():
    z = np.log(np.array([1, 4, 2, 1, 4, 4], np.float64)).astype(np.float32)
    assert decode.sample_row(z, 0.99, k=2) == (4, 0.5)           # the first two of three equals
    assert decode.sample_row(z, 0.99, k=1) == (1, 1.0)
    assert decode.sample_row(z, 0.99, p=0.0)[0] == 1             # at least one token
    assert decode.sample_row(z, 0.99, p=0.5)[0] == 4             # 8 of 16 with two of the 4s
    assert decode.sample_row(z, 0.99, p=0.51)[0] == 5
    assert decode.sample_row(z, 0.99, m=0.9)[0] == 5             # the 4s
    assert decode.sample_row(z, 0.66, m=0.4)[0] == 4             # the 4s and the 2
    assert decode.sample_row(z, 0.0, t=0.0) == (1, 1.0)


def test_rows_without_a_distribution():
    assert decode.sample_row(np.array([0, np.nan], np.float32), 0.5) == (-1, 0.0)
    assert decode.sample_row(np.full(3, -np.inf, np.float32), 0.5) == (-1, 0.0)
    assert decode.sample_row(np.array([0, np.inf, np.inf], np.float32), 0.5) == (2, 0.5)
    assert decode.sample_row(np.array([-np.inf, 3, -np.inf], np.float32), 0.0) == (1, 1.0)


def test_rotation_and_norm():
    x = np.array([3.0, 0.0, 4.0, 0.0])
    y, _ = decode.rope(x, None, 0.0, 1, np.array([math.pi / 2, 0.0]), False)
    assert np.allclose(y, [-4, 0, 3, 0])                          # pairs (0, 2), (1, 3)
    y, _ = decode.rope(x, None, 0.0, 2, np.array([math.pi / 2]), True)
    assert np.allclose(y, [-3, 0, 4, 0])                          # pair (0, 1) by half a turn
    y, _ = decode.rope(x, np.array([2.0, 1, 1, 1]), 0.0, 0, np.zeros(0), False)
    assert np.allclose(y, [2 * 3 / 2.5, 0, 4 / 2.5, 0])


def test_attention_of_a_tree():
    # one request, one cached token, rows 0 -> 1 and 0 -> 2
    keys = np.zeros((1, 4, 1, 2))
    values = np.arange(8.0).reshape(1, 4, 1, 2)
    q = np.zeros((3, 1, 2))
    mask = np.array([[1], [3], [5]], dtype=np.int64)
    out, _, _ = decode.block_attention(q, keys, values, np.array([[0]]), [1], [2], 1.0, mask)
    assert np.allclose(out[:, 0], [[1, 2], [2, 3], [8 / 3, 11 / 3]])
    out, _, _ = decode.block_attention(q, keys, values, np.array([[0]]), [1], [2], 1.0)
    assert np.allclose(out[:, 0], [[1, 2], [2, 3], [3, 4]])
    out, _, _ = decode.block_attention(q, keys, values, np.array([[0]]), [0], [2], 1.0, mask * 0)
    assert (out == 0).all()
    out, _, _ = decode.block_attention(q, keys, values, np.array([[1]]), [1], [2], 1.0)
    assert (out == 0).all()                                        # a page outside the cache
