"""Pins of oracle/tokens.py: hand-worked cases, differences, and the random generator's published outputs."""
import numpy as np
import pytest

import oracle.tokens as T


def test_sorting_worked_by_hand():
    order, offsets, place, token = T.sort_tokens([2, 0, -1, 2, 5, 0], 4, per_token=2)
    assert order.tolist() == [1, 5, 0, 3, 2, 4] and offsets.tolist() == [0, 2, 2, 4, 4]
    assert place.tolist() == [2, 0, -1, 3, -1, 1] and token.tolist() == [0, 2, 0, 1, 1, 2]
    order, offsets, place, token = T.sort_tokens([], 3)
    assert order.size == place.size == token.size == 0 and offsets.tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("counter,key,words", [      # the generator's authors' known answers
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator(counter, key, words):
    assert tuple(T.philox(counter, key)) == words


def test_dropout_is_made_of_the_generator():
    words = T.philox((1, 7, 3, 9), (5, 6))
    u = T.dropout_bits(2, 13, (6 << 32) + 5, layer=9, first_row=(3 << 32) + 6)
    assert [int(v) for v in u[1, 8:13]] == [words[0] % 65536, words[0] >> 16, words[1] % 65536, words[1] >> 16, words[2] % 65536]
    x = np.arange(1.0, 27.0).reshape(2, 13)
    y = T.dropout(x, 0.25, 11)
    kept = T.dropout_bits(2, 13, 11) >= 16384
    assert 0 < kept.sum() < 26 and np.array_equal(y, np.where(kept, x * (4 / 3), 0.0))
    assert np.array_equal(T.dropout(x, 1.0, 11, residual=x), x) and np.array_equal(T.dropout(x, 0.0, 11), x)
    assert np.array_equal(T.dropout(x[1:], 0.5, 11, first_row=1), T.dropout(x, 0.5, 11)[1:])


def test_dropout_keeps_its_share():
    """Of n independent elements a share of 1 - p is kept, to within five standard deviations."""
    n, p = 64 * 256, 0.1
    kept = (T.dropout_bits(64, 256, 3) >= round(p * 65536)).sum()
    assert abs(kept - n * (1 - p)) < 5 * (n * p * (1 - p)) ** 0.5


def test_lookup_and_gradients_against_differences():
    rng = np.random.default_rng(0)
    ids = np.array([[0, 3], [3, 3], [-1, 2], [9, 0]])
    table, weights, dy = rng.standard_normal((4, 5)), rng.standard_normal((4, 2)), rng.standard_normal((4, 5))
    y, size = T.lookup(ids, table, 0.7, weights)
    assert np.allclose(y[1], 0.7 * (weights[1, 0] + weights[1, 1]) * table[3]) and np.allclose(y[2], 0.7 * weights[2, 1] * table[2])
    assert np.all(size >= np.abs(y) - 1e-15)
    dtable, _, dweights, _ = T.lookup_gradients(ids, dy, 4, table, 0.7, weights)
    loss = lambda t, w: np.sum(T.lookup(ids, t, 0.7, w)[0] * dy)
    for at in np.ndindex(4, 5):
        step = np.zeros((4, 5))
        step[at] = 0.5
        assert np.isclose(loss(table + step, weights) - loss(table - step, weights), dtable[at], atol=1e-12)
    for at in np.ndindex(4, 2):
        step = np.zeros((4, 2))
        step[at] = 0.5
        assert np.isclose(loss(table, weights + step) - loss(table, weights - step), dweights[at], atol=1e-12)


def test_grouped_product_worked_by_hand():
    x = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0], [7.0, 8.0]])
    w = np.array([[[1.0, 0.0]], [[0.0, -1.0]]])                     # two groups, one output
    y, size = T.grouped_product(x, w, [0, 1, 3], bias=np.array([[10.0], [20.0]]), y=np.full((4, 1), 9.0))
    assert y.ravel().tolist() == [11.0, 16.0, 14.0, 9.0] and size.ravel().tolist() == [11.0, 24.0, 26.0, 0.0]
    dx, _ = T.grouped_product(y, w, [0, 1, 3], transposed=True)      # the gradient of x for the gradient y: in columns, out rows
    assert dx.tolist() == [[11.0, 0.0], [0.0, -16.0], [0.0, -14.0], [0.0, 0.0]]
