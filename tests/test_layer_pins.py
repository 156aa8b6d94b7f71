"""The layer-wise oracle (oracle/layer.py) against hand-worked values and properties
that follow from the definitions; no GPU."""
import math

import numpy as np
import pytest

from oracle import layer as L


def test_rotation_by_hand():
    x = np.array([1.0, 0.0, 0.0, 1.0, 7.0, 8.0])
    # pair 0 turns by 3 * 100^0 = 3, pair 1 by 3 * 100^(-1/2) = 0.3; dims 4, 5 stay
    want = [math.cos(3), math.sin(3), -math.sin(0.3), math.cos(0.3), 7, 8]
    assert np.allclose(L.rotate(x, 3, 100.0, 4, False), want, atol=1e-15)
    y = np.array([1.0, 0.0, 0.0, 1.0, 7.0, 8.0])  # halves: pairs (0, 2), (1, 3)
    want = [math.cos(3), -math.sin(0.3), math.sin(3), math.cos(0.3), 7, 8]
    assert np.allclose(L.rotate(y, 3, 100.0, 4, True), want, atol=1e-15)
    assert np.array_equal(L.rotate(x, 0, 100.0, 4, True), x)


def test_rotated_products_depend_on_the_distance_alone():
    r = np.random.RandomState(0)
    q, k = r.randn(8), r.randn(8)
    for halves in (False, True):
        dots = [L.rotate(q, p + 5, 1e4, 8, halves) @ L.rotate(k, p, 1e4, 8, halves) for p in (0, 3, 1000)]
        assert np.ptp(dots) < 1e-10


def test_summary_codes_by_hand():
    k = np.zeros((16, 4))
    k[3] = [1.0, -2.5, 0.0, 100.0]
    k[9] = [-1.0, 0.25, 0.0, 99.0]
    mx, mn, e = L.summarize(k)
    assert e == 0 and mx.tolist() == [1, 1, 0, 100] and mn.tolist() == [-1, -3, 0, 0]
    k[0, 3] = 127.5  # ceil is 128: the next scale
    mx, mn, e = L.summarize(k)
    assert e == 1 and mx.tolist() == [1, 1, 0, 64] and mn.tolist() == [-1, -2, 0, 0]
    assert L.summarize(np.zeros((16, 4)))[2] == -64
    k[0, 3] = np.inf
    assert L.summarize(k)[2] == 64 and L.summarize(k)[0][3] == 127


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 1.0, 1e5])
def test_summaries_bound_the_keys(scale):
    k = np.random.RandomState(1).randn(16, 32) * scale
    mx, mn, e = L.summarize(k)
    assert (np.ldexp(mx.astype(float), e) >= k.max(0)).all() and (np.ldexp(mn.astype(float), e) <= k.min(0)).all()
    if scale > 1e-20:
        assert 64 <= max(np.abs(mx).max(), np.abs(mn).max()) <= 127


def test_measure_bounds_the_scores():
    r = np.random.RandomState(2)
    q, k = r.randn(4, 32), r.randn(16, 32)
    up, dn = np.where(q > 0, q, 0).sum(0), np.where(q < 0, q, 0).sum(0)
    mx, mn, e = L.summarize(k)
    assert (up * np.ldexp(mx.astype(float), e) + dn * np.ldexp(mn.astype(float), e)).sum() >= (q.sum(0) @ k.T).max()


def test_chosen_pages():
    k = np.zeros((16 * 6 + 3, 8))
    k[16 * 3 + 5, 0] = 4.0
    q = np.zeros((2, 8))
    q[:, 0] = 1.0
    assert L.chosen_pages(q, k, 7, 0, 1) == list(range(7))
    assert L.chosen_pages(q, k, 2, 0, 1) == [3, 6]
    assert L.chosen_pages(q, k, 3, 1, 2) == [0, 5, 6]
    assert L.chosen_pages(q, k, 4, 0, 1) == [0, 1, 3, 6]  # equal measures: the lower pages


def test_attend_over_all_pages_is_attention():
    from oracle import pced_oracle as O
    r = np.random.RandomState(3)
    q, k, v = r.randn(4, 16), r.randn(37, 16), r.randn(37, 16)
    want = O.attention(q, k[:, None], v[:, None])
    assert np.allclose(L.attend(q, k, v, [0, 1, 2]), want.reshape(4, 16), atol=1e-14)


def test_adjusted_row_by_hand():
    s = [2.0, -2.0, 1.0, 0.5]
    got = L.adjust_row(s, history=[0, 1, 0, -1, 9], repetition=2.0, presence=0.25, frequency=0.5,
                       biases=[(2, 5.0), (2, 1.0), (7, 3.0)], allowed=[True, True, True, False])
    assert got.tolist() == [2 / 2 - 0.5 * 2 - 0.25, -2 * 2 - 0.5 - 0.25, 2.0, -np.inf]


def test_choice_by_hand():
    rows = [[0.0, 0.0, 0.0], [1.0, 3.0, 2.0], [1.0, 3.0, 5.0]]
    assert L.choose(rows, [0.0, 0.0], [0.0, 0.0]) == (2, 2, 5.0, 3.0)
    assert L.choose(rows, [0.0, 0.0], [0.0, 0.0], [True, True, False]) == (1, 1, 3.0, 1.0)
    assert L.choose(rows, [0.0, 0.0], [0.0, 0.0], [False] * 3) == (-1, 0, -np.inf, -np.inf)
    assert L.choose(rows, [0.0, 0.0], [0.0, 0.0], [True, False, False])[3] == -np.inf
