"""The sampling oracle (oracle/sample.py) against worked values."""
import math

import numpy as np
import pytest

from oracle import sample as O

LOGP = np.log([0.1, 0.4, 0.2, 0.3])  # order: 1, 3, 2, 0; sums 0.4, 0.7, 0.9, 1


@pytest.mark.parametrize("u,token", [(0.0, 1), (0.39, 1), (0.41, 3), (0.69, 3), (0.71, 2), (0.89, 2), (0.91, 0), (0.999999, 0)])
def test_places(u, token):
    t, lp, n = O.sample(LOGP, 1.0, u)
    assert t == token and n == 4 and lp == pytest.approx(LOGP[token], abs=1e-12)


def test_filters():
    assert O.sample(LOGP, 1.0, 0.99, top_k=2)[::2] == (3, 2)
    assert O.sample(LOGP, 1.0, 0.99, top_k=2)[1] == pytest.approx(math.log(0.3 / 0.7))
    assert O.sample(LOGP, 1.0, 0.99, top_p=0.69)[::2] == (3, 2)
    assert O.sample(LOGP, 1.0, 0.99, top_p=0.71)[::2] == (2, 3)
    assert O.sample(LOGP, 1.0, 0.99, top_p=0.0)[::2] == (1, 1)
    assert O.sample(LOGP, 1.0, 0.99, top_k=3, top_p=0.75)[::2] == (3, 2)     # 0.75 of 0.9 is 0.675
    assert O.sample(LOGP, 1.0, 0.99, min_p=0.49)[::2] == (2, 3)              # 0.2 / 0.4
    assert O.sample(LOGP, 1.0, 0.99, min_p=0.51)[::2] == (3, 2)
    assert O.sample(LOGP, 1.0, 0.99, min_p=2.0)[::2] == (1, 1)
    assert O.sample(LOGP, 0.0, 0.99) == (1, 0.0, 1) == O.sample(LOGP, math.nan, 0.99) == O.sample(LOGP, -1.0, 0.99)
    hot = O.sample(LOGP, 2.0, 0.0)  # weights go as the root
    assert hot[1] == pytest.approx(math.log(math.sqrt(0.4) / np.sqrt([0.1, 0.4, 0.2, 0.3]).sum()))


def test_ties_and_none():
    assert O.sample(np.zeros(5), 1.0, 0.5)[0] == 2 and O.sample(np.zeros(5), 1.0, 0.5, top_k=2)[0] == 1
    assert O.sample(np.full(3, -np.inf), 1.0, 0.5) == (-1, -math.inf, 0)
    assert O.sample([1.0, np.inf, np.inf], 1.0, 0.6)[::2] == (2, 3)


def test_scores():
    rows = np.array([[0.0, 1.0, 2.0], [1.0, np.nan, 0.0], [0.5, 3.0, 5.0]])
    S, who = O.scores(rows, [1.0, 0.0], [0.0, 1.0], allowed=[True, True, False])
    assert S.tolist() == [2.0, 4.0, -np.inf] and who.tolist() == [1, 2, 0]
