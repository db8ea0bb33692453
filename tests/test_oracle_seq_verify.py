"""The oracle of drafted trees and of their verification: by hand, and the distribution of what it accepts."""
import numpy as np
import pytest

from oracle import seq_oracle as O


def test_trees_by_hand():
    assert O.depths([-1, 0, 0, 1, -2, 4, -1, 7, 3]) == [0, 1, 1, 2, -1, -1, 0, -1, 3]
    see, far = O.tree(None, None, None, [-1, 0, 0, 1], np.array([True, False]), 2)
    assert see.astype(int).tolist() == [[1, 0, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [1, 0, 1, 0, 1, 0], [1, 0, 1, 1, 0, 1]]
    assert far[3].tolist() == [4, 3, 2, 1, 1, 0]
    assert O.tree(None, None, None, [-1, 0, 0, 1], np.array([True, True]), 2, window=2)[0][3].astype(int).tolist() == [0, 0, 0, 1, 0, 1]


def test_draws_by_hand():
    p = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [O._drawn(p, u) for u in (-1.0, 0.0, 0.2499, 0.25, 0.74, 0.75, 0.999, 1.0, 7.0, float("nan"))] == [1, 1, 1, 3, 3, 4, 4, 4, 4, 1]
    assert O._drawn(np.zeros(3), 0.5) == -1
    logits = np.log(np.array([[0.1, 0.6, 0.3], [0.5, 0.25, 0.25], [0.2, 0.2, 0.6]]))
    assert O.verify(logits, [9, 1, 2], [0.3, 0.6, 0.1], [-1, 0, 0]) == ([0, 1], 1)   # draws 1, then 1, which no child has
    assert O.verify(logits, [9, 1, 2], [0.8, 0.6, 0.1], [-1, 0, 0]) == ([0, 2], 0)
    assert O.verify(logits, [9, 1, 2], [0.3, 0.6, 0.1], temperature=0.0) == ([0, 1], 0)
    draft = np.log(np.array([[0.5, 0.4, 0.1], [0.1, 0.1, 0.8]]))
    assert O.verify(logits, [9, 0, 1], [0.3, 0.0, 0.0, 0.51], draft=draft) == ([0], 2)   # 0.1 / 0.5 < 0.3: refused; the rest is (0, 0.2, 0.2), 0.5 its border
    assert O.verify(logits, [9, 0, 1], [0.19, 0.0, 0.0, 0.5], draft=draft) == ([0, 1, 2], 2)
    assert O.verify(logits, [9, 0, -1], [0.19, 0.0, 0.0, 0.5], draft=draft) == ([0, 1], 1)


@pytest.mark.parametrize("drafted", [False, True])
def test_the_first_token_is_distributed_as_the_target_has_it(drafted):
    """Over a grid of 400 x 400 numbers (and the draft's draws, with their probabilities); a share of a grid is off by the number of its steps, 1 / 400 each, at most one for each
    token and direction."""
    g = np.random.default_rng(1)
    logits, draft, share = g.standard_normal((2, 4)), g.standard_normal((1, 4)), np.zeros(4)
    p, q = O._probabilities(logits[0], 1.0), O._probabilities(draft[0], 1.0)
    grid = (np.arange(400) + 0.5) / 400
    for x in range(4):
        for u in grid:
            if drafted:
                for w in grid[::20]:
                    path, token = O.verify(logits, [0, x], [u, 0.0, w], draft=draft)
                    share[x if len(path) > 1 else token] += q[x] / 400 / 20
            else:
                path, token = O.verify(logits, [0, x], [u, 0.5])
                share[x if len(path) > 1 else token] += q[x] / 400
    assert np.abs(share - p).max() < (2 / 400 if not drafted else 2 / 400 + 1 / 20)
