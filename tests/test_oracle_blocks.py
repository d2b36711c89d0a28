"""The oracle's blocks and shared rows: properties that pin them (no GPU)."""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import prompt as op


@pytest.mark.parametrize("rows,n,d", [(16, 70, 8), (32, 64, 5), (64, 63, 4)])
def test_no_logit_is_above_its_block_bound(rows, n, d):
    g = np.random.default_rng(n)
    K, q = g.normal(size=(n, d)), g.normal(size=(3, d))
    b = ob.bounds(K, rows, 3e38)
    assert b.shape == (n // rows, 2, d)
    s = ob.scores(q, b)
    for j in range(n // rows):
        assert (q @ K[j * rows:(j + 1) * rows].T).sum(0).max() <= s[j] + 1e-12
        assert np.isclose(s[j], sum(np.maximum(x * b[j, 0], x * b[j, 1]).sum() for x in q))


def test_bounds_of_values_that_are_not_finite():
    K = np.zeros((16, 3))
    K[3, 0], K[5, 1], K[6, 2] = np.inf, -np.inf, np.nan
    b = ob.bounds(K, 16, 100.0)
    assert b[0, 0].tolist() == [100, 0, 100] and b[0, 1].tolist() == [0, -100, 0]


def test_choice_ties_ends_and_nan():
    s = np.array([1.0, 5.0, 5.0, np.nan, 5.0, -1.0, 0.0])
    assert ob.choose(s, 2) == [1, 2]
    assert ob.choose(s, 3, first=1, last=1) == [0, 1, 6]
    assert ob.choose(s, 7) == list(range(7))
    assert ob.choose(s, 6) == [0, 1, 2, 4, 5, 6]
    assert ob.choose(s, 9) == list(range(7)) + [-1, -1]
    assert ob.choose(np.zeros(0), 2) == [-1, -1]


def test_lists_of_the_caller():
    assert ob.listed([4, 2, 4, 5, -1, 9, 6, 6], 8) == [4, 5, 6]
    assert ob.rows_of([1, 0], 16, 35) == list(range(16, 32)) + [32, 33, 34]


def test_all_blocks_are_all_rows_and_pieces_are_the_whole():
    g = np.random.default_rng(0)
    K, V, q = g.normal(size=(40, 6)), g.normal(size=(40, 6)), g.normal(size=(3, 2, 6))
    mask = op.causal_mask(3)
    want = op.attend_tokens(q, K, V, 37, mask, 0.4)
    at = ob.rows_of(ob.choose(ob.scores(q.reshape(-1, 6), ob.bounds(K[:37], 16, 1e30)), 5), 16, 37) + [37, 38, 39]
    assert at == list(range(40))
    assert np.allclose(op.attend_tokens(q, K[at], V[at], 37, mask, 0.4), want)
    two = [np.concatenate([x[:20], x[20:]]) for x in (K, V)]
    assert np.allclose(op.attend_tokens(q, *two, 37, mask, 0.4), want)
