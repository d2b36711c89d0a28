"""Pins of the binary64 oracle for several tokens at once (no GPU)."""
import numpy as np
import pytest

from oracle import attention as oatt
from oracle import prompt as op


def test_rotation_keeps_norms_and_relative_angles():
    g = np.random.default_rng(1)
    f = 10000.0 ** (-np.arange(8) / 8)
    x, y = g.standard_normal((2, 1, 1, 16))
    for inter in (False, True):
        def turn(v, p):
            return op.norm_rope(v, [p], f, norm=False, interleaved=inter)[0, 0]
        assert np.isclose(np.linalg.norm(turn(x, 77)), np.linalg.norm(x))
        # the product depends on the distance alone
        assert np.isclose(turn(x, 5) @ turn(y, 3), turn(x, 1005) @ turn(y, 1003))
        assert np.allclose(turn(x, 0), x[0, 0])


def test_one_pair_turns_by_its_angle():
    x = np.zeros((1, 1, 16))
    x[0, 0, 0] = 1.0
    half = op.norm_rope(x, [3], [0.5], norm=False)[0, 0]              # rot_dim 2: elements 0 and 1
    assert np.allclose(half[:2], [np.cos(1.5), np.sin(1.5)]) and not half[2:].any()
    f = np.full(8, 0.5)
    half, inter = (op.norm_rope(x, [3], f, norm=False, interleaved=i)[0, 0] for i in (False, True))
    assert np.isclose(half[8], np.sin(1.5)) and np.isclose(inter[1], np.sin(1.5))


def test_norm_has_unit_mean_square_times_gain():
    x = np.random.default_rng(2).standard_normal((3, 2, 64)) * 7
    assert np.allclose((op.norm_rope(x, None, None, eps=0.0) ** 2).mean(-1), 1.0)
    gain = np.arange(64.0)
    assert np.allclose(op.norm_rope(x, None, None, gain=gain), op.norm_rope(x, None, None) * gain)


@pytest.mark.parametrize("n", [1, 2, 9])
def test_a_chain_is_causal(n):
    assert np.array_equal(op.tree_mask(list(range(-1, n - 1))), op.causal_mask(n))


def test_tree_mask_by_hand():
    #      0        3 (a parent that comes later counts as none)
    #     / \
    #    1   2
    m = op.tree_mask([-1, 0, 0, 9])
    assert m.astype(int).tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [1, 0, 1, 0], [0, 0, 0, 1]]


def test_attend_tokens_is_attend_per_token():
    g = np.random.default_rng(3)
    q, K, V = g.standard_normal((3, 2, 8)), g.standard_normal((8, 8)), g.standard_normal((8, 8))
    o = op.attend_tokens(q, K, V, 5, op.causal_mask(3), 0.3)
    for r in range(3):
        assert np.allclose(o[r], oatt.attend(q[r], K[:6 + r], V[:6 + r], 0.3).o)


def test_kept_rows():
    assert op.kept_rows(5, None, None, 5) == [0, 1, 2, 3, 4]
    assert op.kept_rows(5, [0, 2, 4], 2, 3) == [0, 2]
    assert op.kept_rows(3, [-4, 0, 9, 9], None, 4) == [0, 1, 2]
    assert op.kept_rows(5, [1, 3], 7, 2) == [1, 3] and op.kept_rows(5, [1, 3], -1, 2) == []
