"""Several tokens at once: norm and rotation of heads, attention of prompts and of trees
of drafted tokens, and which rows an accepted path leaves, in binary64.

Test infrastructure only (see ``oracle/__init__``).

* norm: x / sqrt(mean(x^2) + eps) * gain over a head;
* rotation: pair i of the first R elements, (i, i + R/2) or interleaved (2i, 2i+1), times
  exp(j pos f_i) as a complex number;
* attention: token r of a sequence with `rows` rows before it sees those and, of the
  sequence's own rows, the set its mask row gives; weights and outputs as ``attention.attend``;
* a tree's mask: node i sees itself and what its parent sees, if that is an earlier node.

Parity pinned by: norms kept and relative angles under rotation, the two ways to pair,
a chain's mask equal to the causal one, attend() per token.
"""
from __future__ import annotations

import numpy as np

from . import attention


def norm_rope(x, pos, inv_freq, gain=None, norm=True, eps=1e-6, interleaved=False):
    """x (N, heads, d) -> binary64 of the same shape."""
    y = np.array(x, np.float64)
    if norm:
        y /= np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps)
        if gain is not None:
            y *= np.asarray(gain, np.float64)
    half = 0 if inv_freq is None else len(inv_freq)
    if half:
        turn = np.exp(1j * np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64))
        a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
        b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
        z = (y[..., a] + 1j * y[..., b]) * turn
        y[..., a], y[..., b] = z.real, z.imag
    return y


def causal_mask(n):
    return np.tril(np.ones((n, n), bool))


def tree_mask(parent):
    n = len(parent)
    m = np.zeros((n, n), bool)
    for i, p in enumerate(parent):
        if 0 <= p < i:
            m[i] = m[p]
        m[i, i] = True
    return m


def attend_tokens(q, K, V, rows, mask, scale):
    """q (n, G, d) of one unit's sequence over K, V (rows + n, d); mask (n, n) -> (n, G, d)."""
    out = np.empty(np.shape(q), np.float64)
    for r in range(len(q)):
        see = np.concatenate([np.ones(rows, bool), mask[r]])
        out[r] = attention.attend(q[r], np.asarray(K)[see], np.asarray(V)[see], scale).o
    return out


def kept_rows(n, path, keep, width):
    """Tokens (numbers within the sequence) whose rows are kept, in order."""
    m = min(n, width)
    if keep is not None:
        m = min(max(int(keep), 0), m)
    return [j if path is None else min(max(int(path[j]), j), n - 1) for j in range(m)]
