"""Blocks of a cache's rows: bounds of their keys, the choice of blocks, and which rows a token then
sees; and rows that sequences have in common, in binary64.

Test infrastructure only (see ``oracle/__init__``).

* bounds: element by element the largest and smallest of a complete block's keys, infinite ones and NaN
  as the type's largest finite number of their sign;
* score of a block for a group of queries: sum of max(q_e hi_e, q_e lo_e) over queries and elements;
* choice: the first and last blocks, then the highest scores, ties to the lower number, NaN lowest;
* attention: chosen rows, or a prefix's, are rows like any other before the tokens (``prompt.attend_tokens``).

Parity pinned by: no logit above its block's bound, a choice of all blocks being plain attention, the
order under ties and NaN, rows in two pieces being the rows in one.
"""
from __future__ import annotations

import numpy as np


def bounds(K, rows, top):
    """K (n, d) -> (n // rows, 2, d); top: the type's largest finite number."""
    K = np.asarray(K, np.float64)
    n = len(K) // rows
    x = np.where(np.isnan(K), np.copysign(top, K), np.clip(K, -top, top))[:n * rows]
    x = x.reshape(n, rows, K.shape[1])
    return np.stack([x.max(1), x.min(1)], 1)


def scores(q, bound):
    """q (queries, d) of one group and KV head, bound (blocks, 2, d) -> (blocks,)."""
    q = np.asarray(q, np.float64)
    up, down = np.where(q < 0, 0, q).sum(0), np.where(q > 0, 0, q).sum(0)
    return bound[:, 0] @ up + bound[:, 1] @ down


def choose(score, count, first=0, last=0):
    """The chosen blocks, ascending, padded with -1."""
    n = len(score)
    held = [j for j in range(n) if j < first or j >= n - last]
    value = [-np.inf if np.isnan(s) else s for s in score]
    rest = sorted(set(range(n)) - set(held), key=lambda j: (bool(np.isnan(score[j])), -value[j], j))
    out = sorted((held + rest)[:count])
    return out + [-1] * (count - len(out))


def listed(entries, complete):
    """The blocks that count of a caller's list: those that exist and are above all such before them."""
    out = []
    for j in entries:
        if 0 <= j < complete and (not out or j > out[-1]):
            out.append(int(j))
    return out


def rows_of(entries, rows, length):
    """Rows before the tokens that a group sees: the chosen blocks' and those behind the last complete one."""
    complete = length // rows
    picked = [r for j in listed(entries, complete) for r in range(j * rows, (j + 1) * rows)]
    return picked + list(range(complete * rows, length))
