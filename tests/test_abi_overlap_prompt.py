"""Outputs of prompt and tree attention inside what the call reads are refused: the cache's rows, lengths, offsets
and parents (no GPU)."""
import os

import pytest

from paper_2608_08878_amd import binding as B

from .test_abi_prompt import _dims, _tok, attend

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

UNSUPPORTED, WORKSPACE = 3, 6
K, V, LENS, CU, PARENT, Q, WS = (x << 32 for x in range(16, 23))      # far apart
DIMS = dict(capacity=50000)                                # (caches long enough for parts, which take a workspace)
OUT, CACHE = 20 * 8 * 128 * 2, 12 * 50000 * 128 * 2        # bytes of 20 tokens' outputs, of a cache's keys


def _call(tree, out):
    return attend(tree, dims=_dims(**DIMS), kv=B.dc_kv(K, V, 40000, LENS), tok=_tok(cu=CU), q=Q, out=out,
                  parent=PARENT, ws=WS, wsb=1 << 31)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("at,size", [(K, CACHE), (V, CACHE), (LENS, 12 * 4), (CU, 3 * 4)])
def test_outputs_inside_the_cache_are_refused(tree, at, size):
    for out in (at - OUT + 16, at, at + size // 2 // 16 * 16, at + (size - 1) // 16 * 16):
        assert _call(tree, out) == UNSUPPORTED, hex(out)


def test_outputs_inside_the_parents_are_refused():
    for out in (PARENT - OUT + 16, PARENT, PARENT + 20 * 4 // 16 * 16 - 16):
        assert _call(True, out) == UNSUPPORTED, hex(out)
