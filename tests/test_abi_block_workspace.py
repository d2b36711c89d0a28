"""The workspace of chosen blocks holds for every shorter cache (no GPU: sizes, and calls that a misaligned workspace
ends on the host right after its size was found large enough)."""
import ctypes
import os

import pytest

from paper_2608_08878_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

UNSUPPORTED, WORKSPACE = 3, 6
MOST = 16384 * 16            # rows of the most blocks of 16 rows that a choice takes
Q, LIST, BOUNDS, ODD = 1 << 40, 1 << 44, 1 << 45, (1 << 46) + 8


def _select(dims, tok, pick, rows, ws_bytes):
    # (over 1024 blocks: such choices take a workspace whatever the lists)
    assert rows >= 1025 * 16
    kv, blocks = B.dc_kv(None, None, rows), B.dc_blocks(16, BOUNDS)
    return B.lib().dc_block_select(ctypes.byref(dims), ctypes.byref(kv), 0, ctypes.byref(tok), ctypes.byref(blocks),
                                   ctypes.byref(pick), Q, LIST, ODD, ws_bytes, None)


@pytest.mark.parametrize("batch,tokens", [(1, 1), (3, 2), (60, 1)])   # (few lists, and many)
def test_it_does_not_fall_where_a_choice_is_refused(batch, tokens):
    dims = B.dc_dims(batch, 1, 8, 8, 128, 400000, B.DC_BF16, 0, 0.0)
    tok, blocks, pick = B.dc_tokens(batch * tokens, tokens, None), B.dc_blocks(16, None), B.dc_pick(48, 1, 0, 0)
    lens = (20000, 200000, MOST - 16, MOST, MOST + 1, MOST + tokens, MOST + 16, MOST + 16 + tokens, 300001, 400000)
    sizes = [B.dc_block_workspace_bytes(dims, tok, blocks, pick, n) for n in lens]
    assert sizes == sorted(sizes) and sizes[0] > 0
    for n, have in zip(lens, sizes):
        for rows in (17000, 19999 - tokens, 150000, 250000, MOST - 16, MOST - 1, MOST, MOST + 15):
            if rows + tokens <= n:
                assert _select(dims, tok, pick, rows, have) == UNSUPPORTED, (n, rows)     # ODD, and large enough
        if n > 200000:
            assert _select(dims, tok, pick, 200000, 0) == WORKSPACE


def test_it_is_the_choice_s_where_the_attention_is_refused():
    # 8 million tokens: the attention's tiles are 2^24 workgroups, the choice's lists 2^22
    dims = B.dc_dims(4096, 1, 64, 8, 128, 21000, B.DC_BF16, 0, 0.0)
    tok, blocks, pick = B.dc_tokens(4096 * 2048, 2048, None), B.dc_blocks(16, None), B.dc_pick(48, 16, 0, 0)
    have = B.dc_block_workspace_bytes(dims, tok, blocks, pick, 20000)
    assert _select(dims, tok, pick, 20000 - 2048, have) == UNSUPPORTED
    assert _select(dims, tok, pick, 20000 - 2048, 0) == WORKSPACE
