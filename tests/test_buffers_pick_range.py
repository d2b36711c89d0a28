"""Counts of a choice that do not fit the C structs' 32 bits are refused, not cut off (no GPU)."""
import os

import pytest
import torch

from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

TOK = B.dc_tokens(12, 3, None)


@pytest.mark.parametrize("big", [2**31, 2**32, 2**32 + 1, 2**40 + 3, -2**31 - 1])
def test_numbers_past_32_bits_are_refused(big):
    # (a share of 2^32 + 1 would be 1 to the kernel: lists for every token into room for one of each sequence)
    buf = DecodeBuffers(4, 1, 4, 1, 128, 40, features=False, device="cpu")
    blocks, q = buf.make_blocks(16), torch.zeros((12, 4, 128), dtype=torch.bfloat16)
    lists = torch.zeros((4, 1, 1, 2), dtype=torch.int32)
    for name in ("share", "first", "last"):
        with pytest.raises(ValueError, match=name if big > 0 or name != "share" else "at least 1"):
            buf.block_select(TOK, blocks, q, 2, **{name: big})
    with pytest.raises(ValueError, match="count"):
        buf.block_select(TOK, blocks, q, big)
    with pytest.raises(ValueError, match="share"):
        buf.block_attention(TOK, blocks, lists, q, share=big)
    with pytest.raises(ValueError, match="share|at least 1"):
        buf.sparse_attention(TOK, blocks, q, 2, share=big)
    with pytest.raises(ValueError, match="share"):
        buf.reserve_block_workspace(TOK, blocks, 2, 30, share=big)
    with pytest.raises(ValueError, match="start"):
        buf.block_bounds(blocks, big)
