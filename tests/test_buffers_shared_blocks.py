"""What the wrappers for shared rows and blocks refuse before any launch (no GPU)."""
import pytest
import torch

from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers, make_shared


def _buffers(batch=4, heads=4, kv=1, cap=40, **kw):
    return DecodeBuffers(batch, 1, heads, kv, 128, cap, features=False, device="cpu", **kw)


def _heads(n, h):
    return torch.zeros((n, h, 128), dtype=torch.bfloat16)


TOK = B.dc_tokens(4, 1, None)


@pytest.mark.parametrize("members", [[4], [1, 2, 1], [3, -1], [0, 0], [1 << 23, 1 << 23]])
def test_members_that_are_no_members_are_refused(members):
    with pytest.raises(ValueError, match="members"):
        make_shared(_buffers(2), members)


def test_prefixes_of_other_heads_types_or_sequences_are_refused():
    buf = _buffers()
    for pre in (_buffers(2, heads=8), _buffers(2, kv=2), _buffers(2, dtype="f32"),
                DecodeBuffers(2, 2, 4, 1, 128, 40, features=False, device="cpu")):
        with pytest.raises(ValueError, match="layers, heads"):
            buf.shared_attention(TOK, make_shared(pre, 2), _heads(4, 4))
    for members in ([3, 2], 1, 3):
        with pytest.raises(ValueError, match="sequences"):
            buf.shared_attention(TOK, make_shared(_buffers(2), members), _heads(4, 4))


def test_prefixes_and_blocks_of_another_device_are_refused():
    buf, shared = _buffers(), make_shared(_buffers(2), 2)
    shared.device = 5
    with pytest.raises(ValueError, match="device"):
        buf.shared_attention(TOK, shared, _heads(4, 4))
    if not torch.cuda.is_available():
        return
    other = DecodeBuffers(4, 1, 4, 1, 128, 40, features=False)
    with pytest.raises(ValueError):
        buf.block_bounds(other.make_blocks(16))


def test_blocks_of_another_cache_and_of_other_sizes_are_refused():
    buf = _buffers()
    for rows in (0, 8, 20, 256):
        with pytest.raises(ValueError, match="blocks"):
            buf.make_blocks(rows)
    assert buf.make_blocks(16).bounds_tensor.shape == (4, 2, 2, 128)
    assert buf.make_blocks(64).bounds is None                # a cache of less than a block
    for other in (_buffers(3), _buffers(cap=64), _buffers(dtype="f32"), _buffers(kv=2)):
        with pytest.raises(ValueError, match="another cache"):
            buf.block_bounds(other.make_blocks(16))
        with pytest.raises(ValueError, match="another cache"):
            buf.block_select(TOK, other.make_blocks(16), _heads(4, 4), 2)


def test_queries_lists_and_counts_are_checked():
    buf = _buffers()
    blocks = buf.make_blocks(16)
    with pytest.raises(ValueError, match="q must"):
        buf.block_select(TOK, blocks, _heads(3, 4), 2)
    with pytest.raises(ValueError, match="q must"):
        buf.block_attention(TOK, blocks, torch.zeros((4, 1, 1, 2), dtype=torch.int32), _heads(4, 4).float())
    for kw in (dict(count=0), dict(count=2, share=0)):
        with pytest.raises(ValueError, match="at least 1"):
            buf.block_select(TOK, blocks, _heads(4, 4), **kw)
    for chosen in (torch.zeros((4, 1, 2), dtype=torch.int32), torch.zeros((4, 2, 1, 2), dtype=torch.int32),
                   torch.zeros((4, 1, 1, 2)), torch.zeros((4, 1, 1, 4), dtype=torch.int32)[..., ::2]):
        with pytest.raises(ValueError, match="chosen"):
            buf.block_attention(TOK, blocks, chosen, _heads(4, 4))
    with pytest.raises(ValueError, match="out"):
        buf.block_select(TOK, blocks, _heads(4, 4), 2, out=torch.zeros((4, 1, 1, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="parent"):
        buf.shared_attention(TOK, make_shared(_buffers(2), 2), _heads(4, 4), parent=torch.zeros(3, dtype=torch.int32))


def test_a_prefix_that_moved_is_followed():
    pre = _buffers(2)
    shared = make_shared(pre, 2)
    pre.cap = 30
    pre.kv.len = 12
    shared.update()
    assert shared.capacity == 30 and shared.kv.contents.len == 12
