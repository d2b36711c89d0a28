"""What the wrappers for several tokens at once refuse before any launch (no GPU)."""
import pytest
import torch

from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers, make_rope, make_tokens


def _buffers():
    return DecodeBuffers(2, 1, 4, 1, 128, 40, features=False, device="cpu")


def _heads(n, h):
    return torch.zeros((n, h, 128), dtype=torch.bfloat16)


def test_vectors_in_host_memory_are_refused():
    for kw in (dict(inv_freq=torch.zeros(64)), dict(q_gain=torch.zeros(128)), dict(k_gain=torch.zeros(128))):
        with pytest.raises(ValueError, match="GPU"):
            make_rope(norm=True, **kw)


def test_offsets_in_host_memory_are_refused():
    for counts in ([3, 4], [4, 4]):
        with pytest.raises(ValueError, match="GPU"):
            make_tokens(counts, device="cpu")


@pytest.mark.parametrize("counts", [[], [3, -1], [1 << 30, 1 << 30]])
def test_counts_that_are_no_counts_are_refused(counts):
    with pytest.raises(ValueError, match="counts"):
        make_tokens(counts)


@pytest.mark.parametrize("length", [64, 127, 129, 256])
def test_gains_of_another_length_are_refused(length):
    buf, tokens = _buffers(), B.dc_tokens(2, 1, None)
    rope = B.dc_rope(1, 1e-6, 0x10000, 0x10000, 0, 0, None)
    rope.gain_len = length                 # as make_rope notes it
    with pytest.raises(ValueError, match="gains"):
        buf.norm_rope(tokens, rope, _heads(2, 4), _heads(2, 1))


def test_vectors_and_offsets_of_another_device_are_refused():
    buf = _buffers()
    rope, tokens = B.dc_rope(1, 1e-6, None, None, 0, 0, None), B.dc_tokens(2, 1, None)
    rope.device = 5
    with pytest.raises(ValueError, match="rotation"):
        buf.norm_rope(tokens, rope, _heads(2, 4), _heads(2, 1))
    tokens.device = 5
    calls = (lambda: buf.norm_rope(tokens, B.dc_rope(), _heads(2, 4), _heads(2, 1)),
             lambda: buf.prompt_attention(tokens, _heads(2, 4)),
             lambda: buf.tree_attention(tokens, torch.zeros(2, dtype=torch.int32), _heads(2, 4)),
             lambda: buf.commit_rows(tokens))
    for call in calls:
        with pytest.raises(ValueError, match="offsets"):
            call()
