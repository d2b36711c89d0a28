"""Several tokens at once on the GPU: what a cache and its buffers keep from call to call."""
import pytest
import torch

from .test_gpu_prompt import Cache

pytestmark = pytest.mark.gpu


def test_a_captured_attention_keeps_its_workspace():
    # outgrown after the capture, with memory of its size taken by others since
    c = Cache([9], 3000, "bf16", 128, 2, 4, seed=50)
    want = c.buf.prompt_attention(c.tokens, c.q)
    assert c.buf.ws_bytes > 0
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.buf.prompt_attention(c.tokens, c.q, out=out)
    size = c.buf.ws_bytes
    c.buf.reserve_workspace(200000)
    assert c.buf.ws_bytes > size
    taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all((x == 255).all() for x in taken)
        assert torch.equal(c.buf.prompt_attention(c.tokens, c.q), want)     # eager, in the present one
