"""Bounds of a ragged cache over parts of prompts and steps: from the shortest unit's rows on, every unit's are current."""
import numpy as np
import pytest
import torch

from oracle import blocks as ob
from paper_2608_08878_amd.buffers import DecodeBuffers, make_rope, make_tokens

from .test_gpu_shared_blocks import np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,rows", [("bf16", 128, 16), ("f32", 64, 32), ("bf16", 64, 64)])
def test_every_unit_s_bounds_are_current_after_each_part(dtype, D, rows):
    g = torch.Generator().manual_seed(rows)
    td, hk, G, layers, batch = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype], 2, 2, 2, 4
    buf = DecodeBuffers(batch, layers, hk * G, hk, D, 900, dtype, features=False, ragged=True)
    blocks, rope = buf.make_blocks(rows), make_rope(10000.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2)))
    blocks.bounds_tensor.fill_(9)
    have = [0] * batch                                     # every sequence's rows: the caller's own count
    for counts in ([70, 200, 3, 129], [1, 1, 1, 1], [0, 100, 60, 1], [1, 0, 1, 1], [64, 64, 64, 64], [1, 1, 1, 1]):
        tok, n = make_tokens(counts), sum(counts)
        pos = torch.cat([torch.arange(h, h + c, dtype=torch.int32) for h, c in zip(have, counts)]).cuda()
        for layer in range(layers):
            x = torch.randn((n, (hk * G + 2 * hk) * D), generator=g).to(td).cuda().unflatten(1, (hk * G + 2 * hk, D))
            buf.prefill(tok, rope, x[:, :hk * G], x[:, hk * G:hk * G + hk], x[:, hk * G + hk:], pos, layer)
        buf.commit_rows(tok)
        buf.block_bounds(blocks, min(have))
        have = [h + c for h, c in zip(have, counts)]
        got = np64(blocks.bounds_tensor)
        per = hk * layers
        for u in range(batch * per):
            m = have[u // per]
            assert int(buf.unit_len[u]) == m
            want = ob.bounds(np64(buf.k[u, :m]), rows, float(torch.finfo(td).max))
            assert np.array_equal(got[u, :m // rows], want), (u, m)
            assert (got[u, m // rows:] == 9).all()
