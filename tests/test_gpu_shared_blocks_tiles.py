"""Every tile shape of the attention over shared rows and chosen blocks against the binary64 oracle, with the helpers and
tolerances of test_gpu_shared_blocks: whole tiles of several waves, keys in parts and in one, rows that are read past
the caches, and unseen rows that are not finite.  That the sizes reach those tiles is a CPU test."""
import pytest
import torch

from oracle import blocks as ob

from . import plan_cases as C
from .test_gpu_shared_blocks import blocks_case, check_blocks, check_shared, shared_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("name", C.SHARED)
def test_shared_tiles(name, tree):
    dtype, D, hk, G, counts, members, plen, rows = C.SHARED[name][0]
    print(f"shared {name} tree={tree}", flush=True)
    buf, pre, tok, sh, q, pt, out, lens, plens = shared_case(counts, members, plen, rows, dtype, D, hk, G, tree=tree, seed=3)
    assert torch.equal(buf.shared_attention(tok, sh, q, pt), out)
    # rows that no token sees: behind the prefixes' and behind the tokens'
    for u, n in enumerate(plens):
        pre.k[u, n:], pre.v[u, n:] = float("nan"), float("inf")
    for u, n in enumerate(lens):
        m = counts[u // hk]
        buf.k[u, n + m:], buf.v[u, n + m:] = float("nan"), float("inf")
    again = buf.shared_attention(tok, sh, q, pt)
    # (where such a value met a weight of 0 the pass is repeated, with weights of at most 1)
    check_shared(again, buf, pre, counts, members, lens, plens, q, dtype, None if pt is None else pt.tolist())


@pytest.mark.parametrize("name", C.SHARED_ONCE)
def test_shared_tiles_of_rows_read_once(name):
    dtype, D, hk, G, counts, members, plen, rows = C.SHARED_ONCE[name][0]
    print(f"shared once {name}", flush=True)
    shared_case(counts, members, plen, rows, dtype, D, hk, G, seed=4)


@pytest.mark.parametrize("rough", [False, True])
@pytest.mark.parametrize("name", C.BLOCKS)
def test_block_tiles(name, rough):
    dtype, D, hk, G, counts, n, rows, count, share = C.BLOCKS[name][0]
    print(f"blocks {name} rough={rough}", flush=True)
    buf, blocks, tok, q, lens, lists, out = blocks_case(counts, n, rows, count, share, dtype, D, hk, G, seed=5, rough=rough)
    assert torch.equal(buf.block_attention(tok, blocks, lists, q, share), out)
    seen = lists.cpu().numpy()
    for u, m in enumerate(lens):                          # rows that no list of the unit names, and behind the tokens
        b, h = divmod(u, hk)
        used = {r for i in range(seen.shape[1]) for r in ob.rows_of(seen[b, i, h], rows, m)}
        free = [r for r in range(m) if r not in used] + list(range(m + counts[b], buf.cap))
        buf.k[u, free], buf.v[u, free] = float("nan"), float("inf")
    again = buf.block_attention(tok, blocks, lists, q, share)
    check_blocks(again, buf, counts, lens, lists, q, rows, share, dtype)


@pytest.mark.parametrize("name", C.BLOCKS_ONCE)
def test_block_tiles_of_rows_read_once(name):
    dtype, D, hk, G, counts, n, rows, count, share = C.BLOCKS_ONCE[name][0]
    print(f"blocks once {name}", flush=True)
    blocks_case(counts, n, rows, count, share, dtype, D, hk, G, seed=6)


def test_whole_prompts_take_no_workspace():
    buf, pre, tok, sh, q, _, out, lens, plens = shared_case([256] * 8, [8], 200, 0, "bf16", 64, 8, 8, seed=7, uneven=False)
    assert buf.ws is None and buf.ws_bytes == 0
    assert torch.equal(buf.shared_attention(tok, sh, q), out)
