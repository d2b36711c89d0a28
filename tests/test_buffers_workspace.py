"""Growth of the workspace that a DecodeBuffers keeps (host memory, no GPU)."""
import os
import weakref

import pytest

from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")


def _buffers():
    return DecodeBuffers(1, 1, 32, 8, 128, 40000, features=False, device="cpu")


def test_outgrown_workspaces_stay_alive():
    # a captured graph holds their addresses
    buf, seen = _buffers(), []
    for n in (100, 5000, 40000):
        buf.reserve_workspace(n)
        seen.append((weakref.ref(buf.ws), buf.ws.data_ptr()))
    buf.reserve_tokens_workspace(B.dc_tokens(2000, 2000, None), 40000)
    assert len({p for _, p in seen}) == 3
    assert all(r() is not None and r().data_ptr() == p for r, p in seen)


def test_they_add_up_to_less_than_the_present_one():
    buf, refs = _buffers(), []
    for n in range(64, 40000, 128):                       # a prompt in parts, each behind a longer cache
        buf.reserve_tokens_workspace(B.dc_tokens(200, 200, None), n + 200)
        if buf.ws is not None and not any(r() is buf.ws for r in refs):
            refs.append(weakref.ref(buf.ws))
    held = [r().numel() for r in refs if r() is not None]
    assert sum(held) < 2 * buf.ws_bytes == 2 * held[-1]
    need = B.dc_tokens_workspace_bytes(buf.dims, B.dc_tokens(200, 200, None), 40000)
    assert need <= buf.ws_bytes and buf.ws.data_ptr() % 16 == 0


def test_the_bound_of_the_rows_comes_down_to_the_longest_unit():
    buf = DecodeBuffers(2, 1, 8, 2, 64, 100, features=False, ragged=True, device="cpu")
    buf.kv.len = 90
    buf.unit_len[:] = 40
    buf.unit_len[2] = 63
    assert buf.tighten_len() == 63 == buf.kv.len
    buf.unit_len[2] = 95                                # past the bound: calls clamp to it
    assert buf.tighten_len() == 63
    buf.unit_len.zero_()
    assert buf.tighten_len() == 0
    even = DecodeBuffers(1, 1, 8, 2, 64, 100, features=False, device="cpu")
    even.kv.len = 12
    assert even.tighten_len() == 12


def test_float32_heads_of_128_are_cut_for_one_workgroup_a_cu():
    # 300 tokens of 32/8 heads: 80 tiles of 128 rows; the parts' outputs and statistics in float32
    dims = B.dc_dims(1, 1, 32, 8, 128, 20000, B.DC_F32, 0, 0.0)
    each = 300 * 32 * (128 + 2) * 4
    for rows in (5000, 16300):
        assert 0 < B.dc_tokens_workspace_bytes(dims, B.dc_tokens(300, 300, None), rows) <= 256 // 80 * each + 255
