"""The workspace of shared attention: none where the prompts' own tiles leave no parts (no GPU: sizes, and calls that
end on the host for their workspace)."""
import ctypes
import os

import pytest

from paper_2608_08878_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

FAR = 1 << 44


def _call(batch, most, heads=32, kv=8, D=128, dtype=B.DC_BF16, tokens=None, prefixes=1, members=None, plen=16384, rows=0):
    dims = B.dc_dims(batch, 1, heads, kv, D, rows + most, dtype, 0, 0.0)
    tok = B.dc_tokens(tokens or batch * most, most, FAR if tokens else None)
    pkv = B.dc_kv(None, None, plen)
    sh = B.dc_shared(ctypes.pointer(pkv), plen + 1, prefixes, members or batch // prefixes, FAR if members else None)
    sh.keep = pkv
    return dims, tok, sh


def _bytes(*args, rows=0, **kw):
    dims, tok, sh = _call(*args, rows=rows, **kw)
    return B.dc_shared_workspace_bytes(dims, tok, sh, rows + tok.max_tokens)


@pytest.mark.parametrize("kw", [
    dict(batch=8, most=2048), dict(batch=16, most=8192, plen=8192), dict(batch=8, most=512), dict(batch=8, most=2048, rows=5000),
    dict(batch=8, most=2048, plen=200000), dict(batch=8, most=2048, plen=1), dict(batch=6, most=4096, prefixes=3),
    dict(batch=16, most=4096, tokens=50000), dict(batch=8, most=8192, heads=8, D=64, dtype=B.DC_F32)])
def test_whole_tiles_of_prompts_take_none(kw):
    kw = dict(kw)
    assert _bytes(kw.pop("batch"), kw.pop("most"), **kw) == 0


@pytest.mark.parametrize("kw", [
    dict(batch=8, most=1), dict(batch=8, most=64), dict(batch=2, most=512),            # few tiles: parts fill the card
    dict(batch=2000, most=1), dict(batch=200, most=33),                              # many, mostly empty
    dict(batch=16, most=4096, members=4, tokens=60000)])                             # most sequences have no prefix
def test_others_take_the_parts(kw):
    kw = dict(kw)
    assert _bytes(kw.pop("batch"), kw.pop("most"), **kw) > 0


def test_a_call_with_parts_refuses_less():
    dims, tok, sh = _call(8, 64)
    sh.kv.contents.k = sh.kv.contents.v = FAR
    kv = B.dc_kv(2 * FAR, 3 * FAR, 0)
    need = B.dc_shared_workspace_bytes(dims, tok, sh, 64)
    for ws, n, want in ((None, need, 6), (FAR, need - 1, 6), (FAR + 8, need, 3)):
        assert B.lib().dc_shared_attention(ctypes.byref(dims), ctypes.byref(kv), 0, ctypes.byref(tok), None,
                                           ctypes.byref(sh), 4 * FAR, 5 * FAR, ws, n, None) == want
