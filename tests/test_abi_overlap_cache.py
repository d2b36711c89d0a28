"""Outputs inside what their call reads are refused: the caches' rows, lengths, parents and offsets (no GPU)."""
import os

import pytest

from paper_2608_08878_amd import binding as B

from .test_abi_shared_blocks import _blocks, _dims, _shared, _tok, attention, bounds, select, shared

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

UNSUPPORTED, WORKSPACE = 3, 6
K, V, PK, PV, LENS, PLENS, CU, FIRST, PARENT, LIST, Q, FREE = (x << 24 for x in range(16, 28))     # far apart
OUT = 60 * 8 * 128 * 2                                     # bytes of 60 tokens' outputs
CACHE, PREFIX = 36 * 300 * 128 * 2, 12 * 500 * 128 * 2     # of a cache's keys, of the prefixes'

KV = B.dc_kv(K, V, 240, LENS)


def _prefix(first=FIRST):
    return _shared(B.dc_kv(PK, PV, 400, PLENS), first=first)


def _across(at, size):
    """Outputs that begin before, within and at the end of an array."""
    return [at - OUT + 16, at, at + size // 2 // 16 * 16, at + (size - 1) // 16 * 16]


ARRAYS = {"keys": (K, CACHE), "values": (V, CACHE), "lengths": (LENS, 36 * 4), "offsets": (CU, 7 * 4)}


@pytest.mark.parametrize("name,at,size", [(n, *x) for n, x in {
    **ARRAYS, "prefix keys": (PK, PREFIX), "prefix values": (PV, PREFIX), "prefix lengths": (PLENS, 12 * 4),
    "members": (FIRST, 3 * 4), "parents": (PARENT, 60 * 4)}.items()])
def test_shared_refuses_outputs_inside_what_it_reads(name, at, size):
    for out in _across(at, size):
        assert shared(kv=KV, tok=_tok(cu=CU), s=_prefix(), parent=PARENT, q=Q, out=out) == UNSUPPORTED, hex(out)
    for out in (at - OUT, at + (size + 15) // 16 * 16):       # beside it: refused for the workspace alone
        assert shared(kv=KV, tok=_tok(cu=CU), s=_prefix(), parent=PARENT, q=Q, out=out) == WORKSPACE
    # a prefix without rows is not read
    empty = _shared(B.dc_kv(PK, PV, 0, PLENS), first=FIRST)
    need = B.dc_tokens_workspace_bytes(_dims(), _tok(cu=CU), 250)
    assert need > 0
    want = UNSUPPORTED if name in ARRAYS or name == "parents" else WORKSPACE
    assert shared(kv=KV, tok=_tok(cu=CU), s=empty, parent=PARENT, q=Q, out=at) == want


@pytest.mark.parametrize("name,at,size", [(n, *x) for n, x in ARRAYS.items()])
def test_chosen_blocks_refuse_outputs_inside_what_they_read(name, at, size):
    for out in _across(at, size):
        assert attention(kv=KV, tok=_tok(cu=CU), q=Q, lst=LIST, out=out) == UNSUPPORTED, hex(out)
    for out in (at - OUT, at + (size + 15) // 16 * 16):
        assert attention(kv=KV, tok=_tok(cu=CU), q=Q, lst=LIST, out=out) == WORKSPACE


def test_absent_arrays_meet_nothing():
    kv = B.dc_kv(K, V, 240, None)
    assert shared(kv=kv, s=_shared(B.dc_kv(PK, PV, 400, None)), q=Q, out=16) == WORKSPACE
    assert attention(kv=kv, q=Q, lst=LIST, out=16) == WORKSPACE


BOUNDS_BYTES, LIST_BYTES = 36 * 4 * 2 * 128 * 2, 6 * 10 * 2 * 4 * 4      # blocks of 64 of 300 rows; 4 of them for every token


@pytest.mark.parametrize("at,size", [(K, CACHE), (LENS, 36 * 4)])
def test_bounds_refuse_what_they_read(at, size):
    for b in (at - BOUNDS_BYTES + 16, at, at + (size - 1) // 16 * 16):
        assert bounds(kv=KV, b=_blocks(bounds=b)) == UNSUPPORTED, hex(b)


def _select(lst, **kw):
    # (a long cache, whose choice takes a workspace: no call goes on to a launch)
    return select(dims=_dims(capacity=70000), kv=B.dc_kv(None, None, 70000, LENS), tok=_tok(cu=CU), b=_blocks(bounds=1 << 36),
                  q=Q, lst=lst)


@pytest.mark.parametrize("at,size", [(LENS, 36 * 4), (CU, 7 * 4), (Q, OUT)])
def test_choices_refuse_what_they_read(at, size):
    for lst in (at - LIST_BYTES + 4, at, at + size - 4):
        assert _select(lst) == UNSUPPORTED, hex(lst)
    for lst in (at - LIST_BYTES, at + size):
        assert _select(lst) == WORKSPACE
