"""Refusals of the entry points for shared rows and blocks of rows: status codes from the host, no device
work, host fields untouched (no GPU)."""
import ctypes
import os

import pytest

from paper_2608_08878_amd import binding as B

FAKE = 0x10000000       # a non-NULL pointer that validation failures never dereference
FAR = FAKE + (1 << 24)
ODD = FAKE + 8          # not a multiple of 16 bytes
BIG = 1 << 40           # a workspace of any size

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

NULL, SHAPE, UNSUPPORTED, CAPACITY, WORKSPACE, VALUE = 1, 2, 3, 4, 6, 8


def _dims(**kw):
    d = dict(batch=6, n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=300, dtype=B.DC_BF16,
             ent_window=64, scale=0.0)
    d.update(kw)
    return B.dc_dims(*[d[f] for f, _ in B.dc_dims._fields_])


def _tok(tokens=60, most=10, cu=None):
    return B.dc_tokens(tokens, most, cu)


def _kv(length=240, unit_len=None, k=FAKE, v=FAKE):
    return B.dc_kv(k, v, length, unit_len)


def _shared(kv=None, capacity=500, prefixes=2, members=3, first=None, no_kv=False):
    kv = kv or _kv(400)
    s = B.dc_shared(None if no_kv else ctypes.pointer(kv), capacity, prefixes, members, first)
    s.keep = kv
    return s


def shared(dims=None, kv=None, layer=1, tok=None, parent=None, s=None, no_s=False, q=FAKE, out=FAR, ws=FAKE, wsb=0):
    return B.lib().dc_shared_attention(ctypes.byref(dims or _dims()), ctypes.byref(kv or _kv()), layer,
                                       ctypes.byref(tok or _tok()), parent,
                                       None if no_s else ctypes.byref(s or _shared()), q, out, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(kv=_kv(k=None)), NULL), (dict(kv=_kv(v=None)), NULL),
    (dict(no_s=True), NULL), (dict(s=_shared(no_kv=True)), NULL), (dict(s=_shared(_kv(400, k=None))), NULL),
    (dict(s=_shared(_kv(400, v=None))), NULL), (dict(dims=_dims(head_dim=96)), UNSUPPORTED), (dict(layer=3), SHAPE),
    (dict(layer=-1), SHAPE), (dict(tok=_tok(61)), SHAPE), (dict(kv=_kv(291)), CAPACITY), (dict(kv=_kv(301)), SHAPE),
    (dict(s=_shared(_kv(501))), SHAPE), (dict(s=_shared(_kv(-1))), SHAPE), (dict(s=_shared(capacity=0)), SHAPE),
    (dict(s=_shared(prefixes=0)), SHAPE), (dict(s=_shared(members=0)), SHAPE), (dict(s=_shared(members=7)), SHAPE),
    (dict(s=_shared(members=2)), SHAPE),                                   # 2 x 2 sequences of 6 without offsets
    (dict(s=_shared(prefixes=(1 << 24) // 6 + 1, members=1, first=FAKE)), UNSUPPORTED),
    (dict(s=_shared(_kv(400, k=ODD))), UNSUPPORTED), (dict(s=_shared(_kv(400, v=ODD))), UNSUPPORTED),
    (dict(q=ODD), UNSUPPORTED), (dict(out=ODD), UNSUPPORTED), (dict(out=FAKE), UNSUPPORTED),
    (dict(out=FAKE + 1024), UNSUPPORTED), (dict(tok=_tok(257 * 6, 257), kv=_kv(10), parent=FAKE), UNSUPPORTED),
    (dict(wsb=0), WORKSPACE), (dict(ws=None, wsb=BIG), WORKSPACE), (dict(ws=ODD, wsb=BIG), UNSUPPORTED),
    (dict(s=_shared(first=FAKE, prefixes=1, members=6)), WORKSPACE)])      # valid but for the workspace
def test_shared_refuses(kw, status):
    assert shared(**kw) == status


def test_shared_workspace_is_exact_and_does_not_shrink():
    d, t, s = _dims(), _tok(), _shared()
    need = B.dc_shared_workspace_bytes(d, t, s, 250)
    assert need > 0 and shared(wsb=need - 1) == WORKSPACE
    last = 0
    for rows in (0, 1, 10, 200, 400):
        for most in (10, 100, 300):
            n = B.dc_shared_workspace_bytes(d, t, _shared(_kv(rows)), most)
            assert n >= (last if most == 10 else n0), (rows, most)
            n0 = n
        last = B.dc_shared_workspace_bytes(d, t, _shared(_kv(rows)), 10)
    assert B.dc_shared_workspace_bytes(d, t, _shared(members=9), 250) == 0
    assert B.dc_shared_workspace_bytes(d, t, s, 0) == 0
    assert B.dc_shared_workspace_bytes(_dims(batch=0), t, s, 10) == 0


def _blocks(rows=64, bounds=FAR + FAR):
    return B.dc_blocks(rows, bounds)


def bounds(dims=None, kv=None, b=None, start=0, no_b=False):
    return B.lib().dc_block_bounds(ctypes.byref(dims or _dims()), ctypes.byref(kv or _kv()),
                                   None if no_b else ctypes.byref(b or _blocks()), start, None)


@pytest.mark.parametrize("kw,status", [
    (dict(kv=_kv(k=None)), NULL), (dict(no_b=True), NULL), (dict(b=_blocks(bounds=None)), NULL),
    (dict(b=_blocks(48)), UNSUPPORTED), (dict(b=_blocks(256)), UNSUPPORTED), (dict(b=_blocks(0)), UNSUPPORTED),
    (dict(b=_blocks(bounds=ODD)), UNSUPPORTED), (dict(kv=_kv(k=ODD)), UNSUPPORTED), (dict(start=-1), SHAPE),
    (dict(start=241), SHAPE), (dict(kv=_kv(301)), SHAPE), (dict(kv=_kv(-1)), SHAPE), (dict(dims=_dims(batch=0)), SHAPE),
    (dict(dims=_dims(dtype=3)), UNSUPPORTED), (dict(b=_blocks(bounds=FAKE)), UNSUPPORTED),
    (dict(b=_blocks(bounds=FAKE - 1024)), UNSUPPORTED)])
def test_bounds_refuses(kw, status):
    assert bounds(**kw) == status


def test_bounds_without_a_complete_block_do_nothing():
    assert bounds(kv=_kv(63)) == 0
    assert bounds(start=192) == 0                      # 240 rows: blocks 0..2 are complete
    assert bounds(dims=_dims(capacity=63), kv=_kv(60), b=_blocks(bounds=None)) == 0


def _pick(count=4, share=1, first=1, last=1):
    return B.dc_pick(count, share, first, last)


def select(dims=None, kv=None, layer=1, tok=None, b=None, p=None, q=FAKE, lst=FAR, no_b=False, no_p=False, no_kv=False):
    return B.lib().dc_block_select(ctypes.byref(dims or _dims()), None if no_kv else ctypes.byref(kv or _kv()), layer,
                                   ctypes.byref(tok or _tok()), None if no_b else ctypes.byref(b or _blocks()),
                                   None if no_p else ctypes.byref(p or _pick()), q, lst, None, 0, None)


def attention(dims=None, kv=None, layer=1, tok=None, b=None, p=None, q=FAKE, lst=FAKE, out=FAR, ws=None, wsb=0,
              no_b=False, no_p=False):
    return B.lib().dc_block_attention(ctypes.byref(dims or _dims()), ctypes.byref(kv or _kv()), layer,
                                      ctypes.byref(tok or _tok()), None if no_b else ctypes.byref(b or _blocks()),
                                      None if no_p else ctypes.byref(p or _pick()), lst, q, out, ws, wsb, None)


COMMON = [(dict(q=None), NULL), (dict(lst=None), NULL), (dict(no_b=True), NULL), (dict(no_p=True), NULL),
          (dict(q=ODD), UNSUPPORTED), (dict(lst=FAKE + 2), UNSUPPORTED), (dict(layer=3), SHAPE), (dict(layer=-1), SHAPE),
          (dict(tok=_tok(61)), SHAPE), (dict(b=_blocks(8)), UNSUPPORTED), (dict(p=_pick(0, first=0, last=0)), SHAPE),
          (dict(p=_pick(share=0)), SHAPE), (dict(p=_pick(2049)), UNSUPPORTED), (dict(p=_pick(4, first=3, last=2)), VALUE),
          (dict(p=_pick(first=-1)), VALUE), (dict(p=_pick(last=-1)), VALUE), (dict(p=_pick(last=2**31 - 1)), VALUE),
          (dict(kv=_kv(301)), SHAPE), (dict(kv=_kv(-1)), SHAPE), (dict(dims=_dims(n_q_heads=6)), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(no_kv=True), NULL), (dict(b=_blocks(bounds=None)), NULL), (dict(b=_blocks(bounds=ODD)), UNSUPPORTED),
    (dict(lst=FAKE + 60 * 2048 - 4), UNSUPPORTED), (dict(b=_blocks(bounds=FAR)), UNSUPPORTED),       # overlaps
    (dict(dims=_dims(capacity=70000), kv=_kv(70000)), WORKSPACE),          # few lists of many blocks
    (dict(dims=_dims(capacity=16385 * 16), kv=_kv(16385 * 16), b=_blocks(16)), UNSUPPORTED)])
def test_select_refuses(kw, status):
    assert select(**kw) == status


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(out=None), NULL), (dict(kv=_kv(k=None)), NULL), (dict(kv=_kv(v=None)), NULL), (dict(out=ODD), UNSUPPORTED),
    (dict(out=FAKE), UNSUPPORTED), (dict(out=FAKE + 512), UNSUPPORTED), (dict(kv=_kv(291)), CAPACITY),
    (dict(lst=FAR + 16), UNSUPPORTED), (dict(lst=FAR - 16), UNSUPPORTED), (dict(kv=_kv(v=ODD)), UNSUPPORTED), (dict(wsb=0), WORKSPACE), (dict(ws=ODD, wsb=BIG), UNSUPPORTED)])
def test_attention_refuses(kw, status):
    assert attention(**kw) == status


def test_block_workspace():
    d, t, b = _dims(), _tok(), _blocks()
    need = B.dc_block_workspace_bytes(d, t, b, _pick(), 250)
    assert need > 0 and attention(ws=FAKE, wsb=need - 1) == WORKSPACE
    sizes = [B.dc_block_workspace_bytes(d, t, b, _pick(), n) for n in (10, 11, 80, 200, 300, 5000, 100000)]
    assert sizes == sorted(sizes)
    for bad in ((_dims(batch=0), t, b, _pick(), 250), (d, t, _blocks(7), _pick(), 250), (d, t, b, _pick(0), 250),
                (d, t, b, _pick(), 9)):
        assert B.dc_block_workspace_bytes(*bad) == 0
