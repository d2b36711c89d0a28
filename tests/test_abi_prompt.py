"""Refusals of the entry points for several tokens at once: status codes from the host, no
device work, host fields untouched (no GPU)."""
import ctypes
import os

import pytest

from paper_2608_08878_amd import binding as B

FAKE = 0x10000          # a non-NULL pointer that validation failures never dereference
ODD = FAKE + 8          # not a multiple of 16 bytes

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")


def _dims(**kw):
    d = dict(batch=2, n_layers=3, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=100, dtype=B.DC_BF16,
             ent_window=64, scale=0.0)
    d.update(kw)
    return B.dc_dims(*[d[f] for f, _ in B.dc_dims._fields_])


def _tok(tokens=20, most=10, cu=None):
    return B.dc_tokens(tokens, most, cu)


def _kv(length=40, unit_len=None, k=FAKE, v=FAKE):
    return B.dc_kv(k, v, length, unit_len)


def _rope(**kw):
    d = dict(norm=1, eps=1e-6, q_gain=None, k_gain=None, rot_dim=128, interleaved=0, inv_freq=FAKE)
    d.update(kw)
    return B.dc_rope(*[d[f] for f, _ in B.dc_rope._fields_])


def rope(dims=None, kv=None, layer=1, tok=None, r=None, q=FAKE, ld_q=1536, k=FAKE, ld_k=1536, v=FAKE, ld_v=1536,
         pos=FAKE, q_out=FAKE + 64, k_out=None, no_kv=False):
    return B.lib().dc_qk_norm_rope(
        ctypes.byref(dims or _dims()), None if no_kv else ctypes.byref(kv or _kv()), layer,
        ctypes.byref(tok or _tok()), ctypes.byref(r or _rope()), q, ld_q, k, ld_k, v, ld_v, pos, q_out, k_out, None)


NULL, SHAPE, UNSUPPORTED, CAPACITY, WORKSPACE, VALUE = 1, 2, 3, 4, 6, 8


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(q_out=None), NULL), (dict(v=None), NULL),
    (dict(pos=None), NULL), (dict(no_kv=True), NULL), (dict(kv=_kv(k=None)), NULL), (dict(kv=_kv(v=None)), NULL),
    (dict(r=_rope(inv_freq=None)), NULL),
    (dict(dims=_dims(batch=0)), SHAPE), (dict(dims=_dims(head_dim=96)), UNSUPPORTED),
    (dict(dims=_dims(dtype=2)), UNSUPPORTED), (dict(layer=-1), SHAPE), (dict(layer=3), SHAPE),
    (dict(tok=_tok(0, 0)), SHAPE), (dict(tok=_tok(19, 10)), SHAPE), (dict(tok=_tok(20, 21, FAKE)), SHAPE),
    (dict(tok=_tok(21, 10, FAKE)), SHAPE), (dict(ld_q=1023), SHAPE), (dict(ld_k=255), SHAPE), (dict(ld_v=255), SHAPE),
    (dict(ld_q=1540), UNSUPPORTED), (dict(ld_k=1540), UNSUPPORTED), (dict(ld_v=1540), UNSUPPORTED),
    (dict(q=ODD), UNSUPPORTED), (dict(k=ODD), UNSUPPORTED), (dict(v=ODD), UNSUPPORTED), (dict(q_out=ODD), UNSUPPORTED),
    (dict(k_out=ODD), UNSUPPORTED), (dict(kv=_kv(k=ODD)), UNSUPPORTED), (dict(kv=_kv(v=ODD)), UNSUPPORTED),
    (dict(q_out=FAKE), UNSUPPORTED), (dict(k_out=FAKE), UNSUPPORTED),      # in place on parts of wider rows
    (dict(r=_rope(norm=2)), VALUE), (dict(r=_rope(interleaved=-1)), VALUE), (dict(r=_rope(eps=-1.0)), VALUE),
    (dict(r=_rope(eps=float("nan"))), VALUE), (dict(r=_rope(eps=float("inf"))), VALUE),
    (dict(r=_rope(rot_dim=-16)), SHAPE), (dict(r=_rope(rot_dim=144)), SHAPE), (dict(r=_rope(rot_dim=24)), UNSUPPORTED),
    (dict(kv=_kv(-1)), SHAPE), (dict(kv=_kv(101)), SHAPE), (dict(kv=_kv(91)), CAPACITY)])
def test_norm_rope_refuses(kw, status):
    assert rope(**kw) == status


def attend(tree, dims=None, kv=None, layer=1, tok=None, q=FAKE, out=FAKE + 64, parent=FAKE, ws=None, wsb=0):
    L, d, c, t = B.lib(), ctypes.byref(dims or _dims()), ctypes.byref(kv or _kv()), ctypes.byref(tok or _tok())
    if tree:
        return L.dc_tree_attention(d, c, layer, t, parent, q, out, ws, wsb, None)
    return L.dc_prompt_attention(d, c, layer, t, q, out, ws, wsb, None)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(kv=_kv(k=None)), NULL), (dict(kv=_kv(v=None)), NULL),
    (dict(dims=_dims(n_q_heads=6, n_kv_heads=4)), SHAPE), (dict(dims=_dims(n_q_heads=6, n_kv_heads=2)), UNSUPPORTED),
    (dict(layer=3), SHAPE), (dict(layer=-1), SHAPE), (dict(tok=_tok(20, 0)), SHAPE), (dict(tok=_tok(-1, 10)), SHAPE),
    (dict(tok=_tok(10, 10)), SHAPE), (dict(kv=_kv(91)), CAPACITY), (dict(q=ODD), UNSUPPORTED),
    (dict(out=ODD), UNSUPPORTED), (dict(out=FAKE), UNSUPPORTED), (dict(kv=_kv(k=ODD)), UNSUPPORTED)])
def test_attention_refuses(tree, kw, status):
    assert attend(tree, **kw) == status


def test_tree_refuses_missing_parents_and_too_many_nodes():
    assert attend(True, parent=None) == NULL
    big = _dims(capacity=1000)
    assert attend(True, dims=big, tok=_tok(514, 257)) == UNSUPPORTED


def test_attention_needs_its_workspace():
    dims, tok, kv = _dims(capacity=50000), _tok(), _kv(40000)
    need = B.dc_tokens_workspace_bytes(dims, tok, 40010)
    assert need > 0
    for tree in (False, True):
        assert attend(tree, dims=dims, tok=tok, kv=kv) == WORKSPACE
        assert attend(tree, dims=dims, tok=tok, kv=kv, ws=FAKE, wsb=need - 1) == WORKSPACE
        assert attend(tree, dims=dims, tok=tok, kv=kv, ws=ODD, wsb=need) == UNSUPPORTED
    assert B.dc_tokens_workspace_bytes(_dims(batch=0), tok, 100) == 0
    assert B.dc_tokens_workspace_bytes(dims, _tok(0, 0), 100) == 0
    assert B.dc_tokens_workspace_bytes(dims, tok, 0) == 0


def test_sizes_past_the_grid_are_refused():
    assert rope(dims=_dims(capacity=1 << 26), tok=_tok(1 << 26, 1 << 25)) == UNSUPPORTED
    # 4096 sequences x 2 KV heads x 3125 tiles of 128 rows
    big = _dims(batch=4096, capacity=1 << 20)
    for tree in (False, True):
        assert attend(tree, dims=big, tok=_tok(1 << 20, 100000, FAKE), ws=FAKE, wsb=1 << 60) == UNSUPPORTED
    assert B.dc_tokens_workspace_bytes(big, _tok(1 << 20, 100000, FAKE), 1 << 20) == 0


def test_workspace_for_longer_caches_covers_shorter_ones():
    for dtype in (B.DC_F32, B.DC_BF16):
        for batch, hk, n in ((1, 1, 1), (1, 8, 13), (2, 2, 300), (16, 8, 32)):
            dims = _dims(batch=batch, n_kv_heads=hk, n_q_heads=4 * hk, capacity=1 << 20, dtype=dtype)
            tok = _tok(batch * n, n)
            sizes = [B.dc_tokens_workspace_bytes(dims, tok, x) for x in range(n, 40000, 117)]
            assert sizes == sorted(sizes), (dtype, batch, hk, n)


def commit(dims=None, kv=None, feat=None, tok=None, path=None, keep=None, width=10):
    kv, f = kv or _kv(), feat
    st = B.lib().dc_commit_rows(ctypes.byref(dims or _dims()), ctypes.byref(kv),
                                ctypes.byref(f) if f is not None else None, ctypes.byref(tok or _tok()), path, keep,
                                width, None)
    return st, kv.len


@pytest.mark.parametrize("kw,status", [
    (dict(kv=_kv(k=None)), NULL), (dict(feat=B.dc_feat(None, FAKE, FAKE, FAKE, FAKE)), NULL),
    (dict(tok=_tok(15, 10, FAKE)), NULL), (dict(keep=FAKE), NULL),            # differing counts take a ragged cache
    (dict(width=0), SHAPE), (dict(width=11), SHAPE), (dict(tok=_tok(19, 10)), SHAPE),
    (dict(kv=_kv(95)), CAPACITY), (dict(kv=_kv(101)), SHAPE),
    (dict(dims=_dims(capacity=1000), tok=_tok(600, 300), path=FAKE), UNSUPPORTED)])
def test_commit_refuses(kw, status):
    kv = kw.get("kv") or _kv()
    before = kv.len
    assert commit(**{**kw, "kv": kv}) == (status, before)


def test_commit_refuses_positions_out_of_range():
    f = B.dc_feat(FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 0, 2**31 - 5)
    assert commit(feat=f) == (SHAPE, 40) and f.next_pos == 2**31 - 5


def test_commit_of_plain_rows_on_the_host():
    # no features, no ragged lengths, no path: nothing but bookkeeping
    kv = _kv()
    assert commit(kv=kv, width=7) == (0, 47)
