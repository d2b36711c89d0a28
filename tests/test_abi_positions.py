"""Host side of the positions of sequences that see different numbers of tokens (no GPU)."""
import ctypes
import os

import pytest

from paper_2608_08878_amd import binding as B

from .test_abi_prompt import FAKE, NULL, SHAPE, _dims, _kv, _tok, commit

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")


def _feat(behind=FAKE, **kw):
    f = B.dc_feat(FAKE, FAKE, FAKE, FAKE, FAKE)
    f.behind = behind
    for name, x in kw.items():
        setattr(f, name, x)
    return f


@pytest.mark.parametrize("kw", [dict(tok=_tok(15, 10, FAKE)), dict(keep=FAKE), dict(path=FAKE, keep=FAKE)])
def test_counts_that_differ_need_a_place_for_the_positions(kw):
    f = _feat(None, next_pos=40)
    assert commit(kv=_kv(unit_len=FAKE), feat=f, **kw) == (NULL, 40) and f.next_pos == 40


def test_it_takes_a_ragged_cache():
    assert commit(kv=_kv(), feat=_feat()) == (NULL, 40)


@pytest.mark.parametrize("name,slot,value", [("behind_row", None, -1), ("behind_row", None, B.BEHIND_ROWS + 1),
                                             ("ring_row", 0, -1), ("ring_row", 63, B.BEHIND_ROWS + 1)])
def test_rows_out_of_range_are_refused(name, slot, value):
    f = _feat(qring=FAKE, qstat=FAKE)
    if slot is None:
        setattr(f, name, value)
    else:
        getattr(f, name)[slot] = value
    kv = _kv(unit_len=FAKE)
    assert commit(kv=kv, feat=f, keep=FAKE)[0] == SHAPE
    d, L = _dims(), B.lib()
    pol = B.dc_policy(4, 1, (ctypes.c_int32 * 2)(8, 0), FAKE, 0)
    f.next_pos = 40
    assert L.dc_decode_step(ctypes.byref(d), ctypes.byref(kv), ctypes.byref(f), FAKE, FAKE, FAKE, FAKE, FAKE,
                            1 << 40, None) == SHAPE
    assert L.dc_score_evict(ctypes.byref(d), ctypes.byref(kv), ctypes.byref(f), ctypes.byref(pol), 8, None, None,
                            FAKE, 1 << 40, None) == SHAPE


def test_init_puts_all_sequences_at_one_position():
    f = _feat(behind_row=7, behind_at=3, next_pos=3, step=9)
    f.ring_row[5] = 7
    kv = _kv(0, unit_len=FAKE)                    # no rows: host fields only
    B.dc_feat_init(_dims(), kv, f, 11)
    assert (f.behind_row, f.behind_at, f.next_pos, f.step) == (0, 11, 11, 0) and not any(f.ring_row)
