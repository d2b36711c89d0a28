"""Outputs that share memory with what a call reads are refused (no GPU)."""
import os

import pytest

from paper_2608_08878_amd import binding as B

from .test_abi_prompt import FAKE, UNSUPPORTED, _tok, attend, rope

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

Q, K, V, OUT, KOUT = (x << 24 for x in range(1, 6))        # far apart
ROW = 8 * 128 * 2                                          # a token's query heads; 20 tokens


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("off", [-20 * ROW + 16, -ROW, 16, ROW, 20 * ROW - 16])
def test_attention_refuses_an_output_across_its_queries(tree, off):
    assert attend(tree, q=Q, out=Q + off) == UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(q_out=Q + 16), dict(q_out=Q - 20 * ROW + 16), dict(q_out=Q + 19 * 1536 * 2 + ROW - 16),
    dict(q_out=K), dict(q_out=K + 16), dict(q_out=V - 16),
    dict(k_out=Q), dict(k_out=K + 16), dict(k_out=OUT + 20 * ROW - 16), dict(k_out=OUT)])
def test_rotation_refuses_outputs_across_its_inputs(kw):
    assert rope(**{**dict(q=Q, k=K, v=V, q_out=OUT), **kw}) == UNSUPPORTED


def test_rotation_in_place_refuses_keys_across_queries():
    # in place for both, the keys inside the queries' memory
    assert rope(q=Q, ld_q=1024, k=Q + ROW, ld_k=256, q_out=Q, k_out=Q + ROW) == UNSUPPORTED
    assert rope(tok=_tok(2, 1), q=FAKE, ld_q=1024, k=FAKE, ld_k=256, q_out=FAKE, k_out=FAKE) == UNSUPPORTED
