"""The cuts that the GPU tests of shared rows and chosen blocks rely on: each of their sizes reaches the tiles that it is
there for (host code, no GPU)."""
import pytest

from . import plan_cases as C
from . import plans as P

pytestmark = pytest.mark.skipif(not P.can_ask(), reason="library not built or no C++ compiler")


def _check(cases, line):
    got = P.ask([line(*args) for args, _ in cases.values()])
    for (name, (_, (bm, through, parts, once))), (ok, *g) in zip(cases.items(), got):
        assert ok and (g[0], g[1], g[3] > 1, g[4]) == (bm, through, parts, once), (name, g)


def test_shared_cases_reach_their_tiles():
    _check({**C.SHARED, **{"once " + k: v for k, v in C.SHARED_ONCE.items()}}, P.shared_line)


def test_block_cases_reach_their_tiles():
    _check({**C.BLOCKS, **{"once " + k: v for k, v in C.BLOCKS_ONCE.items()}}, P.blocks_line)


def test_every_shape_of_a_tile_is_there():
    """(32 rows: the small cases of the GPU tests.)  In float32 there are no tiles of 64 rows, and in bf16 none for heads of
    128 that these plans choose."""
    shared = {(a[0], a[1], e[0], e[1], e[2]) for a, e in C.SHARED.values()}
    for through, parts in ((0, True), (1, False), (1, True)):
        want = {("bf16", 64, 64), ("bf16", 64, 128), ("bf16", 128, 128), ("f32", 64, 128), ("f32", 128, 128)}
        assert {s[:3] for s in shared if s[3:] == (through, parts)} == want
    blocks = {(a[0], a[1], e[0], e[2]) for a, e in C.BLOCKS.values()}
    for parts in (False, True):
        assert {s[:3] for s in blocks if s[3] == parts} == want
    # several waves of rows in a tile
    for a, e in [*C.SHARED.values()]:
        assert max(a[4]) * a[3] > 32 or sum(a[4]) * a[3] > 32
    for a, e in [*C.BLOCKS.values()]:
        assert min(max(a[4]), a[8]) * a[3] > 32


def test_prompts_that_fill_the_card_take_one_part_whatever_the_lengths():
    lines = [P.shared_line("bf16", 128, 8, 4, [2048] * 8, [8], plen, rows) for plen in (1, 100, 16384, 1 << 20)
             for rows in (0, 700, 20000)]
    for ok, bm, through, psplits, splits, _ in P.ask(lines):
        assert ok and through == 1 and psplits == 0 and splits == 1


def test_grids_of_joins_that_are_not_launched_refuse_nothing():
    # 4 million tokens are 2^23 tiles of 32 rows and 2^26 workgroups of a join: taken, in one part
    (ok, _, _, _, splits, _), (past, *_) = P.ask([P.blocks_line("bf16", 128, 8, 8, [n] * 4096, 3000, 16, 48, 16)
                                                 for n in (1024, 2048)])
    assert ok and splits == 1 and not past
    (ok, _, _, _, splits, _), = P.ask([P.shared_line("bf16", 128, 8, 8, [32768] * 64, [64], 1000, 0)])
    assert ok and splits == 1


def test_large_calls_of_single_tokens_take_tiles_of_32_rows():
    """Two calls of test_gpu_shared_blocks by many workgroups: 197 and 147 MB of rows, under the 256 MiB from which rows are
    read past the caches, so they run the tiles of 32 rows that smaller ones do (C.SHARED_ONCE, C.BLOCKS_ONCE are larger)."""
    got = P.ask([P.shared_line("bf16", 128, 8, 4, [1] * 12, [6, 6], 15000, 1500),
                 P.blocks_line("bf16", 128, 4, 4, [1] * 32, 2600, 64, 34, 1)])
    assert [(g[1], g[5]) for g in got] == [(32, 0), (32, 0)]
