// Attention of sequences that have rows in common: how a call is cut, and its launches (the kernels
// are in dc_attend.hpp).
//
// Eight rollouts of 8192 rows (32/8 heads of 128, 40 MB) 12.8 us and 5.6 for the join: a workgroup's start, the
// chain of lengths and first loads, is most of it (the walk is two tiles of keys).  50 sequences over four
// prefixes of up to 16384 rows, 370 MB, 67 us = 5.5 TB/s, bound by HBM.  Eight prompts of 512 tokens behind
// 16384 shared rows 1076 us = 1.04 PFLOP/s, bound as the prompts are.
#include "dc_attend.hpp"

namespace dc {

namespace {

template <int DT, int D>
int launch_type(const SharedArgs& a, hipStream_t s) {
  const int64_t wgs = a.shared_wgs + (int64_t)a.batch * a.hk * a.ntiles * (a.splits - a.psplits);
  const int rc = a.parent ? launch_tiles<DT, D, SHARED_TREE>(a, wgs, s) : launch_tiles<DT, D, SHARED>(a, wgs, s);
  return rc == 0 && a.splits > 1 ? launch_join<DT, D, SHARED>(a, s) : rc;
}

}  // namespace

bool shared_plan(SharedArgs& a, int dtype, int D, int L, int Lp) {
  const int64_t prows = (int64_t)a.group_tokens << a.gshift, rows = (int64_t)a.tok.max_tokens << a.gshift;
  const int64_t ppairs = (int64_t)a.prefixes * a.hk, pairs = (int64_t)a.batch * a.hk;
  const int64_t all = ((int64_t)a.tok.tokens << a.gshift) * a.hk;
  // workgroups of bm rows: the packed tokens' and a part of one for every prefix (sequence)
  auto tiles = [&](int bm, int64_t np, int64_t longest) {
    const int64_t packed = all / bm + np, nt = (longest + bm - 1) / bm * np;
    return packed < nt ? packed : nt;
  };
  const int64_t bytes = (ppairs * Lp + pairs * L) * 2 * D * (dtype == 1 ? 2 : 4);
  // Parts of a row at most: what fills the card by the shared rows' tiles of 128, whatever the lengths.  One, and so
  // no workspace, where the sequences' own tiles of 128 fill the card twice over and are all full, or eight times over and
  // are full to 98 %: there are as many tiles over the shared rows by themselves, and parts are worth nothing.
  // Where sequences without a prefix must be among them, they leave the tiles too uneven for that.  (8 prompts of 2048
  // tokens behind 16384 rows, 32/8 heads of 128, 4295 us, would have to bring 545 MB for parts that nobody writes.
  // Of uneven prompts whose tiles are full to 95 %, some are up to 16 % faster in two parts.)
  const int64_t own128 = tiles(128, pairs, rows);
  const bool whole = (all == own128 * 128 ? own128 >= 4 * CUS : own128 >= 16 * CUS && all * 50 >= own128 * 128 * 49) &&
                     (int64_t)a.prefixes * a.max_members >= a.batch;
  int64_t most = whole ? 1 : 2 + 4 * CUS / tiles(128, ppairs, prows);
  most = most > MAX_PARTS ? MAX_PARTS : most;
  // Tiles and parts by their time.  Either parts of equal length of the shared rows, for tiles of all their
  // sequences' tokens, and of the own rows; or tiles of one sequence through both, which read the shared
  // rows once per sequence and leave nothing to join where they take no parts (eight prompts of 512
  // tokens behind 16384 rows 1155 -> 1066 us; the step of eight rollouts 19 us, through both 42).
  const int64_t longest = L > Lp ? L : Lp;
  double least = -1.0;
  for (int bm = 32; bm <= 128; bm *= 2) {
    if (bm == 64 && dtype != 1) continue;
    const int64_t ptiles = tiles(bm, ppairs, prows), otiles = tiles(bm, pairs, rows);
    for (int through = 0; through < 2; ++through) {
      const Cut cut = cut_of(dtype, D, bm, through || rows > prows ? rows : prows);
      // (32 bits: this is host time of every call)
      const uint32_t padded = (Lp + cut.bn - 1u) / cut.bn * cut.bn, own = through ? padded + L : L;
      const uint32_t walk = through ? own : longest;
      const double keys = ((double)otiles * own + (through ? 0.0 : (double)ptiles * Lp)) / cut.bn;
      uint32_t last = 0;
      for (const uint32_t n : PARTS) {
        if (n > most) break;
        const uint32_t c = ((walk + n - 1) / n + MIN_CHUNK - 1) / MIN_CHUNK * MIN_CHUNK;
        const uint32_t ps = through ? 0 : (Lp + c - 1) / c, os = (own + c - 1) / c;
        if (ps + os > most || c == last) continue;
        last = c;
        const double wgs = (double)ptiles * ps + (double)otiles * os;
        const double us = cut_us(cut, wgs / (cut.per_cu * CUS), ((c < walk ? c : walk) + cut.bn - 1) / cut.bn, keys / wgs,
                                 ps + os, (double)a.tok.tokens * a.hq, D);
        if (least >= 0.0 && us >= least) continue;
        least = us;
        a.bm = bm;
        a.bn = cut.bn;
        a.through = through;
        a.psplits = (int)ps;
        a.splits = (int)(ps + os);
        a.chunk = a.pchunk = (int)c;
      }
    }
  }
  const int64_t nt = (rows + a.bm - 1) / a.bm, pt = (prows + a.bm - 1) / a.bm;
  a.most_splits = (int)most;
  a.once = nt == 1 && pt == 1 && bytes > BIG_CACHE && !a.through;
  a.ntiles = (int)nt;
  a.shared_wgs = (int)(ppairs * pt * a.psplits);
  // a launch counts its threads in 32 bits: 2^24 workgroups of 256
  return (ppairs * ((prows + 31) / 32) + pairs * ((rows + 31) / 32)) * most < (1 << 24) &&
         (most == 1 || pairs * ((rows + 3) / 4) < (1 << 24));
}

int launch_shared(const SharedArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? launch_type<1, 128>(a, s) : launch_type<1, 64>(a, s);
  return D == 128 ? launch_type<0, 128>(a, s) : launch_type<0, 64>(a, s);
}

}  // namespace dc
