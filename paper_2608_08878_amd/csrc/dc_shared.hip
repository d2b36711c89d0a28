// Attention of sequences that have rows in common: how a call is cut, and its launches (the kernels
// are in dc_attend.hpp).
#include "dc_attend.hpp"

namespace dc {

namespace {

template <int DT, int D>
int launch_type(const SharedArgs& a, hipStream_t s) {
  const int64_t wgs = a.shared_wgs + (int64_t)a.batch * a.hk * a.ntiles * (a.splits - a.psplits);
  const int rc = a.parent ? launch_tiles<DT, D, SHARED_TREE>(a, wgs, s) : launch_tiles<DT, D, SHARED>(a, wgs, s);
  return rc == 0 ? launch_join<DT, D, SHARED>(a, s) : rc;
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
  // as in attend_plan
  const bool stream = dtype == 1 && D == 128 && bytes > BIG_CACHE / 4 * 3;
  const int64_t parts = tiles(128, ppairs, prows) * ((Lp + MIN_CHUNK - 1) / MIN_CHUNK) +
                        tiles(128, pairs, rows) * ((L + MIN_CHUNK - 1) / MIN_CHUNK);
  int bm = 128;
  if (!stream && (prows <= 32 || parts < CUS)) bm = 32;
  else if (!stream && prows <= 64 && dtype == 1) bm = 64;
  const int per_cu = dtype == 1 ? (bm == 128 || D == 64 ? 2 : 1) : bm == 128 && D == 64 ? 2 : 1;
  const int64_t ptiles = tiles(bm, ppairs, prows), otiles = tiles(bm, pairs, rows);
  // Parts of a row at most: what fills the card by the shared rows' tiles of 128, whatever the lengths
  int64_t most = 2 + 4 * CUS / tiles(128, ppairs, prows);
  most = most > MAX_PARTS ? MAX_PARTS : most;
  // Parts of equal length on both sides, by the time of their walk and of the join (as in attend_plan)
  const int bn = bm == 128 ? (dtype == 1 ? 64 : 32) : dtype == 1 || D == 64 ? 128 : 64;
  const double step = dtype == 1 ? 0.5 + 0.8 * D / 128 : 3.6 * D / 128;
  const int64_t longest = L > Lp ? L : Lp;
  double least = -1.0;
  for (int64_t c = MIN_CHUNK;; c += (c / 10 + MIN_CHUNK - 1) / MIN_CHUNK * MIN_CHUNK) {
    const int64_t ps = (Lp + c - 1) / c, os = (L + c - 1) / c;
    if (ps + os <= most || c >= longest) {
      const int64_t wgs = ptiles * ps + otiles * os, rounds = (wgs + per_cu * CUS - 1) / (per_cu * CUS);
      const double walk = (double)rounds * (c / bn) * step * (per_cu == 2 && wgs > CUS ? 1.55 : 1.0);
      const double join = (double)a.tok.tokens * a.hq * (ps + os) * D * 8 / 3.5e6;
      if (least < 0.0 || walk + join < least) {
        least = walk + join;
        a.psplits = (int)ps;
        a.splits = (int)(ps + os);
        a.chunk = a.pchunk = (int)c;
      }
    }
    if (c >= longest) break;
  }
  const int64_t nt = (rows + bm - 1) / bm, pt = (prows + bm - 1) / bm;
  a.most_splits = (int)most;
  a.bm = bm;
  a.once = nt == 1 && pt == 1 && bytes > BIG_CACHE;
  a.ntiles = (int)nt;
  const int64_t wgs = ppairs * pt * a.psplits + pairs * nt * (a.splits - a.psplits);
  a.shared_wgs = (int)(ppairs * pt * a.psplits);
  // a launch counts its threads in 32 bits: 2^24 workgroups of 256
  return (ppairs * pt + pairs * nt) * most < (1 << 24) && wgs < (1 << 24) && pairs * ((rows + 3) / 4) < (1 << 24);
}

int launch_shared(const SharedArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? launch_type<1, 128>(a, s) : launch_type<1, 64>(a, s);
  return D == 128 ? launch_type<0, 128>(a, s) : launch_type<0, 64>(a, s);
}

}  // namespace dc
