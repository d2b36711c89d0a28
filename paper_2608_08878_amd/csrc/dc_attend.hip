// Attention of several new tokens per sequence over cache rows: how a call is cut, and its launches
// (the kernels are in dc_attend.hpp).
#include "dc_attend.hpp"

namespace dc {

namespace {

template <int DT, int D>
int launch_type(const AttendArgs& a, hipStream_t s) {
  const int64_t wgs = (int64_t)a.batch * a.hk * a.ntiles * a.splits;
  int rc = a.parent ? launch_tiles<DT, D, TREE>(a, wgs, s) : launch_tiles<DT, D, PROMPT>(a, wgs, s);
  if (rc == 0 && a.splits > 1) rc = launch_join<DT, D, PROMPT>(a, s);
  return rc;
}

}  // namespace

bool attend_plan(AttendArgs& a, int dtype, int D, int L) {
  const int64_t rows = (int64_t)a.tok.max_tokens << a.gshift;
  const int64_t pairs = (int64_t)a.batch * a.hk;
  // workgroups of bm rows: the packed tokens' and a part of one for every sequence
  auto tiles = [&](int bm) {
    const int64_t all = ((int64_t)a.tok.tokens << a.gshift) * a.hk / bm + pairs, nt = (rows + bm - 1) / bm;
    return all < nt * pairs ? all : nt * pairs;
  };
  const int64_t parts = (L + MIN_CHUNK - 1) / MIN_CHUNK;
  const int64_t bytes = pairs * L * 2 * D * (dtype == 1 ? 2 : 4);      // of K and V
  // Rows of a tile.  32, the keys cut among the waves, for up to 32 rows and where tiles of 128 would
  // leave CUs idle (measured against 128: 512 float32 tokens of 4/2 heads of 64 11.7 and 17.7 us, 256
  // tokens of 32/8 heads 9.3 and 10.5, one token of 8 sequences in float32 109 and 190; past that point
  // 128 rows are faster, 512 tokens 16.2 and with 32 18.4).  64 and two groups of keys for up to 64 bf16
  // rows (13 tokens behind 4096 13.5 us, with 128 rows 14.8).  Both hold a CU's LDS alone with heads of
  // 128 elements, and caches that only HBM holds stream faster by two workgroups: there 128 rows (one
  // token of 16 sequences of 4096 rows 49 us, with 32 rows 56; 16 tokens, 16384 rows, 188, with 64 206).
  const bool stream = dtype == 1 && D == 128 && bytes > BIG_CACHE / 4 * 3;
  int bm = 128;
  if (!stream && (rows <= 32 || tiles(128) * parts < CUS)) bm = 32;
  else if (!stream && rows <= 64 && dtype == 1) bm = 64;
  // Parts of the key range, at most as many as the CUs hold workgroups at a time.  More parts shorten
  // a workgroup's walk over the keys and lengthen the join, whose outputs in float32 are written and
  // read: the number with the least of both, from what was measured (us): a walk's step of `bn` keys
  // 1.3 alone on a CU and 2 beside another (bf16, 128 elements), joined outputs at 3.5 TB/s.  One prompt
  // of 512 tokens 21 -> 16 us against as many parts as fit, of 1024 37 -> 27; 256 behind 16384 rows
  // 94, with half as many parts 102, in one 330.
  // Workgroups that a CU holds (Cfg::WAVES): two, but one of the small tiles whose buffers are a CU's LDS
  // (float32, and bf16 with 128 elements) and of the 128-row float32 tiles with 128 elements, whose
  // registers are a CU's.  For those one against two: 1000 tokens of 32/8 heads 151 and 169 us, 64 tokens
  // of 8 sequences behind 4096 rows 326 and 353; where two parts are a few workgroups more than one
  // round it is the slower (3 x 700 tokens behind 900 rows of 8/4 heads 234 and 203).
  const int per_cu = dtype == 1 ? (bm == 128 || D == 64 ? 2 : 1) : bm == 128 && D == 64 ? 2 : 1;
  int64_t most = per_cu * CUS / tiles(bm);
  most = most > parts ? parts : most;
  most = most > MAX_PARTS ? MAX_PARTS : most < 1 ? 1 : most;
  const int bn = bm == 128 ? (dtype == 1 ? 64 : 32) : dtype == 1 || D == 64 ? 128 : 64;
  const double step = dtype == 1 ? 0.5 + 0.8 * D / 128 : 3.6 * D / 128;
  const double seen = 1.0 - 0.5 * a.tok.max_tokens / L;       // of the parts, by the average row
  int64_t splits = 1, chunk = (L + MIN_CHUNK - 1) / MIN_CHUNK * MIN_CHUNK;
  double least = 0.0;
  for (int64_t n = 1; n <= most; ++n) {
    const int64_t c = ((L + n - 1) / n + MIN_CHUNK - 1) / MIN_CHUNK * MIN_CHUNK, real = (L + c - 1) / c;
    const double walk = (double)((c + bn - 1) / bn) * step * (per_cu == 2 && tiles(bm) * real > CUS ? 1.55 : 1.0);
    const double join = n > 1 ? 3.0 + (double)a.tok.tokens * a.hq * real * seen * D * 8 / 3.5e6 : 0.0;
    if (n == 1 || walk + join < least) {
      least = walk + join;
      splits = real;
      chunk = c;
    }
  }
  a.most_splits = (int)most;
  const int64_t nt = (rows + bm - 1) / bm;
  a.bm = bm;
  // Rows that one row tile reads, once, and that no cache holds anyway: non-temporal (320 drafted
  // tokens of 16 sequences over up to 16k rows, 834 MB, 191 -> 180 us; 13 over 4k rows, 17 MB, 15.6 -> 16.8)
  a.once = nt == 1 && bytes > BIG_CACHE;
  a.splits = (int)splits;
  a.chunk = (int)chunk;
  a.ntiles = (int)nt;
  // a launch counts its threads in 32 bits: 2^24 workgroups of 256
  return pairs * nt * most < (1 << 24) && (most == 1 || pairs * ((rows + 3) / 4) < (1 << 24));
}

int launch_attend(const AttendArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? launch_type<1, 128>(a, s) : launch_type<1, 64>(a, s);
  return D == 128 ? launch_type<0, 128>(a, s) : launch_type<0, 64>(a, s);
}

}  // namespace dc
