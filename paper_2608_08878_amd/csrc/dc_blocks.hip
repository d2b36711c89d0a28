// Blocks of a cache's rows on gfx950: the bounds of their keys, the choice of blocks by a bound of
// the logits, and the launches of the attention over chosen ones (its kernels are in dc_attend.hpp).
//
// A query's logit with any key of a block is at most scale * sum_e max(q_e hi_e, q_e lo_e), hi and lo
// being the largest and smallest elements of the block's keys.  Summed over the queries that choose
// together that is one product of length 2 D per block,
//   score = Q+ . hi + Q- . lo,   Q+ = sum max(q, 0), Q- = sum min(q, 0),
// whatever the number of queries.
#include "dc_attend.hpp"

#pragma clang fp contract(off)

namespace dc {

namespace {

// ------------------------------------------------------------------------ bounds

typedef short i16x2_t __attribute__((ext_vector_type(2)));

// Numbers as integers of the same order and back (their own inverse), two bf16 or one float32 a word.
template <int DT>
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  if constexpr (DT == 1) {
    const i16x2_t x = __builtin_bit_cast(i16x2_t, w);
    return w ^ (__builtin_bit_cast(uint32_t, x >> 15) & 0x7FFF7FFFu);
  } else {
    return w ^ ((uint32_t)((int32_t)w >> 31) & 0x7FFFFFFFu);
  }
}
template <int DT>
__device__ __forceinline__ uint32_t more(uint32_t a, uint32_t b) {
  if constexpr (DT == 1)
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2_t, a),
                                                                  __builtin_bit_cast(i16x2_t, b)));
  else
    return (int32_t)a > (int32_t)b ? a : b;
}
template <int DT>
__device__ __forceinline__ uint32_t less(uint32_t a, uint32_t b) {
  if constexpr (DT == 1)
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2_t, a),
                                                                  __builtin_bit_cast(i16x2_t, b)));
  else
    return (int32_t)a < (int32_t)b ? a : b;
}
// The largest and smallest finite numbers in that order.
template <int DT>
constexpr uint32_t TOP = DT == 1 ? 0x7F7F7F7Fu : 0x7F7FFFFFu;
template <int DT>
constexpr uint32_t BOTTOM = DT == 1 ? 0x80808080u : 0x80800000u;

constexpr int BT = 256;

// A wave takes NB blocks at a time, 16 bytes a lane, LPR lanes a row.  Infinite elements and NaN count as the
// largest numbers of their sign: scores of finite queries stay finite, and a block that holds
// one ranks high rather than out of sight.
template <int DT, int D, int SHIFT>
__global__ void __launch_bounds__(BT) bounds_kernel(BoundsArgs a, int per_block) {
  using R = RowT<DT, D>;
  constexpr int S = 1 << SHIFT, LPR = R::LPR, RPI = 64 / LPR, NL = S / RPI;   // rows and number of a block's loads
  constexpr int NB = NL < 8 ? 8 / NL : 1, UN = NL < 16 ? NL : 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int u = a.y0 + blockIdx.y;
  const int end = rows_before(a.unit_len, a.len, u) >> SHIFT;
  const int j0 = (a.from >> SHIFT) + blockIdx.x * per_block;
  const int j1 = j0 + per_block < end ? j0 + per_block : end;
  const char* k = (const char*)a.k + (size_t)u * a.cap * (D * R::ELT) + lane * 16;
  char* out = (char*)a.bounds + (size_t)u * (a.cap >> SHIFT) * (2 * D * R::ELT);
  for (int j = j0 + wave * NB; j < j1; j += BT / 64 * NB) {
    uint4 hi[NB], lo[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      hi[b] = make_uint4(BOTTOM<DT>, BOTTOM<DT>, BOTTOM<DT>, BOTTOM<DT>);
      lo[b] = make_uint4(TOP<DT>, TOP<DT>, TOP<DT>, TOP<DT>);
    }
#pragma unroll
    for (int i0 = 0; i0 < NL; i0 += UN) {
      uint4 w[NB][UN];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int jb = j + b < j1 ? j + b : j1 - 1;
#pragma unroll
        for (int i = 0; i < UN; ++i)
          w[b][i] = ldg16_nt(k + ((size_t)jb * NL + i0 + i) * 1024);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          const uint4 x = make_uint4(ordered<DT>(w[b][i].x), ordered<DT>(w[b][i].y), ordered<DT>(w[b][i].z),
                                     ordered<DT>(w[b][i].w));
          hi[b] = make_uint4(more<DT>(hi[b].x, x.x), more<DT>(hi[b].y, x.y), more<DT>(hi[b].z, x.z),
                             more<DT>(hi[b].w, x.w));
          lo[b] = make_uint4(less<DT>(lo[b].x, x.x), less<DT>(lo[b].y, x.y), less<DT>(lo[b].z, x.z),
                             less<DT>(lo[b].w, x.w));
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      uint32_t h[4] = {hi[b].x, hi[b].y, hi[b].z, hi[b].w}, l[4] = {lo[b].x, lo[b].y, lo[b].z, lo[b].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int off = LPR; off < 64; off *= 2) {
          h[e] = more<DT>(h[e], __shfl_xor(h[e], off));
          l[e] = less<DT>(l[e], __shfl_xor(l[e], off));
        }
        h[e] = ordered<DT>(less<DT>(h[e], TOP<DT>));
        l[e] = ordered<DT>(more<DT>(l[e], BOTTOM<DT>));
      }
      if (j + b < j1 && lane < 2 * LPR) {
        const bool low = lane >= LPR;
        *reinterpret_cast<uint4*>(out + (size_t)(j + b) * (2 * D * R::ELT) + lane * 16) =
            make_uint4(low ? l[0] : h[0], low ? l[1] : h[1], low ? l[2] : h[2], low ? l[3] : h[3]);
      }
    }
  }
}

template <int DT, int D>
int bounds_type(const BoundsArgs& a, hipStream_t s) {
  const int n = (a.len >> a.bshift) - (a.from >> a.bshift);        // blocks of the longest unit
  if (n <= 0) return 0;
  // a workgroup's waves take a few blocks each
  int per = 4096 >> a.bshift;
  per = per < 32 ? 32 : per;
  const int gx = (n + per - 1) / per;
  for_grid_y(a.units, [&](int y0, int ny) {
    BoundsArgs b = a;
    b.y0 = y0;
    const dim3 grid(gx, ny);
    switch (a.bshift) {
      case 4: hipLaunchKernelGGL((bounds_kernel<DT, D, 4>), grid, dim3(BT), 0, s, b, per); break;
      case 5: hipLaunchKernelGGL((bounds_kernel<DT, D, 5>), grid, dim3(BT), 0, s, b, per); break;
      case 6: hipLaunchKernelGGL((bounds_kernel<DT, D, 6>), grid, dim3(BT), 0, s, b, per); break;
      default: hipLaunchKernelGGL((bounds_kernel<DT, D, 7>), grid, dim3(BT), 0, s, b, per);
    }
  });
  return (int)hipGetLastError();
}

// ------------------------------------------------------------------------ choice

constexpr int ST = 512;                  // threads of a workgroup
constexpr int SW = ST / 64;
constexpr int MAX_BLOCKS = 16384;        // of a unit: their ranks fill the LDS

// Scores as integers of the same order: NaN below every number, -0 equal to +0.
__device__ __forceinline__ uint64_t rank_of(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  if (x != x) return 0;
  return b >> 63 ? ~b : b | (1ull << 63);
}

__device__ __forceinline__ double shfl_xor_f64(double x, int mask) {
  const int lo = __shfl_xor(__double2loint(x), mask), hi = __shfl_xor(__double2hiint(x), mask);
  return __hiloint2double(hi, lo);
}

// A sum over the workgroup, for all (two cells of LDS in turn).
__device__ __forceinline__ int count_all(int x, int* cell) {      // x uniform over a wave
  if ((threadIdx.x & 63) == 0) cell[threadIdx.x >> 6] = x;
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int w = 0; w < SW; ++w) n += cell[w];
  return n;
}

// One workgroup per list.  The scores are binary64: products of bf16 elements are exact there and sums all
// but exact, so that a choice next to its limit does not hang on the order of a sum.
template <int DT, int D>
__global__ void __launch_bounds__(ST) select_kernel(SelectArgs a) {
  using R = RowT<DT, D>;
  constexpr int LPR = R::LPR, EPL = R::EPL, LPB = 2 * LPR, GROUPS = ST / LPR, BPL = 64 / LPB;
  constexpr int UN = 8;                       // loads of a lane under way
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ double qs[2 * D];
  __shared__ int cells[2][SW];
  __shared__ uint64_t ends[2][SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int pairs = a.batch * a.hk, pair = blockIdx.x % pairs, group = blockIdx.x / pairs;
  const int b = pair / a.hk, g = pair % a.hk, u = (b * a.n_layers + a.layer) * a.hk + g;
  int t0, n;
  token_range(a.tok, b, t0, n);
  int32_t* list = a.list + ((size_t)(b * a.groups + group) * a.hk + g) * a.count;
  const int r0 = group * a.share, r1 = r0 + a.share < n ? r0 + a.share : n;
  const int cand = r0 < n ? rows_before(a.unit_len, a.len, u) >> a.bshift : 0;
  if (cand <= a.count) {                      // all of them, or a group without tokens
    for (int i = tid; i < a.count; i += ST) list[i] = i < cand ? i : -1;
    return;
  }
  // sums of the queries' positive and negative elements: a lane group a row, the groups in turn
  const int rows = (r1 - r0) << a.gshift, used = rows < GROUPS ? rows : GROUPS;
  double* part = reinterpret_cast<double*>(lds);            // [used][2][D]
  {
    const int c = tid % LPR, at = tid / LPR;
    double up[EPL] = {}, down[EPL] = {};
    for (int i = at; i < rows; i += GROUPS) {
      const size_t row = (size_t)(t0 + r0 + (i >> a.gshift)) * a.hq + (g << a.gshift) + (i & ((1 << a.gshift) - 1));
      float f[EPL];
      unpack_slice<DT>(ldg16((const char*)a.q + row * (D * R::ELT) + c * 16), f);
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        // (NaN stays one in both)
        up[e] += f[e] < 0.0f ? 0.0 : (double)f[e];
        down[e] += f[e] > 0.0f ? 0.0 : (double)f[e];
      }
    }
    if (at < used)
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        part[(at * 2) * D + c * EPL + e] = up[e];
        part[(at * 2 + 1) * D + c * EPL + e] = down[e];
      }
  }
  __syncthreads();
  for (int e = tid; e < 2 * D; e += ST) {
    double s = part[e];
    for (int i = 1; i < used; ++i) s += part[i * 2 * D + e];
    qs[e] = s;
  }
  __syncthreads();
  // scores: LPB lanes a block, 16 bytes each
  uint64_t* keys = reinterpret_cast<uint64_t*>(lds);
  const int c = lane % LPB;
  double q[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) q[e] = qs[c * EPL + e];
  const char* bounds = (const char*)a.bounds + (size_t)u * (a.cap >> a.bshift) * (2 * D * R::ELT) + c * 16;
  for (int j0 = wave * UN * BPL; j0 < cand; j0 += SW * UN * BPL) {
    uint4 w[UN];
    double s[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int j = j0 + i * BPL + lane / LPB;
      w[i] = ldg16(bounds + (size_t)(j < cand ? j : cand - 1) * (2 * D * R::ELT));
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      float f[EPL];
      unpack_slice<DT>(w[i], f);
      s[i] = 0.0;
#pragma unroll
      for (int e = 0; e < EPL; ++e) s[i] = __builtin_fma((double)f[e], q[e], s[i]);
    }
    // sums over the block's lanes: three steps that also hand each lane one of the eight
#pragma unroll
    for (int half = UN / 2, bit = 1; half >= 1; half /= 2, bit *= 2) {
      const bool odd = lane & bit;
#pragma unroll
      for (int i = 0; i < half; ++i) {
        const double give = odd ? s[i] : s[i + half], keep = odd ? s[i + half] : s[i];
        s[i] = keep + shfl_xor_f64(give, bit);
      }
    }
#pragma unroll
    for (int bit = UN; bit < LPB; bit *= 2) s[0] += shfl_xor_f64(s[0], bit);
    // lane c < 8 of a block's has the sum of load: bits of c from the highest half down
    const int i = (lane & 1) * 4 + (lane & 2) + ((lane >> 2) & 1), j = j0 + i * BPL + lane / LPB;
    if (c < UN && j < cand) keys[j] = rank_of(s[0]);
  }
  __syncthreads();
  // The first and last blocks are in; of the others the `need` highest, by halving an interval of ranks:
  // at least `need` are at or above lo, fewer at or above hi.
  const int head = a.first < cand ? a.first : cand, tail = cand - a.last > head ? cand - a.last : head;
  const int need = a.count - head - (cand - tail);
  uint64_t lo = ~0ull, hi = 0;
  for (int j = head + tid; j < tail; j += ST) {
    const uint64_t x = keys[j];
    lo = x < lo ? x : lo;
    hi = x > hi ? x : hi;
  }
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const uint64_t x = __shfl_xor(lo, off), y = __shfl_xor(hi, off);
    lo = x < lo ? x : lo;
    hi = y > hi ? y : hi;
  }
  if (lane == 0) {
    ends[0][wave] = lo;
    ends[1][wave] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SW; ++w) {
    lo = ends[0][w] < lo ? ends[0][w] : lo;
    hi = ends[1][w] > hi ? ends[1][w] : hi;
  }
  ++hi;
  int ties = need, turn = 0;                    // of those equal to lo, the lowest numbers
  if (need <= 0) {
    lo = hi;
    ties = 0;
  }
  while (hi - lo > 1) {
    const uint64_t mid = lo + (hi - lo) / 2;
    int x = 0;
    for (int j0 = head; j0 < tail; j0 += ST) x += __popcll(__ballot(j0 + tid < tail && keys[j0 + tid] >= mid));
    x = count_all(x, cells[turn]);
    turn ^= 1;
    if (x >= need) lo = mid;
    else {
      hi = mid;
      ties = need - x;
    }
    if (x == need) {                            // exactly these
      --lo;
      ties = 0;
      break;
    }
  }
  // in ascending order: above lo, and of those at lo the first `ties`
  int at = 0, tied = 0;
  for (int j0 = 0; j0 < cand; j0 += ST) {
    const int j = j0 + tid;
    const bool in = j < cand, forced = in && (j < head || j >= tail);
    const uint64_t x = in ? keys[j] : 0;
    const bool above = in && !forced && x > lo, equal = in && !forced && x == lo;
    const uint64_t eq = __ballot(equal), below = (1ull << lane) - 1;
    __syncthreads();
    if (lane == 0) cells[0][wave] = __popcll(eq);
    __syncthreads();
    int before = tied;
#pragma unroll
    for (int w = 0; w < SW; ++w) {
      if (w < wave) before += cells[0][w];
      tied += cells[0][w];
    }
    const bool take = forced || above || (equal && before + __popcll(eq & below) < ties);
    const uint64_t m = __ballot(take);
    if (lane == 0) cells[1][wave] = __popcll(m);
    __syncthreads();
    int to = at;
#pragma unroll
    for (int w = 0; w < SW; ++w) {
      if (w < wave) to += cells[1][w];
      at += cells[1][w];
    }
    if (take) list[to + __popcll(m & below)] = j;
  }
}

template <int DT, int D>
int select_type(const SelectArgs& a, hipStream_t s) {
  constexpr int GROUPS = ST / RowT<DT, D>::LPR;
  const int64_t rows = (int64_t)(a.share < a.tok.max_tokens ? a.share : a.tok.max_tokens) << a.gshift;
  const size_t sums = (size_t)(rows < GROUPS ? rows : GROUPS) * 2 * D * 8, keys = (size_t)(a.len >> a.bshift) * 8;
  const size_t bytes = sums > keys ? sums : keys;
  allow_lds((const void*)select_kernel<DT, D>, bytes);
  hipLaunchKernelGGL((select_kernel<DT, D>), dim3((unsigned)(a.batch * a.hk * a.groups)), dim3(ST), bytes, s, a);
  return (int)hipGetLastError();
}

// ------------------------------------------------------------------------ attention

template <int DT, int D>
int blocks_type(const BlockArgs& a, hipStream_t s) {
  const int64_t wgs = (int64_t)a.batch * a.hk * a.ntiles * a.splits;
  const int rc = launch_tiles<DT, D, BLOCKS>(a, wgs, s);
  return rc == 0 && a.splits > 1 ? launch_join<DT, D, BLOCKS>(a, s) : rc;
}

}  // namespace

int launch_bounds(const BoundsArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? bounds_type<1, 128>(a, s) : bounds_type<1, 64>(a, s);
  return D == 128 ? bounds_type<0, 128>(a, s) : bounds_type<0, 64>(a, s);
}

bool select_fits(const SelectArgs& a, size_t& key_bytes) {
  key_bytes = 0;
  return (a.len >> a.bshift) <= MAX_BLOCKS && (int64_t)a.batch * a.hk * a.groups < (1 << 23);
}

int launch_select(const SelectArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? select_type<1, 128>(a, s) : select_type<1, 64>(a, s);
  return D == 128 ? select_type<0, 128>(a, s) : select_type<0, 64>(a, s);
}

bool block_plan(BlockArgs& a, int dtype, int D, int L) {
  const int S = 1 << a.bshift;
  const int64_t share = a.share < a.tok.max_tokens ? a.share : a.tok.max_tokens, rows = share << a.gshift;
  const int64_t lists = (int64_t)a.batch * a.hk * a.groups;
  // keys of a list: the chosen blocks, and the rows behind the complete ones
  const int64_t old = L - a.tok.max_tokens, whole = (int64_t)a.count * S < old / S * S ? (int64_t)a.count * S : old / S * S;
  const int64_t keys = whole + (old < S - 1 ? old : S - 1) + a.tok.max_tokens;
  auto tiles = [&](int bm) { return lists * ((rows + bm - 1) / bm); };
  const int64_t bytes = lists * keys * 2 * D * (dtype == 1 ? 2 : 4);
  // as in attend_plan
  const bool stream = dtype == 1 && D == 128 && a.groups == 1 && bytes > BIG_CACHE / 4 * 3;
  const int64_t parts = (keys + MIN_CHUNK - 1) / MIN_CHUNK;
  int bm = 128;
  if (!stream && (rows <= 32 || tiles(128) * parts < CUS)) bm = 32;
  else if (!stream && rows <= 64 && dtype == 1) bm = 64;
  const int per_cu = dtype == 1 ? (bm == 128 || D == 64 ? 2 : 1) : bm == 128 && D == 64 ? 2 : 1;
  // (parts by the tiles of 128 at most, whatever the lengths: the workspace grows with the cache)
  int64_t most = 4 * CUS / tiles(128);
  most = most > parts ? parts : most;
  most = most > MAX_PARTS ? MAX_PARTS : most < 1 ? 1 : most;
  const int bn = bm == 128 ? (dtype == 1 ? 64 : 32) : dtype == 1 || D == 64 ? 128 : 64;
  const double step = dtype == 1 ? 0.5 + 0.8 * D / 128 : 3.6 * D / 128;
  double least = -1.0;
  for (int64_t n = 1; n <= most; ++n) {
    const int64_t c = ((keys + n - 1) / n + MIN_CHUNK - 1) / MIN_CHUNK * MIN_CHUNK, real = (keys + c - 1) / c;
    const int64_t wgs = tiles(bm) * real, rounds = (wgs + per_cu * CUS - 1) / (per_cu * CUS);
    const double walk = (double)rounds * ((c + bn - 1) / bn) * step * (per_cu == 2 && wgs > CUS ? 1.55 : 1.0);
    const double join = real > 1 ? 3.0 + (double)a.tok.tokens * a.hq * real * D * 8 / 3.5e6 : 0.0;
    if (least < 0.0 || walk + join < least) {
      least = walk + join;
      a.splits = (int)real;
      a.chunk = (int)c;
    }
  }
  a.most_splits = (int)most;
  a.bm = bm;
  a.group_tiles = (int)((rows + bm - 1) / bm);
  a.ntiles = a.groups * a.group_tiles;
  a.once = a.ntiles == 1 && bytes > BIG_CACHE;
  return tiles(32) * most < (1 << 24) &&
         (int64_t)a.batch * a.hk * ((((int64_t)a.tok.max_tokens << a.gshift) + 3) / 4) < (1 << 24);
}

int launch_blocks(const BlockArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? blocks_type<1, 128>(a, s) : blocks_type<1, 64>(a, s);
  return D == 128 ? blocks_type<0, 128>(a, s) : blocks_type<0, 64>(a, s);
}

}  // namespace dc
