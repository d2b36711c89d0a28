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

// One pass over the keys: 128 units of 16384 rows of 128 bf16, 554 MB, 90 us = 6.1 TB/s, of the 6.3 that reads reach.
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
  // A workgroup's waves take one pass each, two where that still makes two workgroups a CU (4096 rows of 8 units of 128
  // bf16: 3.8 and 5.1 us; of 32 units of 8192 rows 12.4 and 11.6, with 16 passes 33.6)
  constexpr int RPI = 64 / RowT<DT, D>::LPR;
  const int loads = (1 << a.bshift) / RPI, pass = BT / 64 * (loads < 8 ? 8 / loads : 1);
  const int per = (int64_t)n * a.units >= 4 * CUS * pass ? 2 * pass : pass;
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

constexpr int ST = 256;                  // threads of a workgroup
constexpr int SW = ST / 64;
constexpr int MAX_BLOCKS = 16384;        // of a unit: their ranks fill a workgroup's registers
constexpr int QG = 8, QN = 8;            // lane groups that sum the queries, and loads of each under way

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

template <int CTRL>
__device__ __forceinline__ double dpp_f64(double x) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, 0xF, 0xF, true);
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, 0xF, 0xF, true), lo);
}

// Of 2 N numbers the sums with the partner lane's of N: the upper ones where `upper`, as it is not there.
template <int CTRL, int N>
__device__ __forceinline__ void fold(double* s, bool upper) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double give = upper ? s[i] : s[i + N], keep = upper ? s[i + N] : s[i];
    s[i] = keep + dpp_f64<CTRL>(give);
  }
}

// Where a list is, and its candidates.
struct Choice {
  int b, g, u, t0, r0, r1, cand;
  int32_t* list;
};
__device__ __forceinline__ Choice choice_of(const SelectArgs& a, int index) {
  Choice c;
  const int pairs = a.batch * a.hk, pair = index % pairs, group = index / pairs;
  int n;
  c.b = pair / a.hk;
  c.g = pair % a.hk;
  c.u = (c.b * a.n_layers + a.layer) * a.hk + c.g;
  token_range(a.tok, c.b, c.t0, n);
  c.r0 = group * a.share;
  c.r1 = c.r0 + a.share < n ? c.r0 + a.share : n;
  c.cand = c.r0 < n ? 1 : 0;               // (candidates_of counts them)
  c.list = a.list + ((size_t)(c.b * a.groups + group) * a.hk + c.g) * a.count;
  return c;
}

__device__ __forceinline__ void candidates_of(const SelectArgs& a, Choice& c) {
  if (c.cand) c.cand = __builtin_amdgcn_readfirstlane(rows_before(a.unit_len, a.len, c.u) >> a.bshift);
}

// Ranks of the blocks j0 .. j0 + chunk - 1 to keys[j]; false if there are none or no choice is to be made.
// The scores are binary64: products of bf16 elements are exact there and sums all but exact, so that a choice
// next to its limit does not hang on the order of a sum.
template <int DT, int D>
__device__ __forceinline__ bool score_blocks(const SelectArgs& a, Choice& w, int j0, int chunk, double* part,
                                             uint64_t* keys) {
  using R = RowT<DT, D>;
  constexpr int LPR = R::LPR, EPL = R::EPL, LPB = 2 * LPR, BPL = 64 / LPB;
  constexpr int UN = 8, STEP = UN * BPL;      // loads of a lane at a time, and the blocks of a wave's
  __shared__ double qs[2 * D];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // LPB lanes a block, 16 bytes each; the first ones are under way while the queries are summed
  const int c = lane % LPB;
  const char* bounds = (const char*)a.bounds + (size_t)w.u * (a.cap >> a.bshift) * (2 * D * R::ELT) + c * 16;
  uint4 x[UN];
  auto load = [&](int j, int end) DC_INLINE {
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int at = j + i * BPL + lane / LPB;
      x[i] = ldg16(bounds + (size_t)(at < end ? at : end - 1) * (2 * D * R::ELT));
    }
  };
  // sums of the queries' positive and negative elements: a lane group a row, QG of them in turn, QN rows under way
  const int rows = (w.r1 - w.r0) << a.gshift, used = rows < QG ? rows : QG;
  const int qc = tid % LPR, qg = tid / LPR;
  uint4 qr[QN];
  auto load_rows = [&](int i0) DC_INLINE {
#pragma unroll
    for (int x = 0; x < QN; ++x) {
      int i = i0 + x * QG;
      i = i < rows ? i : rows - 1;
      const size_t row = (size_t)(w.t0 + w.r0 + (i >> a.gshift)) * a.hq + (w.g << a.gshift) + (i & ((1 << a.gshift) - 1));
      qr[x] = ldg16((const char*)a.q + row * (D * R::ELT) + qc * 16);
    }
  };
  static_assert(ST / LPR >= QG, "a lane group for each");
  const int bound = a.len >> a.bshift;
  int j = j0 + wave * STEP;
  if (bound > a.count && w.cand) {
    if (qg < used) load_rows(qg);
    load(j, bound);                  // (the unit's own length is still on its way)
  }
  candidates_of(a, w);
  const int j1 = j0 + chunk < w.cand ? j0 + chunk : w.cand;
  if (w.cand <= a.count || j0 >= j1) return false;
  if (qg < used) {
    double up[EPL] = {}, down[EPL] = {};
    for (int i0 = qg;;) {
#pragma unroll
      for (int x = 0; x < QN; ++x) {
        float f[EPL];
        unpack_slice<DT>(qr[x], f);
        if (i0 + x * QG < rows) {
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            // (NaN stays one in both)
            up[e] += f[e] < 0.0f ? 0.0 : (double)f[e];
            down[e] += f[e] > 0.0f ? 0.0 : (double)f[e];
          }
        }
      }
      i0 += QN * QG;
      if (i0 >= rows) break;
      load_rows(i0);
    }
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      part[(qg * 2) * D + qc * EPL + e] = up[e];
      part[(qg * 2 + 1) * D + qc * EPL + e] = down[e];
    }
  }
  __syncthreads();
  for (int e = tid; e < 2 * D; e += ST) {
    double s = part[e];
    for (int i = 1; i < used; ++i) s += part[i * 2 * D + e];
    qs[e] = s;
  }
  __syncthreads();
  double q[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) q[e] = qs[c * EPL + e];
  for (; j < j1; j += SW * STEP) {
    double s[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      float f[EPL];
      unpack_slice<DT>(x[i], f);
      s[i] = 0.0;
#pragma unroll
      for (int e = 0; e < EPL; ++e) s[i] = __builtin_fma((double)f[e], q[e], s[i]);
    }
    load(j + SW * STEP, j1);
    // sums over the block's lanes: three exchanges in a row of 16 that also leave each lane two of the eight, then
    // one, and with its neighbour's
    fold<DPP_MIRROR, 4>(s, lane & 8);
    fold<DPP_HALF_MIRROR, 2>(s, lane & 4);
    fold<DPP_XOR1, 1>(s, lane & 1);
    s[0] += dpp_f64<DPP_XOR2>(s[0]);
#pragma unroll
    for (int bit = 16; bit < LPB; bit *= 2) s[0] += shfl_xor_f64(s[0], bit);
    const int at = j + ((c >> 1 & 4) + (c >> 1 & 2) + (c & 1)) * BPL + lane / LPB;
    if (c < 16 && !(c & 2) && at < j1) keys[at] = rank_of(s[0]);
  }
  return true;
}

// The first and last blocks are in; of the others, head .. tail - 1, the `need` highest.  They are found by halving
// an interval of ranks: at least `need` are at or above lo, fewer at or above hi, until exactly `need` are
// at or above its middle or lo is the last of them, whose equals are taken by the lowest numbers.
struct Limits {
  int head, tail, need;
};
__device__ __forceinline__ Limits limits_of(const SelectArgs& a, int cand) {
  Limits l;
  l.head = a.first < cand ? a.first : cand;
  l.tail = cand - a.last > l.head ? cand - a.last : l.head;
  l.need = a.count - l.head - (cand - l.tail);
  return l;
}

__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)), lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  return (uint64_t)hi << 32 | lo;
}

// Exclusive sums of N counts in LDS, in place, by the first wave.
template <int N>
__device__ __forceinline__ void sum_counts(int* x) {
  const int lane = threadIdx.x & 63;
  int before = 0;
#pragma unroll
  for (int i = 0; i < N; i += 64) {
    const int y = i + lane < N ? x[i + lane] : 0;
    int s = y;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const int o = __shfl_up(s, off);
      s = lane >= off ? s + o : s;
    }
    if (i + lane < N) x[i + lane] = before + s - y;
    before += __shfl(s, 63);
  }
}

// By W waves, K ranks a lane in registers: x[k] of number (k W + wave) 64 + lane.
template <int K, int W>
__device__ __forceinline__ void pick(const Limits& l, int cand, uint64_t* x, int32_t* list) {
  __shared__ int cells[2][W], counts[K * W];
  __shared__ uint64_t ends[2][W];
  const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
  uint64_t lo = ~0ull, hi = 0;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int j = (k * W + wave) * 64 + lane;
    const bool in = j >= l.head && j < l.tail;
    lo = in && x[k] < lo ? x[k] : lo;
    hi = in && x[k] > hi ? x[k] : hi;
    if (!in) x[k] = 0;                       // (no limit that is counted against is 0)
  }
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const uint64_t y = __shfl_xor(lo, off), z = __shfl_xor(hi, off);
    lo = y < lo ? y : lo;
    hi = z > hi ? z : hi;
  }
  if constexpr (W > 1) {
    if (lane == 0) {
      ends[0][wave] = lo;
      ends[1][wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = ends[0][w] < lo ? ends[0][w] : lo;
      hi = ends[1][w] > hi ? ends[1][w] : hi;
    }
  }
  lo = uniform(lo);
  hi = uniform(hi) + 1;
  int ties = l.need;
  if (l.need <= 0) {
    lo = hi;
    ties = 0;
  }
  for (int step = 0; hi - lo > 1; ++step) {
    const uint64_t mid = lo + (hi - lo) / 2;
    int n = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) n += __popcll(__ballot(x[k] >= mid));
    if constexpr (W > 1) {                   // (two cells in turn: one barrier a step)
      if (lane == 0) cells[step & 1][wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) n += cells[step & 1][w];
      n = __builtin_amdgcn_readfirstlane(n);
    }
    if (n >= l.need) lo = mid;
    else {
      hi = mid;
      ties = l.need - n;
    }
    if (n == l.need) {
      --lo;
      ties = 0;
      break;
    }
  }
  const uint64_t below = (1ull << lane) - 1;
  auto is_in = [&](int k) DC_INLINE {
    const int j = (k * W + wave) * 64 + lane;
    return j >= l.head && j < l.tail;
  };
  int first[K];
  auto tally = [&](auto flag) DC_INLINE {       // first[k]: flags before number k of this wave's
    int at = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int n = __popcll(__ballot(flag(k)));
      first[k] = at;
      at += n;
      if (W > 1 && lane == 0) counts[k * W + wave] = n;
    }
    if constexpr (W > 1) {
      __syncthreads();
      if (wave == 0) sum_counts<K * W>(counts);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) first[k] = counts[k * W + wave];
    }
  };
  tally([&](int k) DC_INLINE { return is_in(k) && x[k] == lo; });
  uint64_t taken = 0;                           // bit k: number k of this lane's is taken
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int j = (k * W + wave) * 64 + lane;
    const bool in = is_in(k), equal = in && x[k] == lo;
    const int before = first[k] + __popcll(__ballot(equal) & below);
    if ((j < cand && !in) || (in && x[k] > lo) || (equal && before < ties)) taken |= 1ull << k;
  }
  if constexpr (W > 1) __syncthreads();         // all have read the counts
  tally([&](int k) DC_INLINE { return (taken >> k) & 1; });
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const bool take = (taken >> k) & 1;
    const uint64_t m = __ballot(take);
    if (take) list[first[k] + __popcll(m & below)] = (k * W + wave) * 64 + lane;
  }
}

constexpr int ONE_WAVE = 512;            // most candidates that one wave picks among
constexpr int ONE_LAUNCH = 1024;         // most of the kernel that also scores

template <int K, int W>
__device__ __forceinline__ void pick_from(const SelectArgs& a, const Choice& w, const uint64_t* keys) {
  const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : threadIdx.x >> 6;
  uint64_t x[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int j = (k * W + wave) * 64 + lane;
    x[k] = j < w.cand ? keys[j] : 0;
  }
  pick<K, W>(limits_of(a, w.cand), w.cand, x, w.list);
}

// Lists whose choice is all candidates, or that no token has.
__device__ __forceinline__ void pick_whole(const SelectArgs& a, const Choice& w) {
  for (int i = threadIdx.x; i < a.count; i += blockDim.x) w.list[i] = i < w.cand ? i : -1;
}

// One workgroup per list.  64 of up to 512 blocks for 128 lists 13 us (in two launches 8.9 + 5.9): latency of queries and
// first bounds, then about 1 us for every 64 blocks, the vector instructions of the list's CU (512 and 1024 threads take
// 12.8 and 12.9).  1056 lists of 256 blocks 20 us, with 512 threads 25.  (Matrix cores form binary64 products at
// the vector rate, so they stay here.)
template <int DT, int D>
__global__ void __launch_bounds__(ST) select_kernel(SelectArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Choice w = choice_of(a, blockIdx.x);
  uint64_t* keys = reinterpret_cast<uint64_t*>(lds);
  if (!score_blocks<DT, D>(a, w, 0, MAX_BLOCKS, reinterpret_cast<double*>(lds), keys)) {
    pick_whole(a, w);
    return;
  }
  __syncthreads();
  if (w.cand > ONE_WAVE) pick_from<ONE_LAUNCH / ST, SW>(a, w, keys);
  else if (threadIdx.x < 64) w.cand <= 256 ? pick_from<4, 1>(a, w, keys) : pick_from<8, 1>(a, w, keys);
}

// Few lists of many blocks (1562 for 8 lists: 4.7 + 7.7 us, in one launch 45): `chunk` blocks of a list a
// workgroup to the workspace, then a workgroup per list.
template <int DT, int D>
__global__ void __launch_bounds__(ST) score_kernel(SelectArgs a) {
  __shared__ double part[QG * 2 * D];
  const int lists = a.batch * a.hk * a.groups, index = blockIdx.x % lists;
  Choice w = choice_of(a, index);
  score_blocks<DT, D>(a, w, (int)(blockIdx.x / lists) * a.chunk, a.chunk, part, a.keys + (size_t)index * a.ld_keys);
}

template <int K, int W>
__global__ void __launch_bounds__(64 * W) pick_kernel(SelectArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bound = a.len >> a.bshift;
  const uint64_t* keys = a.keys + (size_t)blockIdx.x * a.ld_keys;
  uint64_t x[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {             // (within the longest unit's: the unit's own length is still on its way)
    const int j = (k * W + wave) * 64 + lane;
    x[k] = keys[j < bound ? j : bound - 1];
  }
  Choice w = choice_of(a, blockIdx.x);
  candidates_of(a, w);
  if (w.cand <= a.count) pick_whole(a, w);
  else pick<K, W>(limits_of(a, w.cand), w.cand, x, w.list);
}

template <int K, int W>
void launch_pick(const SelectArgs& a, int lists, hipStream_t s) {
  hipLaunchKernelGGL((pick_kernel<K, W>), dim3((unsigned)lists), dim3(64 * W), 0, s, a);
}

template <int DT, int D>
int select_type(const SelectArgs& a, hipStream_t s) {
  const int lists = a.batch * a.hk * a.groups, blocks = a.len >> a.bshift;
  const size_t ranks = (size_t)blocks * 8;
  if (a.keys) {
    hipLaunchKernelGGL((score_kernel<DT, D>), dim3((unsigned)(lists * ((blocks + a.chunk - 1) / a.chunk))), dim3(ST), 0, s,
                       a);
    if (blocks <= 256) launch_pick<4, 1>(a, lists, s);
    else if (blocks <= ONE_WAVE) launch_pick<8, 1>(a, lists, s);
    else if (blocks <= 1024) launch_pick<4, SW>(a, lists, s);
    else if (blocks <= 2048) launch_pick<8, SW>(a, lists, s);
    else if (blocks <= 4096) launch_pick<16, SW>(a, lists, s);
    else launch_pick<MAX_BLOCKS / ST, SW>(a, lists, s);
    return (int)hipGetLastError();
  }
  const size_t sums = QG * 2 * D * sizeof(double), bytes = sums > ranks ? sums : ranks;
  allow_lds((const void*)select_kernel<DT, D>, bytes);
  hipLaunchKernelGGL((select_kernel<DT, D>), dim3((unsigned)lists), dim3(ST), bytes, s, a);
  return (int)hipGetLastError();
}

// ------------------------------------------------------------------------ attention
// 16 tokens over 64 of 512 blocks of 64 rows (32/8 heads of 128), 270 MB, 46 us = 5.9 TB/s and 4.6 for the join; 512
// tokens, 32 of them together over 64 blocks, 61 and 7.6: waits for tiles in 48 % of the waves' cycles (56 % of their
// lines come from beyond the L2), and parts of the longest list that there may be, which are longer than these lists need.

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

bool select_plan(SelectArgs& a, size_t& key_bytes) {
  const int blocks = a.len >> a.bshift;
  const int64_t lists = (int64_t)a.batch * a.hk * a.groups;
  key_bytes = 0;
  a.chunk = 0;
  if (blocks > MAX_BLOCKS || lists >= (1 << 23)) return false;
  if (blocks > a.count && ((lists < CUS && blocks > ONE_WAVE) || blocks > ONE_LAUNCH)) {
    // chunks that make about two workgroups a CU, of a step of the workgroup at least
    const int64_t per = (2 * CUS + lists - 1) / lists;
    const int64_t chunk = ((blocks + per - 1) / per + 63) / 64 * 64;
    a.chunk = (int)chunk;
    a.ld_keys = (blocks + 1) / 2 * 2;
    key_bytes = ((size_t)lists * a.ld_keys * 8 + 255) & ~(size_t)255;
  }
  return true;
}

int select_max_blocks() { return MAX_BLOCKS; }

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
  const int64_t old = L - a.tok.max_tokens, chosen = (int64_t)a.count * S;
  const int64_t whole = chosen < old / S * S ? chosen : old / S * S;
  const int64_t keys = whole + (old < S - 1 ? old : S - 1) + a.tok.max_tokens;
  auto tiles = [&](int bm) { return lists * ((rows + bm - 1) / bm); };
  const int64_t bytes = lists * keys * 2 * D * (dtype == 1 ? 2 : 4);
  const int64_t parts = (keys + MIN_CHUNK - 1) / MIN_CHUNK;
  // (parts by the tiles of 128 at most, whatever the lengths: the workspace grows with the cache)
  int64_t most = 4 * CUS / tiles(128);
  most = most > parts ? parts : most;
  most = most > MAX_PARTS ? MAX_PARTS : most < 1 ? 1 : most;
  // Tiles and parts by their time; the lists are alike, so a last round of few workgroups is a whole one
  double least = -1.0;
  for (int bm = 32; bm <= 128; bm *= 2) {
    if (bm == 64 && dtype != 1) continue;
    const Cut cut = cut_of(dtype, D, bm, rows);
    const int64_t slots = cut.per_cu * CUS, all = tiles(bm);
    const uint32_t walk = keys;
    uint32_t last = 0;
    for (const uint32_t n : PARTS) {
      if (n > most) break;
      const uint32_t c = ((walk + n - 1) / n + MIN_CHUNK - 1) / MIN_CHUNK * MIN_CHUNK, real = (walk + c - 1) / c;
      if (c == last) continue;
      last = c;
      const int64_t wgs = all * real;
      const double us = cut_us(cut, (double)((wgs + slots - 1) / slots), ((c < walk ? c : walk) + cut.bn - 1) / cut.bn,
                               (double)keys / cut.bn / real, real, (double)a.tok.tokens * a.hq, D);
      if (least >= 0.0 && us >= least) continue;
      least = us;
      a.bm = bm;
      a.splits = (int)real;
      a.chunk = (int)c;
    }
  }
  a.most_splits = (int)most;
  a.group_tiles = (int)((rows + a.bm - 1) / a.bm);
  a.ntiles = a.groups * a.group_tiles;
  a.once = a.ntiles == 1 && bytes > BIG_CACHE;
  return tiles(32) * most < (1 << 24) &&
         (most == 1 || (int64_t)a.batch * a.hk * ((((int64_t)a.tok.max_tokens << a.gshift) + 3) / 4) < (1 << 24));
}

int launch_blocks(const BlockArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1) return D == 128 ? blocks_type<1, 128>(a, s) : blocks_type<1, 64>(a, s);
  return D == 128 ? blocks_type<0, 128>(a, s) : blocks_type<0, 64>(a, s);
}

}  // namespace dc
