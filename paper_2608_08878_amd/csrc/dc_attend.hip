// Attention of several new tokens per sequence over cache rows, on gfx950 matrix cores:
// a prompt (or its next chunk), causal, or a tree of drafted tokens.  The tokens' own K/V
// rows are in the cache already, behind the rows that were there (slots len_u + r).
//
//   o = sum_i a_i v_i,  a = softmax_i(scale q.k_i)  over the rows i that the token sees:
// every row below len_u, and of the tokens' own row len_u + r' for r' <= r (prompt) or for r' = r
// and the ancestors of r (tree).
//
// A row here is a (token, query head) pair of one KV head, token-major (row = token G + j), so the
// G heads that share K/V share its tiles.  A wave owns 32 rows and walks key tiles with a running
// maximum and sum.  It computes S^T = K Q^T with 32x32 MFMAs: the accumulator then holds 16 keys
// of one row per lane, so the softmax is lane-local but for one exchange between the wave's halves,
// and the same registers are the right operand of O^T += V^T P^T without any movement, the key
// order of the sum being free as long as V is read in the same one.  K and V tiles go from memory
// to LDS directly (their 16-byte chunks permuted at the source so that operand reads spread over the
// banks); bf16 V is read through the transposing LDS load.
#include <type_traits>

#include "dc_device.hpp"
#include "dc_kernels.hpp"
#include "distillcache.h"

#pragma clang fp contract(off)

namespace dc {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef short i16x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_c_t;

#define DC_INLINE __attribute__((always_inline))

constexpr int MAX_NODES = DC_TREE_MAX_NODES;
constexpr int MASK_WORDS = MAX_NODES / 32;
constexpr float NEG_INF = -__builtin_huge_valf();

// Rows of K and V in LDS.  Chunk c (16 bytes) of row r sits at position c ^ kx(r), c ^ vx(r).
template <int DT, int D>
struct KVT {
  static constexpr int E = DT == 0 ? 4 : 2;
  static constexpr int RB = D * E;            // bytes of a row
  static constexpr int CH = RB / 16;          // chunks of a row
  static constexpr int KT = CH / 2;           // 16-byte operand steps of a dot product
  // K: 32 lanes read the same chunk of 32 rows; 16 bank groups of 16 bytes
  __device__ static __forceinline__ int kx(int r) { return r & (CH < 16 ? CH - 1 : 15); }
  // V, bf16: 16 lanes read 32 bytes of each of 4 rows; f32: 32 lanes read 128 bytes of row r,
  // the others of row r + 4
  __device__ static __forceinline__ int vx(int r) {
    if constexpr (DT == 0) return 8 * ((r >> 2) & 1);
    return CH == 16 ? 4 * (r & 3) : 4 * ((r >> 1) & 1);
  }
};

__device__ __forceinline__ float half_max(float x) {   // over the wave's two halves
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(lds_c_t*)p;
}

// Factor of sums taken against the maximum m when the maximum becomes mn.  Maxima are kept as
// fl(scale log2(e) max s), the number that the exponents subtract, so that its rounding is the
// same in every term of a row and cancels.
__device__ __forceinline__ float rescale(float m, float mn) {
  return m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
}

// A row keeps its maximum while no key exceeds it by more than this (in powers of two): weights are
// then at most 2^SLACK instead of 1, which float32 sums and bf16 weights hold as well, and the
// accumulators are rescaled once or twice in a long row instead of at every new maximum.  Values near the
// type's largest can overflow by it; the pass that follows a result that is not finite keeps none.
constexpr float SLACK = 8.0f;

// Key held by accumulator register i of a lane in half h of the wave: bit i of a 32-key block.
__device__ __forceinline__ int key_of(int i, int h) { return 8 * (i / 4) + 4 * h + i % 4; }

// S^T of 32 keys (LDS rows kr .. kr + 31 at k) and the wave's 32 rows.
template <int DT, int D>
__device__ __forceinline__ f32x16_t scores32(const char* k, const uint4* qf, int lane) {
  using T = KVT<DT, D>;
  const int r = lane & 31, h = lane >> 5;
  const char* row = k + r * T::RB;
  f32x16_t s = {};
#pragma unroll
  for (int t = 0; t < T::KT; ++t) {
    const uint4 kf = *reinterpret_cast<const uint4*>(row + ((2 * t + h) ^ T::kx(r)) * 16);
    if constexpr (DT == 1) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf),
                                                  __builtin_bit_cast(bf16x8_t, qf[t]), s, 0, 0, 0);
    } else {
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.x), __uint_as_float(qf[t].x), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.y), __uint_as_float(qf[t].y), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.z), __uint_as_float(qf[t].z), s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf.w), __uint_as_float(qf[t].w), s, 0, 0, 0);
    }
  }
  return s;
}

// The weights of 32 keys as the matrix cores take them; p[i] is that of key key_of(i, h).  bf16: each
// is rounded by up to half a step, 2^-8 of itself.  Their sum is taken of the rounded ones, so that
// the output is a mean by the weights that were used: where one key has nearly all weight its rounding
// cancels (relative error of the outputs, two prompts of 8192 tokens: 0.0017, with the sum of the unrounded
// ones 0.0019).
template <int DT>
struct Weights {
  f32x16_t f;
  __device__ __forceinline__ void set(const f32x16_t& p, float& l) {
    f = p;
#pragma unroll
    for (int i = 0; i < 16; ++i) l += p[i];
  }
};
template <>
struct Weights<1> {
  bf16x8_t b[2];
  __device__ __forceinline__ void set(const f32x16_t& p, float& l) {
    const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f32x8_t x;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = p[8 * s + j];
      b[s] = __builtin_convertvector(x, bf16x8_t);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        l = __builtin_amdgcn_fdot2_f32_bf16(bf16x2_t{b[s][2 * j], b[s][2 * j + 1]}, one, l, false);
    }
  }
};

// O^T += V^T P^T over 32 keys.
template <int DT, int D>
__device__ __forceinline__ void values32(const char* v, const Weights<DT>& p, f32x16_t* o, int lane) {
  using T = KVT<DT, D>;
  const int h = lane >> 5;
  if constexpr (DT == 1) {
    const int i = lane & 15, dsub = (lane >> 4) & 1;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int r0 = 16 * s + 4 * h + i / 4, r1 = r0 + 8;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int c = 4 * db + 2 * dsub + (i & 3) / 2, off = (i & 1) * 8;
        const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) i16x4_t*)(v + r0 * T::RB + (c ^ T::vx(r0)) * 16 + off));
        const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) i16x4_t*)(v + r1 * T::RB + (c ^ T::vx(r1)) * 16 + off));
        const i16x8_t vf = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf), p.b[s], o[db], 0, 0, 0);
      }
    }
  } else {
    const int dl = lane & 31;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = key_of(i, h);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int c = 8 * db + dl / 4;
        const float vf = *reinterpret_cast<const float*>(v + r * T::RB + (c ^ T::vx(r)) * 16 + (dl & 3) * 4);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, p.f[i], o[db], 0, 0, 0);
      }
    }
  }
}

// The same sum key by key, leaving out the keys whose bit in `sees` is clear: a masked value row
// that is infinite or NaN reaches no row that does not see it (0 times it is NaN).
template <int DT, int D>
__device__ __forceinline__ void values32_masked(const char* v, const f32x16_t& p, uint32_t sees, f32x16_t* o,
                                             int lane) {
  using T = KVT<DT, D>;
  const int h = lane >> 5;
  for (int kk = 0; kk < 32; ++kk) {
    float w = 0.0f;
    const int i = 4 * (kk / 8) + kk % 4, hk = (kk >> 2) & 1;
#pragma unroll
    for (int x = 0; x < 16; ++x) w = i == x ? p[x] : w;
    w = __shfl(w, (lane & 31) + 32 * hk);
    if constexpr (DT == 1) w = __builtin_bit_cast(float, (uint32_t)f32_to_bf16_bits(w) << 16);
    const bool on = (sees >> kk) & 1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int d = 32 * db + key_of(x, h);
        const char* at = v + kk * T::RB + ((d * T::E / 16) ^ T::vx(kk)) * 16 + (d * T::E) % 16;
        float vf;
        if constexpr (DT == 1) vf = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16);
        else vf = *reinterpret_cast<const float*>(at);
        if (on) o[db][x] = __builtin_fmaf(w, vf, o[db][x]);
      }
  }
}

// Row tiles of 32 RW rows; the key tile of SK KW keys is shared by the RW row waves, or cut among
// KW groups of them, whose partial results are joined at the end.
template <int DT, int D, int RW, int KW, int SK>
struct Cfg {
  static constexpr int NW = RW * KW, THREADS = 64 * NW, BM = 32 * RW, BN = SK * KW;
  static constexpr int TILE = BN * KVT<DT, D>::RB;        // bytes of a K (or V) tile
  static constexpr int BUF = 2 * TILE;
  static constexpr int OB = 32 * D * 4 + 256;             // one wave's partial result
  static constexpr int LDS = 2 * BUF;
  // workgroups of a CU by their LDS; their waves on a SIMD
  static constexpr int WAVES = 2 * LDS <= 144 * 1024 && NW == 4 && !(DT == 0 && D == 128) ? 2 : 1;
  static_assert((KW - 1) * RW * OB <= LDS && RW * 128 * D <= LDS, "results fit the tile buffers");
  static_assert(TILE % 1024 == 0 && SK % 32 == 0, "tile shape");
};

// Where a workgroup's row tile and keys are.
struct Place {
  int u, g, t0, n;              // unit, KV head, first packed token and tokens of the sequence
  int start, total;             // rows before the tokens' own, and with them
  int rows, row0;               // (token, head) rows, the tile's first
  int split, k0, k1;            // the part of the keys: k0 .. k1 - 1
};

// One launch index per (row tile, key part, sequence and KV head), the pairs fastest: with a
// multiple of 8 of them a pair's workgroups share one XCD's L2.  The tiles with the most keys
// go first.  False where nothing is to be done (the whole workgroup).
template <bool TREE>
__device__ __forceinline__ bool locate(const AttendArgs& a, int bm, Place& w) {
  const int pairs = a.batch * a.hk;
  const int pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
  const int tile = a.ntiles - 1 - rest / a.splits;
  const int b = pair / a.hk;
  w.split = rest % a.splits;
  w.g = pair % a.hk;
  w.u = (b * a.n_layers + a.layer) * a.hk + w.g;
  token_range(a.tok, b, w.t0, w.n);
  w.t0 = __builtin_amdgcn_readfirstlane(w.t0);      // uniform, and known to be
  w.n = __builtin_amdgcn_readfirstlane(w.n);
  w.rows = w.n << a.gshift;
  w.row0 = tile * bm;
  if (w.row0 >= w.rows) return false;
  w.start = __builtin_amdgcn_readfirstlane(rows_before(a.unit_len, a.len, w.u));
  w.total = w.start + w.n;
  const int last = (w.row0 + bm < w.rows ? w.row0 + bm : w.rows) - 1;
  const int kend = TREE ? w.total : w.start + (last >> a.gshift) + 1;   // keys any row of the tile sees
  w.k0 = w.split * a.chunk;
  w.k1 = w.k0 + a.chunk < kend ? w.k0 + a.chunk : kend;
  return w.k0 < w.k1;
}

// Ancestors of every node as bits (a node is its own), by doubling the step up the tree.  A parent
// that is not an earlier node of the sequence counts as none.
template <int THREADS>
__device__ __forceinline__ void ancestors(const AttendArgs& a, const Place& w, uint32_t* anc, int* up) {
  constexpr int PER = (MAX_NODES + THREADS - 1) / THREADS;       // nodes of a thread
  const int n = w.n, words = (n + 31) / 32;
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int p = a.parent[w.t0 + i];
    up[i] = p >= 0 && p < i ? p : -1;
    for (int x = 0; x < words; ++x) anc[i * MASK_WORDS + x] = x == i / 32 ? 1u << (i & 31) : 0u;
  }
  __syncthreads();
  for (int step = 1; step < n; step *= 2) {
    uint32_t m[PER][MASK_WORDS];
    int p[PER], pp[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = threadIdx.x + k * THREADS;
      p[k] = i < n ? up[i] : -1;
      pp[k] = p[k] >= 0 ? up[p[k]] : -1;
#pragma unroll
      for (int x = 0; x < MASK_WORDS; ++x) m[k][x] = p[k] >= 0 && x < words ? anc[p[k] * MASK_WORDS + x] : 0u;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = threadIdx.x + k * THREADS;
      if (p[k] < 0) continue;
      up[i] = pp[k];
#pragma unroll
      for (int x = 0; x < MASK_WORDS; ++x)
        if (x < words) anc[i * MASK_WORDS + x] |= m[k][x];
    }
    __syncthreads();
  }
}

// Which keys of the block kb .. kb + 31 token r sees.
template <bool TREE>
__device__ __forceinline__ uint32_t sees32(const Place& w, const uint32_t* anc, int r, int kb) {
  if constexpr (TREE) {
    const int d = kb - w.start;
    if (d <= -32) return ~0u;
    const uint32_t* m = anc + r * MASK_WORDS;
    const int words = (w.n + 31) / 32;
    if (d < 0) return m[0] << -d | ((1u << -d) - 1u);
    const int x = d >> 5, s = d & 31;
    const uint32_t lo = x < words ? m[x] : 0u, hi = x + 1 < words ? m[x + 1] : 0u;
    return s ? lo >> s | hi << (32 - s) : lo;
  } else {
    const int nv = w.start + r + 1 - kb;
    return nv >= 32 ? ~0u : nv <= 0 ? 0u : (1u << nv) - 1u;
  }
}

// Scores of the keys that a lane's row does not see become minus infinity.
__device__ __forceinline__ void mask32(f32x16_t& s, uint32_t sees, int h) {
  sees >>= 4 * h;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = (sees >> (8 * (i / 4) + i % 4)) & 1 ? s[i] : NEG_INF;
}

// A lane's row of the output (l over all its keys), or of its key part's share.
template <int DT, int D>
__device__ __forceinline__ void store_row(const AttendArgs& a, size_t qrow, int split, const f32x16_t* o, float m,
                                          float l, int h) {
  if (a.splits > 1) {
    float* po = a.part + (qrow * a.splits + split) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(po + 32 * db + 8 * q + 4 * h) =
            make_float4(o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]);
    if (h == 0)
      *reinterpret_cast<float2*>(a.part + (size_t)a.tok.tokens * a.hq * a.splits * D +
                                 (qrow * a.splits + split) * 2) = make_float2(m, l);
    return;
  }
  const float inv = 1.0f / l;
  char* out = (char*)a.out + qrow * KVT<DT, D>::RB;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = 32 * db + 8 * q + 4 * h;
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = o[db][4 * q + e] * inv;
      if constexpr (DT == 1)
        *reinterpret_cast<uint2*>(out + d * 2) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
      else
        *reinterpret_cast<float4*>(out + d * 4) = make_float4(f[0], f[1], f[2], f[3]);
    }
}

// The same of the wave's 32 rows.  A lane holds pieces of 16 bytes of one row; they cross LDS (`st`,
// 128 D bytes of the wave's own, chunk c of row r at c ^ r) so that the stores are whole rows (16
// prompts of up to 255 tokens 24.0 -> 20.6 us; a call of few rows, whose latency counts, is faster
// without: 512 float32 tokens 12.2, with 12.9).
template <int DT, int D>
__device__ __forceinline__ void store_rows(const AttendArgs& a, const Place& w, int wrow, char* st, const f32x16_t* o,
                                           float m, float l, int lane) {
  constexpr int CH = D / 4;                       // chunks of four floats of a row
  const int q = lane & 31, h = lane >> 5;
  const bool parts = a.splits > 1;
  const float inv = parts ? 1.0f : 1.0f / l;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      *reinterpret_cast<float4*>(st + (q * CH + ((8 * db + 2 * y + h) ^ (q & (CH - 1)))) * 16) =
          make_float4(o[db][4 * y] * inv, o[db][4 * y + 1] * inv, o[db][4 * y + 2] * inv, o[db][4 * y + 3] * inv);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // all pieces are in LDS before other lanes read them
  auto chunk = [&](int r, int c) DC_INLINE {
    return *reinterpret_cast<const float4*>(st + (r * CH + (c ^ (r & (CH - 1)))) * 16);
  };
  auto place = [&](int row) DC_INLINE -> size_t {
    return (size_t)(w.t0 + (row >> a.gshift)) * a.hq + (w.g << a.gshift) + (row & ((1 << a.gshift) - 1));
  };
  if (DT == 0 || parts) {
    float* to = parts ? a.part : (float*)a.out;
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      const int r = i * (64 / CH) + lane / CH, c = lane % CH;
      if (wrow + r < w.rows) {
        const size_t at = parts ? place(wrow + r) * a.splits + w.split : place(wrow + r);
        *reinterpret_cast<float4*>(to + at * D + c * 4) = chunk(r, c);
      }
    }
    if (parts && h == 0 && wrow + q < w.rows)
      reinterpret_cast<float2*>(a.part + (size_t)a.tok.tokens * a.hq * a.splits * D)[place(wrow + q) * a.splits +
                                                                                    w.split] = make_float2(m, l);
  } else {
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) {
      const int r = i * (128 / CH) + lane / (CH / 2), c = lane % (CH / 2);
      const float4 x = chunk(r, 2 * c), y = chunk(r, 2 * c + 1);
      if (wrow + r < w.rows)
        *reinterpret_cast<uint4*>((char*)a.out + place(wrow + r) * (2 * D) + c * 16) =
            make_uint4(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w), pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    }
  }
}

// Two prompts of 8192 tokens (32/8 heads of 128) 1045-1090 us = 1.0 PFLOP/s, where a large library product
// reaches 1.35: matrix cores busy 52 % of the cycles, vector instructions issued in 47 %, at a clock that the
// card's power holds at 1.6 to 1.8 GHz (the call on zeros 860).  Two waves a SIMD (256 registers each; one wave
// 1861) overlap one's softmax with the other's products.  Tried and not kept: three key blocks in hand in a
// wave 1075-1086, 64 rows a wave 1455, eight waves a workgroup 1105, tiles of 32 keys 1112.  64-element heads
// (4 x 2048 tokens, 64/8 heads, 180 us = 0.76 PFLOP/s; tiles of 128 keys 209) take twice the exponentials for a
// product: vector instructions in 64 %, matrix cores 37 %, and most products come right behind a wait for
// their operands from LDS.
// The compiler cannot see that the wait at a step's head covers the Q rows' loads too, and waits for them again
// before the step's first products, which by then is a wait for the next tile.  Prompts do not show it: built
// with those waits ahead of the loop they take the same (8192 tokens 1044 us, 64 elements 178), the tiles being
// in the L2.  Drafts over caches in HBM do: 320 tokens over 16 caches of up to 16384 rows, 834 MB, 171-178 us,
// without the waits 163.  The rest of that call is the lengths: parts are cut by the longest cache, so the
// shorter ones' last workgroups leave at once (16 caches of 16384 rows, 1.07 GB, one token each: 171).
template <int DT, int D, int RW, int KW, int SK, bool TREE>
__global__ void __launch_bounds__(64 * RW * KW, (Cfg<DT, D, RW, KW, SK>::WAVES)) attend_kernel(AttendArgs a) {
  using T = KVT<DT, D>;
  using C = Cfg<DT, D, RW, KW, SK>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  __shared__ uint32_t anc[TREE ? MAX_NODES * MASK_WORDS : 1];
  __shared__ int up[TREE ? MAX_NODES : 1];
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rw = wave % RW, kw = wave / RW;
  Place w;
  if (!locate<TREE>(a, C::BM, w)) return;
  const int k0 = w.k0, k1 = w.k1, total = w.total;
  // tile loads: 1024 bytes an instruction, the waves in turn; rows past the last are read as the last
  constexpr int LPW = C::TILE / 1024 / C::NW, RPI = 1024 / T::RB;    // instructions of a wave, rows of one
  const char* kc = (const char*)a.k + ((size_t)w.u * a.cap + k0) * T::RB;
  const char* vc = (const char*)a.v + ((size_t)w.u * a.cap + k0) * T::RB;
  const uint32_t lds0 = lds_offset(lds);
  uint32_t ko[LPW], vo[LPW];
#pragma unroll
  for (int x = 0; x < LPW; ++x) {
    const int row = (x * C::NW + wave) * RPI + lane / T::CH, p = lane % T::CH;
    ko[x] = row * T::RB + (p ^ T::kx(row)) * 16;
    vo[x] = row * T::RB + (p ^ T::vx(row)) * 16;
  }
  auto load_tile = [&](int it, int buf) DC_INLINE {
    const size_t at = (size_t)it * C::TILE;
    const int left = total - k0 - it * C::BN;
#pragma unroll
    for (int x = 0; x < LPW; ++x) {
      uint32_t back = 0;
      if (left < C::BN) {
        const int row = (x * C::NW + wave) * RPI + lane / T::CH;
        if (row >= left) back = (row - left + 1) * T::RB;
      }
      const uint32_t dst = lds0 + buf * C::BUF + (x * C::NW + wave) * 1024;
      if (a.once) {
        load_to_lds16_at_nt(kc + at, ko[x] - back, dst);
        load_to_lds16_at_nt(vc + at, vo[x] - back, dst + C::TILE);
      } else {
        load_to_lds16_at(kc + at, ko[x] - back, dst);
        load_to_lds16_at(vc + at, vo[x] - back, dst + C::TILE);
      }
    }
  };
  const int ntile = (k1 - k0 + C::BN - 1) / C::BN;
  load_tile(0, 0);        // under way while the rest is set up

  // this lane's row
  const int wrow = w.row0 + 32 * rw;
  const int myrow = wrow + (lane & 31) < w.rows ? wrow + (lane & 31) : w.rows - 1;
  const int r = myrow >> a.gshift;
  const bool active = wrow < w.rows;
  const size_t qrow = (size_t)(w.t0 + r) * a.hq + (w.g << a.gshift) + (myrow & ((1 << a.gshift) - 1));
  uint4 qf[T::KT];
#pragma unroll
  for (int t = 0; t < T::KT; ++t) qf[t] = ldg16((const char*)a.q + qrow * T::RB + (2 * t + h) * 16);
  const int wfirst = (wrow < w.rows ? wrow : w.rows - 1) >> a.gshift;            // the wave's first token
  const int wlast = (wrow + 31 < w.rows ? wrow + 31 : w.rows - 1) >> a.gshift;   // and its last
  const int full = TREE ? w.start : w.start + wfirst + 1;   // keys below are seen by all its rows
  const int some = TREE ? w.total : w.start + wlast + 1;    // keys from here on by none
  if constexpr (TREE) ancestors<C::THREADS>(a, w, anc, up);

  const float c = a.scale * LOG2E;
  f32x16_t o[D / 32];
  float m, l;
  // One pass over the keys.  CAREFUL: masked blocks go key by key, and weights are at most 1.
  auto pass = [&](auto careful) DC_INLINE {
    constexpr bool CAREFUL = decltype(careful)::value;
    m = NEG_INF;
    l = 0.0f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16_t{};
    // a tile in buffer BUF; the next one's loads go out first
    auto tile_step = [&](int it, auto bufc) DC_INLINE {
      constexpr int BUF = decltype(bufc)::value;
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
      if (it + 1 < ntile) load_tile(it + 1, 1 - BUF);
      const int kt = k0 + it * C::BN;
      const int kb = kt + kw * SK;
      if (!active || kb >= k1 || kb >= some) return;
      const char* kl = lds + BUF * C::BUF + kw * SK * T::RB;
      const char* vl = kl + C::TILE;
      f32x16_t s[SK / 32];
      float mx = NEG_INF;
      const bool masked = kb + SK > full;
#pragma unroll
      for (int x = 0; x < SK / 32; ++x) s[x] = scores32<DT, D>(kl + 32 * x * T::RB, qf, lane);
      if (masked) {
#pragma unroll
        for (int x = 0; x < SK / 32; ++x) mask32(s[x], sees32<TREE>(w, anc, r, kb + 32 * x), h);
      }
#pragma unroll
      for (int x = 0; x < SK / 32; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[x][i]);
      const float mn = fmaxf(m, half_max(mx) * c);
      if (__any(mn > m + (CAREFUL ? 0.0f : SLACK))) {
        const float f = rescale(m, mn);
        l *= f;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[db][i] *= f;
        m = mn;
      }
      const float mc = m == NEG_INF ? 0.0f : m;
#pragma unroll
      for (int x = 0; x < SK / 32; ++x) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i], c, -mc));
        Weights<DT> p;
        p.set(s[x], l);
        const char* vx = vl + 32 * x * T::RB;
        if (CAREFUL && masked)
          values32_masked<DT, D>(vx, s[x], sees32<TREE>(w, anc, r, kb + 32 * x), o, lane);
        else
          values32<DT, D>(vx, p, o, lane);
      }
    };
    if constexpr (CAREFUL) load_tile(0, 0);
    for (int it = 0; it < ntile; it += 2) {
      tile_step(it, std::integral_constant<int, 0>{});
      if (it + 1 < ntile) tile_step(it + 1, std::integral_constant<int, 1>{});
    }
  };
  pass(std::false_type{});
  // Again, carefully, only if a masked value row was met that is not finite (0 times it is NaN), or the
  // sums left float32's range.
  float z = 0.0f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[db][i], 0.0f, z);
  if (__syncthreads_or(active && !(z == 0.0f))) {
    pass(std::true_type{});
    __syncthreads();
  }
  l = half_sum(l);

  // join the key groups: group 0 takes the others' results from LDS
  if constexpr (KW > 1) {
    if (kw > 0) {
      char* p = lds + ((kw - 1) * RW + rw) * C::OB;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) reinterpret_cast<float*>(p)[(db * 16 + i) * 64 + lane] = o[db][i];
      if (h == 0) {
        reinterpret_cast<float*>(p + 32 * D * 4)[lane] = m;
        reinterpret_cast<float*>(p + 32 * D * 4)[32 + lane] = l;
      }
    }
    __syncthreads();
    if (kw > 0) return;
    float mm = m;
#pragma unroll
    for (int x = 1; x < KW; ++x)
      mm = fmaxf(mm, reinterpret_cast<const float*>(lds + ((x - 1) * RW + rw) * C::OB + 32 * D * 4)[lane & 31]);
    float f = rescale(m, mm);
    l *= f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= f;
#pragma unroll
    for (int x = 1; x < KW; ++x) {
      const char* p = lds + ((x - 1) * RW + rw) * C::OB;
      const float* ml = reinterpret_cast<const float*>(p + 32 * D * 4);
      const float mx = ml[lane & 31];
      f = rescale(mx, mm);
      l = __builtin_fmaf(ml[32 + (lane & 31)], f, l);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          o[db][i] = __builtin_fmaf(reinterpret_cast<const float*>(p)[(db * 16 + i) * 64 + lane], f, o[db][i]);
    }
    m = mm;
  }
  if constexpr (KW > 1) {
    if (wrow + (lane & 31) < w.rows) store_row<DT, D>(a, qrow, w.split, o, m, l, h);
  } else if (active) {
    store_rows<DT, D>(a, w, wrow, lds + rw * 128 * D, o, m, l, lane);
  }
}

// Joins the parts of the key range, a wave per row: lane x holds part x's maximum and sum, then the
// wave adds the parts' outputs, eight loads under way.
template <int DT, int D>
__global__ void __launch_bounds__(256) attend_join_kernel(AttendArgs a) {
  constexpr int EPL = D / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pairs = a.batch * a.hk;
  const int pair = blockIdx.x % pairs, row = (blockIdx.x / pairs) * 4 + wave;
  const int b = pair / a.hk, g = pair % a.hk;
  const int u = (b * a.n_layers + a.layer) * a.hk + g;
  int t0, n;
  token_range(a.tok, b, t0, n);
  if (row >= n << a.gshift) return;
  const int r = row >> a.gshift, head = (g << a.gshift) + (row & ((1 << a.gshift) - 1));
  const int keys = rows_before(a.unit_len, a.len, u) + (a.parent ? n : r + 1);
  const int parts = (keys + a.chunk - 1) / a.chunk;       // those that a kernel wrote: at most MAX_PARTS
  const size_t qrow = (size_t)(t0 + r) * a.hq + head;
  const float* po = a.part + qrow * a.splits * D + lane * EPL;
  const float2* ml = reinterpret_cast<const float2*>(a.part + (size_t)a.tok.tokens * a.hq * a.splits * D) +
                     qrow * a.splits;
  const float2 mine = lane < parts ? ml[lane] : make_float2(NEG_INF, 0.0f);
  float m = mine.x;
#pragma unroll
  for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
  const float f = lane < parts ? rescale(mine.x, m) : 0.0f;
  float l = mine.y * f, o[EPL] = {};
#pragma unroll
  for (int x = 1; x < 64; x *= 2) l += __shfl_xor(l, x);
  for (int s = 0; s < parts; s += 8) {
    float v[8][EPL];
#pragma unroll
    for (int y = 0; y < 8; ++y)
#pragma unroll
      for (int e = 0; e < EPL; ++e) v[y][e] = s + y < parts ? po[(size_t)(s + y) * D + e] : 0.0f;
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const float fy = __shfl(f, s + y);
#pragma unroll
      for (int e = 0; e < EPL; ++e) o[e] = __builtin_fmaf(v[y][e], fy, o[e]);
    }
  }
  const float inv = 1.0f / l;
  const size_t at = qrow * D + lane * EPL;
  if constexpr (DT == 1 && EPL == 2)
    reinterpret_cast<uint32_t*>(a.out)[at / 2] = pack_bf16(o[0] * inv, o[1] * inv);
  else if constexpr (DT == 1)
    reinterpret_cast<uint16_t*>(a.out)[at] = (uint16_t)f32_to_bf16_bits(o[0] * inv);
  else
#pragma unroll
    for (int e = 0; e < EPL; ++e) reinterpret_cast<float*>(a.out)[at + e] = o[e] * inv;
}

constexpr int CUS = 256;
constexpr int MIN_CHUNK = 128;       // keys of a part, at least; a multiple of every key tile
constexpr int64_t BIG_CACHE = 256ll << 20;      // the memory-side cache
constexpr int MAX_PARTS = 64;        // of a key range: a lane each in the joining kernel

template <int DT, int D, int RW, int KW, int SK>
int launch_cfg(const AttendArgs& a, hipStream_t s) {
  using C = Cfg<DT, D, RW, KW, SK>;
  const dim3 grid((unsigned)((int64_t)a.batch * a.hk * a.ntiles * a.splits));
  if (a.parent) {
    const auto k = attend_kernel<DT, D, RW, KW, SK, true>;
    allow_lds((const void*)k, C::LDS);
    hipLaunchKernelGGL(k, grid, dim3(C::THREADS), C::LDS, s, a);
  } else {
    const auto k = attend_kernel<DT, D, RW, KW, SK, false>;
    allow_lds((const void*)k, C::LDS);
    hipLaunchKernelGGL(k, grid, dim3(C::THREADS), C::LDS, s, a);
  }
  return (int)hipGetLastError();
}

// Row tiles of 32 rows with the keys cut among the waves, of 64 and two groups, or of 128 rows.
// (float32 tiles of 32 rows of 128 elements: two key groups; what four need does not fit the LDS)
template <int DT, int D>
int launch_type(const AttendArgs& a, hipStream_t s) {
  int rc;
  if constexpr (DT == 1)
    rc = a.bm == 32 ? launch_cfg<DT, D, 1, 4, 32>(a, s) : a.bm == 64 ? launch_cfg<DT, D, 2, 2, 64>(a, s)
                                                                     : launch_cfg<DT, D, 4, 1, 64>(a, s);
  else
    rc = a.bm == 32 ? launch_cfg<DT, D, 1, D == 64 ? 4 : 2, 32>(a, s) : launch_cfg<DT, D, 4, 1, 32>(a, s);
  if (rc == 0 && a.splits > 1) {
    const int64_t rows = (int64_t)a.tok.max_tokens << a.gshift;
    hipLaunchKernelGGL((attend_join_kernel<DT, D>), dim3((unsigned)(a.batch * a.hk * ((rows + 3) / 4))),
                       dim3(256), 0, s, a);
    rc = (int)hipGetLastError();
  }
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
