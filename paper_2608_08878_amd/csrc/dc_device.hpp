// Device-side building blocks shared by the decode-step kernels (gfx950, wave64).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dc_kernels.hpp"

namespace dc {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float NEG_BIG = -1.0e30f;   // "minus infinity" that keeps 0 * x finite

// Dynamic LDS beyond the 64 KB a launch has by default (static LDS here stays under
// 16 KB) has to be allowed; the call is host time on every launch, so small ones skip it.
inline void allow_lds(const void* kernel, size_t bytes) {
  if (bytes > 48 * 1024) hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

// Row layout: one lane owns 16 contiguous bytes of a key/value row.
template <int DTYPE, int D>
struct RowT {
  static constexpr int ELT = DTYPE == 0 ? 4 : 2;    // bytes per element
  static constexpr int EPL = 16 / ELT;              // elements per lane
  static constexpr int LPR = D / EPL;               // lanes per row: 8, 16 or 32
  static_assert(LPR == 8 || LPR == 16 || LPR == 32, "row layout");
};

__device__ __forceinline__ float bf16lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t f32_to_bf16_bits(float f) {
  uint32_t b = __float_as_uint(f);
  if ((b & 0x7F800000u) == 0x7F800000u && (b & 0x007FFFFFu)) return (b >> 16) | 0x40u;  // NaN stays NaN
  return (b + 0x7FFFu + ((b >> 16) & 1u)) >> 16;
}

// Two float32 numbers rounded to bf16 (to nearest even, NaN kept) in one instruction.
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}

// Partial dot product of the lane's 16-byte slices (fixed evaluation order).
template <int DTYPE>
__device__ __forceinline__ float dot_slice(const uint4& q, const uint4& k) {
  if constexpr (DTYPE == 1) {
    float acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, q.x),
                                                __builtin_bit_cast(bf16x2_t, k.x), 0.0f, false);
    acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, q.y),
                                          __builtin_bit_cast(bf16x2_t, k.y), acc, false);
    acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, q.z),
                                          __builtin_bit_cast(bf16x2_t, k.z), acc, false);
    acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, q.w),
                                          __builtin_bit_cast(bf16x2_t, k.w), acc, false);
    return acc;
  } else {
    float acc = __uint_as_float(q.x) * __uint_as_float(k.x);
    acc = __builtin_fmaf(__uint_as_float(q.y), __uint_as_float(k.y), acc);
    acc = __builtin_fmaf(__uint_as_float(q.z), __uint_as_float(k.z), acc);
    acc = __builtin_fmaf(__uint_as_float(q.w), __uint_as_float(k.w), acc);
    return acc;
  }
}

// Unpack a lane slice to float.
template <int DTYPE>
__device__ __forceinline__ void unpack_slice(const uint4& v, float* f) {
  if constexpr (DTYPE == 1) {
    f[0] = bf16lo(v.x); f[1] = bf16hi(v.x); f[2] = bf16lo(v.y); f[3] = bf16hi(v.y);
    f[4] = bf16lo(v.z); f[5] = bf16hi(v.z); f[6] = bf16lo(v.w); f[7] = bf16hi(v.w);
  } else {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
}

// DPP lane exchanges inside a 16-lane row.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int DPP_XOR1 = 0xB1;         // quad_perm [1,0,3,2]
constexpr int DPP_XOR2 = 0x4E;         // quad_perm [2,3,0,1]
constexpr int DPP_HALF_MIRROR = 0x141; // lane i <- lane 7-i within 8
constexpr int DPP_MIRROR = 0x140;      // lane i <- lane 15-i within 16

// Sum over the LPR lanes of a row group; every lane receives the same bits
// (each step adds two values in either order, and + is commutative).
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<DPP_XOR1>(x);
  x += dpp<DPP_XOR2>(x);
  x += dpp<DPP_HALF_MIRROR>(x);
  if constexpr (LPR >= 16) x += dpp<DPP_MIRROR>(x);
  if constexpr (LPR >= 32) x += __shfl_xor(x, 16);
  return x;
}

// One unit of attention weight, exp(s - m) / l, evaluated identically wherever
// it is needed (the retire step recomputes exactly what was added w steps ago).
__device__ __forceinline__ float attn_weight(float s, float m, float invl) {
  return __builtin_amdgcn_exp2f((s - m) * LOG2E) * invl;
}

// Feature contributions of one row for one step from its weights a_j:
//   cz = sum_j a_j,  cn = sum_j a_j H_j,
// summed in order within blocks of four heads, blocks added in order.
template <int G>
__device__ __forceinline__ void contrib_from_weights(const float* a, const float* H, float& cz,
                                                     float& cn) {
  cz = 0.0f;
  cn = 0.0f;
#pragma unroll
  for (int b = 0; b < G; b += 4) {
    float z = 0.0f, n = 0.0f;
#pragma unroll
    for (int j = b; j < (b + 4 < G ? b + 4 : G); ++j) {
      z = z + a[j];
      n = n + a[j] * H[j];
    }
    cz = cz + z;
    cn = cn + n;
  }
}

template <int G>
__device__ __forceinline__ void row_contrib(const float* s, const float* m, const float* invl,
                                            const float* H, float& cz, float& cn) {
  float a[G];
#pragma unroll
  for (int j = 0; j < G; ++j) a[j] = attn_weight(s[j], m[j], invl[j]);
  contrib_from_weights<G>(a, H, cz, cn);
}

// sigma_i: variance over the G heads of the weights a row received this step,
// (1/G) sum_j (a_j - mean)^2 (two passes: no cancellation; 0 for G = 1).
template <int G>
__device__ __forceinline__ float head_variance(const float* a) {
  float m = a[0];
#pragma unroll
  for (int j = 1; j < G; ++j) m = m + a[j];
  m = m * (1.0f / G);
  float v = 0.0f;
#pragma unroll
  for (int j = 0; j < G; ++j) {
    const float d = a[j] - m;
    v = __builtin_fmaf(d, d, v);
  }
  return v * (1.0f / G);
}

__device__ __forceinline__ uint4 ldg16(const void* p) { return *reinterpret_cast<const uint4*>(p); }
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 ldg16_nt(const void* p) {
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}

// The packed tokens t0 .. t0 + n - 1 of sequence b.  Offsets that are no ascending
// partition of the tokens are clamped, so that no index leaves the arrays.
__device__ __forceinline__ void token_range(const TokenArgs& t, int b, int& t0, int& n) {
  if (!t.cu) {
    t0 = b * t.max_tokens;
    n = t.max_tokens;
    return;
  }
  const int c0 = t.cu[b], c1 = t.cu[b + 1];
  t0 = c0 < 0 ? 0 : c0 > t.tokens ? t.tokens : c0;
  const int t1 = c1 < t0 ? t0 : c1 > t.tokens ? t.tokens : c1;
  n = t1 - t0 < t.max_tokens ? t1 - t0 : t.max_tokens;
}

// The sequence of packed token t: the last b with cu[b] <= t of the ascending offsets, found by the
// wave together, 64 offsets a step (all its lanes take part, with the same t).
__device__ __forceinline__ int sequence_of(const TokenArgs& tok, int batch, int t) {
  if (!tok.cu) return t / tok.max_tokens;
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 1; b0 < batch; b0 += 64) {
    const int b = b0 + lane;
    const uint64_t m = __ballot(b < batch && tok.cu[b < batch ? b : 0] <= t);
    before += __popcll(m);
    if (m != ~0ull) break;
  }
  return before;
}

// Rows of unit u before a call's own (len: their bound).
__device__ __forceinline__ int rows_before(const int32_t* unit_len, int len, int u) {
  if (!unit_len) return len;
  const int x = unit_len[u];
  return x < 0 ? 0 : x > len ? len : x;
}

// Tokens that unit u's sequence has seen (a sequence of an uneven batch: behind[u] fewer than
// the batch's count), at least 1.
template <typename Args>
__device__ __forceinline__ int tokens_of(const Args& a, int u) {
  if (!a.behind) return a.T;
  const int t = a.T - __builtin_amdgcn_readfirstlane(a.behind[u]);
  return t < 1 ? 1 : t;
}
// Largest position of unit u at the step that leaves the window.
__device__ __forceinline__ int retired_pmax(const DecodeArgs& a, int u) {
  return a.behind_ret ? a.pmax_ret - __builtin_amdgcn_readfirstlane(a.behind_ret[u]) : a.pmax_ret;
}

__device__ __forceinline__ void compiler_fence() { asm volatile("" ::: "memory"); }

// 16 bytes per lane from global memory to LDS byte lds + 16 lane (lds uniform).
// Issued from inline assembly, out of the compiler's sight: the caller waits
// for it explicitly (vmcnt; loads complete in issue order).  A load into LDS
// needs one wait state after a scalar write of M0 (the s_nop).
__device__ __forceinline__ void load_to_lds16(const void* g, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               : : "v"(g), "s"(lds) : "memory", "m0");
}

// The same from byte voff of a uniform address: no vector instruction advances it.
__device__ __forceinline__ void load_to_lds16_at(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               : : "v"(voff), "s"(base), "s"(lds) : "memory", "m0");
}

__device__ __forceinline__ void load_to_lds16_at_nt(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
               : : "v"(voff), "s"(base), "s"(lds) : "memory", "m0");
}

}  // namespace dc
