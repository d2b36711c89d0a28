// Rows of several tokens on their way into a cache, on gfx950: the norm of query and
// key heads with the rotation by position, and the commit of rows behind the cache's
// length (a prompt's, or the accepted path of a draft tree).  Both move bytes.
#include "dc_device.hpp"
#include "dc_kernels.hpp"

#pragma clang fp contract(off)

namespace dc {

namespace {

constexpr int RT = 256;               // threads of a workgroup
constexpr int MAX_PAIRS = 64;         // rotated pairs of a head of 128
constexpr double INV_2PI = 0.15915494309189533577;

template <int DTYPE>
__device__ __forceinline__ uint4 pack_slice(const float* f) {
  if constexpr (DTYPE == 1)
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  else
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
}

// y = x / sqrt(mean x^2 + eps) * gain, then pairs (a, b) of the first rot elements turn
// by phi = pos f_i: (a cos phi - b sin phi, a sin phi + b cos phi), pair i being
// elements (i, i + rot / 2), or (2 i, 2 i + 1) interleaved.  float32 between the load
// and the one rounding at the store.  A far position times a frequency is a million
// radians and more, of which float32 keeps no useful fraction of a turn: the product is
// formed in binary64 (31 + 24 bits, one rounding) and taken to turns there; the
// remaining fraction goes to float32 sinpi / cospi.
// A workgroup takes up to TPB tokens.  It first puts their angles and places in LDS, one
// angle per thread, for every head; then LPR lanes work on a head row, 16 bytes each, the
// half-split partner a lane exchange away, with BATCH rows' loads under way at a time.
// One token and one row per lane group where that makes no more than FEW_WGS workgroups, else TPB
// tokens: a workgroup's angles and places are a chain of loads before its first store, which many
// small ones repeat and few large ones show (32 + 16 heads of 128, one token at a time and by four:
// 64 tokens 4.3 and 12.7 us, 1024 9.2 and 15.6, 4096 29.9 and 31.4, 19564 142 and 107).
// 19564 tokens, 481 MB, 107 us = 4.5 TB/s, of the 4.8 that a copy reaches.
constexpr int TPB = 4;               // (a wave each for their places)
constexpr int FEW_WGS = 16384;
static_assert(TPB * 64 <= RT, "a wave per token");

template <int DTYPE, int D, int BATCH>
__global__ void __launch_bounds__(RT) norm_rope_kernel(NormRopeArgs a, int per_block, int passes) {
  using R = RowT<DTYPE, D>;
  constexpr int LPR = R::LPR, EPL = R::EPL, ELT = R::ELT, GROUPS = RT / LPR;
  __shared__ __attribute__((aligned(16))) float cs[TPB][MAX_PAIRS], sn[TPB][MAX_PAIRS];
  __shared__ __attribute__((aligned(16))) float gain[2 * D];
  __shared__ int seq[TPB], num[TPB];                  // a token's sequence and number there, or -1
  const int tid = threadIdx.x, c = tid % LPR, grp = tid / LPR;
  const int half = a.rot / 2, dist = half / EPL;      // half-split partner: dist lanes away
  const int nrows = a.hq + a.hk + (a.k_out ? 0 : a.hk);
  const int first = blockIdx.x * per_block;
  const int count = a.tok.tokens - first < per_block ? a.tok.tokens - first : per_block;
  // this workgroup's rows of every token: GROUPS a pass
  const int row0 = blockIdx.y * passes * GROUPS;
  const int items = count * passes;

  uint4 w[BATCH];
  auto load = [&](int i) -> uint4 {
    const int t = i / passes, row = row0 + (i - t * passes) * GROUPS + grp;
    if (i >= items || row >= nrows) return make_uint4(0, 0, 0, 0);
    const bool isq = row < a.hq, isv = row >= a.hq + a.hk;
    const int h = isq ? row : isv ? row - a.hq - a.hk : row - a.hq;
    const char* base = (const char*)(isq ? a.q : isv ? a.v : a.k);
    const int64_t ld = isq ? a.ld_q : isv ? a.ld_v : a.ld_k;
    return ldg16_nt(base + ((size_t)(first + t) * ld + (size_t)h * D) * ELT + c * 16);
  };
#pragma unroll
  for (int x = 0; x < BATCH; ++x) w[x] = load(x);

  for (int i = tid; i < count * half; i += RT) {
    const int t = i / half, p = i - t * half;
    const double turns = (double)a.pos[first + t] * (double)a.inv_freq[p] * INV_2PI;
    sincospif((float)(2.0 * (turns - rint(turns))), &sn[t][p], &cs[t][p]);
  }
  if (!a.k_out) {             // a token per wave
    const int x = tid >> 6;
    if (x < count) {
      const int b = sequence_of(a.tok, a.batch, first + x);
      int t0, n;
      token_range(a.tok, b, t0, n);
      const int r = first + x - t0;
      seq[x] = b;
      num[x] = r >= 0 && r < n ? r : -1;
    }
  }
  // gains through LDS: a load a thread (each lane its 16 of them straight into registers took
  // 9 us more of 512 tokens' 15)
  if (a.norm && tid < 2 * D) {
    const float* from = tid < D ? a.q_gain : a.k_gain;
    gain[tid] = from ? from[tid % D] : 1.0f;
  }
  __syncthreads();
  float gq[EPL], gk[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    gq[e] = gain[c * EPL + e];
    gk[e] = gain[D + c * EPL + e];
  }

  auto finish = [&](int i, uint4 x16) {
    const int t = i / passes, row = row0 + (i - t * passes) * GROUPS + grp;
    if (i >= items || row >= nrows) return;
    const bool isq = row < a.hq, isv = row >= a.hq + a.hk;
    const int h = isq ? row : isv ? row - a.hq - a.hk : row - a.hq;
    if (!isv) {
      float x[EPL];
      unpack_slice<DTYPE>(x16, x);
      if (a.norm) {
        float s = x[0] * x[0];
#pragma unroll
        for (int e = 1; e < EPL; ++e) s = __builtin_fmaf(x[e], x[e], s);
        s = row_sum<LPR>(s);
        const float inv = rsqrtf(s * (1.0f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = x[e] * inv * (isq ? gq[e] : gk[e]);
      }
      if (a.interleaved) {
        if (c * EPL < a.rot) {
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            const float co = cs[t][(c * EPL + e) / 2], si = sn[t][(c * EPL + e) / 2];
            const float p = x[e], o = x[e + 1];
            x[e] = __builtin_fmaf(p, co, -(o * si));
            x[e + 1] = __builtin_fmaf(p, si, o * co);
          }
        }
      } else if (half) {
        const bool low = c < dist, in = c < 2 * dist;
        const int from = in ? (low ? c + dist : c - dist) : c;
        const int i0 = in ? (low ? c : c - dist) * EPL : 0;
        float o[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] = __shfl(x[e], from, LPR);
        if (in) {
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            const float co = cs[t][i0 + e], si = low ? -sn[t][i0 + e] : sn[t][i0 + e];
            x[e] = __builtin_fmaf(x[e], co, o[e] * si);
          }
        }
      }
      x16 = pack_slice<DTYPE>(x);
    }
    char* dst;
    if (isq) {
      dst = (char*)a.q_out + ((size_t)(first + t) * a.hq + h) * D * ELT;
    } else if (a.k_out) {
      dst = (char*)a.k_out + ((size_t)(first + t) * a.hk + h) * D * ELT;
    } else {
      const int u = (seq[t] * a.n_layers + a.layer) * a.hk + h;
      if (num[t] < 0) return;
      dst = (char*)(isv ? a.vc : a.kc) +
            ((size_t)u * a.cap + rows_before(a.unit_len, a.len, u) + num[t]) * D * ELT;
    }
    *reinterpret_cast<uint4*>(dst + c * 16) = x16;
  };
  for (int i = 0; i < items; i += BATCH) {
    uint4 y[BATCH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      y[x] = w[x];
      w[x] = load(i + BATCH + x);
    }
#pragma unroll
    for (int x = 0; x < BATCH; ++x) finish(i + x, y[x]);
  }
}

// Rows that unit u keeps of its n new ones.
__device__ __forceinline__ int rows_kept(const CommitArgs& a, int b, int n) {
  int m = n < a.width ? n : a.width;
  if (a.keep) {
    const int x = a.keep[b];
    m = x < 0 ? 0 : x < m ? x : m;
  }
  return m;
}

// Tokens fewer than the batch's count that unit u's sequence had seen, and has once it keeps `keep`
// rows of a call that counts for a.width.
__device__ __forceinline__ int behind_of(const CommitArgs& a, int u) { return a.behind ? a.behind[u] : 0; }
__device__ __forceinline__ void store_behind(const CommitArgs& a, int u, int keep) {
  if (a.behind_next) a.behind_next[u] = behind_of(a, u) + a.width - keep;
}

// Feature state of a row as dc_feat_init leaves it (lane c of the row's LPR); first_pos: position
// of the call's first row.
template <int DTYPE, int D>
__device__ __forceinline__ void init_row(const CommitArgs& a, int u, int slot, int first_pos, int j,
                                         const uint4& v, int c) {
  using R = RowT<DTYPE, D>;
  float f[R::EPL];
  unpack_slice<DTYPE>(v, f);
  float s = f[0] * f[0];
#pragma unroll
  for (int e = 1; e < R::EPL; ++e) s = __builtin_fmaf(f[e], f[e], s);
  s = row_sum<R::LPR>(s);
  if (c == 0) {
    const size_t i = (size_t)u * a.cap + slot;
    a.alpha[i] = 0.0f;
    a.num[i] = 0.0;
    a.den[i] = 0.0;
    a.pos[i] = first_pos + j;
    a.vnorm[i] = sqrtf(s);
    if (a.sigma) a.sigma[i] = 0.0f;
  }
}

// An accepted path: row len + j <- row len + path[j].  One workgroup per unit walks the
// path in passes of RT / LPR rows; a pass has read its rows before it writes, and an
// entry below its own index counts as that index, so no later pass reads a row that an
// earlier one has written.
template <int DTYPE, int D>
__global__ void __launch_bounds__(RT) commit_path_kernel(CommitArgs a) {
  using R = RowT<DTYPE, D>;
  constexpr int LPR = R::LPR, RPP = RT / LPR;
  const int u = a.y0 + blockIdx.y, b = u / a.per_seq;
  const int c = threadIdx.x % LPR, jr = threadIdx.x / LPR;
  int t0, n;
  token_range(a.tok, b, t0, n);
  const int start = rows_before(a.unit_len, a.len, u), keep = rows_kept(a, b, n);
  const int first_pos = a.next_pos - behind_of(a, u);
  for (int j0 = 0; j0 < keep; j0 += RPP) {
    const int j = j0 + jr;
    const bool on = j < keep;
    int src = j < a.width ? a.path[(size_t)b * a.width + j] : 0;
    src = src < j ? j : src >= n ? n - 1 : src;
    const size_t from = (((size_t)u * a.cap + start + src) * LPR + c) * 16;
    const size_t to = (((size_t)u * a.cap + start + j) * LPR + c) * 16;
    uint4 kw = make_uint4(0, 0, 0, 0), vw = kw;
    if (on) {
      kw = ldg16((const char*)a.k + from);
      vw = ldg16((const char*)a.v + from);
    }
    __syncthreads();
    if (on) {
      *reinterpret_cast<uint4*>((char*)a.k + to) = kw;
      *reinterpret_cast<uint4*>((char*)a.v + to) = vw;
    }
    if (a.alpha && on) init_row<DTYPE, D>(a, u, start + j, first_pos, j, vw, c);
  }
  if (a.unit_len) {
    __syncthreads();
    if (threadIdx.x == 0) {
      a.unit_len[u] = start + keep;
      store_behind(a, u, keep);
    }
  }
}

// The first rows as they are: only their feature state is written.
template <int DTYPE, int D>
__global__ void __launch_bounds__(RT) commit_rows_kernel(CommitArgs a) {
  using R = RowT<DTYPE, D>;
  constexpr int LPR = R::LPR, RPP = RT / LPR;
  const int u = a.y0 + blockIdx.y, b = u / a.per_seq;
  const int c = threadIdx.x % LPR;
  int t0, n;
  token_range(a.tok, b, t0, n);
  const int start = rows_before(a.unit_len, a.len, u), keep = rows_kept(a, b, n);
  const int first_pos = a.next_pos - behind_of(a, u);
  for (int j = blockIdx.x * RPP + threadIdx.x / LPR; j < keep; j += gridDim.x * RPP)
    init_row<DTYPE, D>(a, u, start + j, first_pos, j,
                       ldg16((const char*)a.v + (((size_t)u * a.cap + start + j) * LPR + c) * 16), c);
}

__global__ void commit_len_kernel(CommitArgs a) {
  const int u = blockIdx.x * RT + threadIdx.x;
  if (u >= a.units) return;
  const int b = u / a.per_seq;
  int t0, n;
  token_range(a.tok, b, t0, n);
  const int keep = rows_kept(a, b, n);
  a.unit_len[u] = rows_before(a.unit_len, a.len, u) + keep;
  store_behind(a, u, keep);
}

template <int DTYPE, int D>
void norm_rope(const NormRopeArgs& a, hipStream_t s) {
  constexpr int GROUPS = RT / RowT<DTYPE, D>::LPR;
  const int nrows = a.hq + a.hk + (a.k_out ? 0 : a.hk), passes = (nrows + GROUPS - 1) / GROUPS;
  const int64_t one = (int64_t)a.tok.tokens * passes;
  if (one <= FEW_WGS)
    hipLaunchKernelGGL((norm_rope_kernel<DTYPE, D, 1>), dim3(a.tok.tokens, passes), dim3(RT), 0, s, a, 1, 1);
  else
    hipLaunchKernelGGL((norm_rope_kernel<DTYPE, D, 2>), dim3((a.tok.tokens + TPB - 1) / TPB), dim3(RT), 0, s, a,
                       TPB, passes);
}

template <int DTYPE, int D>
void commit(const CommitArgs& a, hipStream_t s) {
  if (a.path) {
    for_grid_y(a.units, [&](int y0, int ny) {
      CommitArgs b = a;
      b.y0 = y0;
      hipLaunchKernelGGL((commit_path_kernel<DTYPE, D>), dim3(1, ny), dim3(RT), 0, s, b);
    });
    return;
  }
  if (a.alpha) {
    constexpr int RPP = RT / RowT<DTYPE, D>::LPR;
    const int gx = (a.width + RPP - 1) / RPP < 64 ? (a.width + RPP - 1) / RPP : 64;
    for_grid_y(a.units, [&](int y0, int ny) {
      CommitArgs b = a;
      b.y0 = y0;
      hipLaunchKernelGGL((commit_rows_kernel<DTYPE, D>), dim3(gx, ny), dim3(RT), 0, s, b);
    });
  }
  if (a.unit_len) hipLaunchKernelGGL(commit_len_kernel, dim3((a.units + RT - 1) / RT), dim3(RT), 0, s, a);
}

}  // namespace

int launch_norm_rope(const NormRopeArgs& a, int dtype, int D, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1 && D == 128) norm_rope<1, 128>(a, s);
  else if (dtype == 1) norm_rope<1, 64>(a, s);
  else if (D == 128) norm_rope<0, 128>(a, s);
  else norm_rope<0, 64>(a, s);
  return (int)hipGetLastError();
}

int launch_commit(const CommitArgs& a, int dtype, int D, void* stream) {
  if (!a.path && !a.alpha && !a.unit_len) return 0;      // the host's lengths say it all
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 1 && D == 128) commit<1, 128>(a, s);
  else if (dtype == 1) commit<1, 64>(a, s);
  else if (D == 128) commit<0, 128>(a, s);
  else commit<0, 64>(a, s);
  return (int)hipGetLastError();
}

}  // namespace dc
