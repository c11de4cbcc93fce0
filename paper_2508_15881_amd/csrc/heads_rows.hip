// Rows of queries and keys of every head: norm over the row, position, and the way into the paged cache.
//
//   y = x / sqrt(mean(x^2) + eps) * weight;   pairs (y_a, y_b) of the first rot columns turn by pos f_j as in rotary.hip
//
// Memory-bound.  A row is held by 2^k >= d / 8 lanes of a wave, 8 columns each: its mean square is a sum over those lanes, and the partner
// of a pair of halves lies in another one of them.  The first rows of a thread are on their way while the sines of the token, shared by
// all its heads, are taken.
#include "heads.h"

#include <algorithm>

namespace tpla {

constexpr int HR_THREADS = 256;
constexpr int HR_BATCH = 3;        // rows per thread on their way together

template <typename T>
struct Piece8;
template <>
struct Piece8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4*>(p);
    b = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ __forceinline__ void get(float (&y)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = a[e];
      y[4 + e] = b[e];
    }
  }
  __device__ __forceinline__ void set(const float (&y)[8]) {
    a = f32x4{y[0], y[1], y[2], y[3]};
    b = f32x4{y[4], y[5], y[6], y[7]};
  }
  __device__ __forceinline__ void store(float* p, bool past) const {
    if (past) {
      __builtin_nontemporal_store(a, reinterpret_cast<f32x4*>(p));
      __builtin_nontemporal_store(b, reinterpret_cast<f32x4*>(p) + 1);
    } else {
      *reinterpret_cast<f32x4*>(p) = a;
      *(reinterpret_cast<f32x4*>(p) + 1) = b;
    }
  }
};
template <>
struct Piece8<bf16_t> {
  bf16x8 a;
  __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const bf16x8*>(p); }
  __device__ __forceinline__ void get(float (&y)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (float)a[e];
  }
  __device__ __forceinline__ void set(const float (&y)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = (bf16_t)y[e];
  }
  __device__ __forceinline__ void store(bf16_t* p, bool past) const {
    if (past)
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, a), reinterpret_cast<u32x4*>(p));
    else
      *reinterpret_cast<bf16x8*>(p) = a;
  }
};

// What a row's columns are multiplied with: y' = y cos + z sin, z the partner's column (the sign of sin is the place in the pair).
struct Turn8 {
  float c[8], s[8];
};

// grid: (tokens, blocks of rows).  The rows of a token are its H heads of queries, its H_kv of keys and, with slots, its H_kv of values.  LDS: (cos,
// sin) of the token's rot / 2 pairs, amplitude included.  LPR: lanes per row.  WHOLE: columns in eights are turned alike: rot / 2 a multiple of 8, or
// pairs side by side with rot one.
template <typename T, int LPR, bool WHOLE>
__global__ void __launch_bounds__(HR_THREADS) head_rows_kernel(HeadRowsArgs a, int block_rows) {
  extern __shared__ float2 turns[];
  constexpr int AT_ONCE = HR_THREADS / LPR;
  const int tid = threadIdx.x, lane = tid & 63, part = tid % LPR, c = 8 * part, pairs = a.rot / 2;
  const int64_t t = blockIdx.x;
  const int nq = a.q ? a.H : 0, nk = a.k ? a.H_kv : 0, nv = a.slots ? a.H_kv : 0;
  const int r0 = blockIdx.y * block_rows, r1 = min(r0 + block_rows, nq + nk + nv);
  const int slot = a.slots ? a.slots[t] : 0;
  const bool half = a.layout == TPLA_ROTARY_HALF;

  Piece8<T> x[HR_BATCH], wq, wk;
  auto request = [&](int first) {
#pragma unroll
    for (int k = 0; k < HR_BATCH; ++k) {
      const int r = first + k * AT_ONCE;
      if (r >= r1) continue;
      const bool is_q = r < nq, is_k = !is_q && r < nq + nk;
      if (c >= (is_q || is_k ? a.d_k : a.d_v)) continue;
      const T* src = is_q   ? static_cast<const T*>(a.q) + t * a.q_ts + r * a.q_hs
                     : is_k ? static_cast<const T*>(a.k) + t * a.k_ts + (r - nq) * a.k_hs
                            : static_cast<const T*>(a.v) + t * a.v_ts + (r - nq - nk) * a.v_hs;
      x[k].load(src + c);
    }
  };
  int first = r0 + tid / LPR;
  request(first);
  {
    float one[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) one[e] = 1.f;
    wq.set(one);
    wk.set(one);
  }
  if (a.q_weight && c < a.d_k) wq.load(static_cast<const T*>(a.q_weight) + c);
  if (a.k_weight && c < a.d_k) wk.load(static_cast<const T*>(a.k_weight) + c);
  for (int p = tid; p < pairs; p += HR_THREADS) {
    const double turn = (double)a.positions[t] * (a.freq[p] * 0.15915494309189533577);
    float s, co;
    sincospif((float)(2.0 * (turn - rint(turn))), &s, &co);
    turns[p] = make_float2(co * a.amplitude, s * a.amplitude);
  }
  __syncthreads();
  const int page = a.slots && slot >= 0 ? slot / a.page_tokens : 0, at = slot - page * a.page_tokens;
  Turn8 turn;
  if constexpr (WHOLE) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool low = half ? c < pairs : (e & 1) == 0;
      const float2 cs = c < a.rot ? turns[half ? (low ? c + e : c + e - pairs) : (c + e) / 2] : make_float2(1.f, 0.f);
      turn.c[e] = cs.x;
      turn.s[e] = low ? -cs.y : cs.y;
    }
  }
  const int partner = (c < pairs ? lane + pairs / 8 : lane - pairs / 8) & 63;
  const bool opposite = pairs == 4 * LPR;              // halves of whole rows: the partner is lane ^ LPR / 2
  const float inv_d = 1.0f / (float)a.d_k;
  for (; first - tid / LPR < r1; first += HR_BATCH * AT_ONCE) {        // (whole waves stay together: lanes exchange columns)
#pragma unroll
    for (int k = 0; k < HR_BATCH; ++k) {
      const int r = first + k * AT_ONCE;
      const bool is_q = r < nq, is_k = !is_q && r < nq + nk;
      const bool turned = (is_q || is_k) && r < r1, inside = r < r1 && c < (turned ? a.d_k : a.d_v);
      if (first - tid / LPR + k * AT_ONCE >= r1) continue;             // (no row for any thread)
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = 0.f;
      if (inside && turned) x[k].get(y);
      if (a.eps >= 0.f) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(y[e], y[e], sum);
        if constexpr (LPR > 1) sum += lane_xor<1>(sum, lane);
        if constexpr (LPR > 2) sum += lane_xor<2>(sum, lane);
        if constexpr (LPR > 4) sum += lane_xor<4>(sum, lane);
        if constexpr (LPR > 8) sum += lane_xor<8>(sum, lane);
        if constexpr (LPR > 16) sum += lane_xor<16>(sum, lane);
        const float by = __builtin_amdgcn_rsqf(fmaf(sum, inv_d, a.eps));
        float w[8];
        Piece8<T> mine = wk;
        if (is_q) mine = wq;
        mine.get(w);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= by * w[e];
      }
      if constexpr (WHOLE) {
        float z[8];
        if (!half) {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = y[e ^ 1];
        } else if (opposite) {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = lane_xor<LPR / 2>(y[e], lane);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], partner);
        }
        if (c < a.rot) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = fmaf(z[e], turn.s[e], y[e] * turn.c[e]);
        }
      } else if (half) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {                  // columns c + e -+ pairs: one of 8 values of some lane
          const int col = c + e < pairs ? c + e + pairs : c + e - pairs, other = (lane - part + (col >> 3)) & 63;
          z[e] = 0.f;
#pragma unroll
          for (int f = 0; f < 8; ++f) {
            const float v = __shfl(y[f], other);
            z[e] = (col & 7) == f ? v : z[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int col = c + e;
          if (col < a.rot) {
            const float2 cs = turns[col < pairs ? col : col - pairs];
            y[e] = col < pairs ? y[e] * cs.x - z[e] * cs.y : z[e] * cs.y + y[e] * cs.x;
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          if (c + e < a.rot) {
            const float2 cs = turns[(c + e) / 2];
            const float u = y[e], v = y[e + 1];
            y[e] = u * cs.x - v * cs.y;
            y[e + 1] = u * cs.y + v * cs.x;
          }
      }
      if (!inside) continue;
      if (turned) x[k].set(y);
      T* dst;
      if (is_q)
        dst = static_cast<T*>(a.q_out) + t * a.qo_ts + r * a.qo_hs;
      else if (!a.slots)
        dst = static_cast<T*>(a.k_out) + t * a.ko_ts + (r - nq) * a.ko_hs;
      else if (slot < 0)
        continue;
      else
        dst = is_k ? static_cast<T*>(a.k_out) + (((int64_t)page * a.H_kv + (r - nq)) * a.page_tokens + at) * a.d_k
                   : static_cast<T*>(a.v_pool) + (((int64_t)page * a.H_kv + (r - nq - nk)) * a.page_tokens + at) * a.d_v;
      x[k].store(dst + c, true);
    }
    if (first - tid / LPR + HR_BATCH * AT_ONCE < r1) request(first + HR_BATCH * AT_ONCE);
  }
}

template <typename T, bool WHOLE>
static auto head_rows_kernel_of(int lpr) -> void (*)(HeadRowsArgs, int) {
  return lpr == 4 ? head_rows_kernel<T, 4, WHOLE> : lpr == 8 ? head_rows_kernel<T, 8, WHOLE> : lpr == 16 ? head_rows_kernel<T, 16, WHOLE> : head_rows_kernel<T, 32, WHOLE>;
}

static int launch_head_rows_tokens(const HeadRowsArgs& a, int dtype, hipStream_t st) {
  const int widest = a.slots && a.d_v > a.d_k ? a.d_v : a.d_k, lpr = widest <= 32 ? 4 : widest <= 64 ? 8 : widest <= 128 ? 16 : 32;
  const int rows = (a.q ? a.H : 0) + (a.k ? a.H_kv : 0) + (a.slots ? a.H_kv : 0);
  // a token's rows in one workgroup, or in several where there are few tokens
  const int step = HR_BATCH * (HR_THREADS / lpr);
  const int block_rows = a.T >= 2 * device_cu_count() ? rows : std::min(rows, step);
  const dim3 grid((unsigned)a.T, (unsigned)((rows + block_rows - 1) / block_rows));
  const bool whole = a.rot % (a.layout == TPLA_ROTARY_HALF ? 16 : 8) == 0;
  void (*fn)(HeadRowsArgs, int) = dtype == TPLA_F32 ? (whole ? head_rows_kernel_of<float, true>(lpr) : head_rows_kernel_of<float, false>(lpr))
                                                    : (whole ? head_rows_kernel_of<bf16_t, true>(lpr) : head_rows_kernel_of<bf16_t, false>(lpr));
  hipLaunchKernelGGL(fn, grid, dim3(HR_THREADS), std::max(1, a.rot / 2) * sizeof(float2), st, a, block_rows);
  return check_launch("head_rows_kernel");
}

// A launch holds fewer than 2^32 threads along a dimension: longer calls go in parts.
int launch_head_rows(HeadRowsArgs a, int dtype, hipStream_t st) {
  constexpr int64_t MOST = (int64_t)1 << 23;
  const int64_t T = a.T, esz = dtype == TPLA_F32 ? 4 : 2;
  const auto ahead = [](const void* p, int64_t bytes) { return p ? static_cast<const char*>(p) + bytes : nullptr; };
  const auto out_ahead = [](void* p, int64_t bytes) { return p ? static_cast<char*>(p) + bytes : nullptr; };
  for (int64_t t = 0; t < T; t += MOST) {
    HeadRowsArgs part = a;
    part.T = std::min(MOST, T - t);
    part.positions = a.positions ? a.positions + t : nullptr;
    part.slots = a.slots ? a.slots + t : nullptr;
    part.q = ahead(a.q, t * a.q_ts * esz);
    part.k = ahead(a.k, t * a.k_ts * esz);
    part.v = ahead(a.v, t * a.v_ts * esz);
    part.q_out = out_ahead(a.q_out, t * a.qo_ts * esz);
    if (!a.slots) part.k_out = out_ahead(a.k_out, t * a.ko_ts * esz);
    const int rc = launch_head_rows_tokens(part, dtype, st);
    if (rc) return rc;
  }
  return TPLA_OK;
}

}  // namespace tpla
