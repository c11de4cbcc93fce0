// Rows of queries and keys of every head: norm over the row, position, and the way into the paged cache.
//
//   y = x / sqrt(mean(x^2) + eps) * weight;   pairs (y_a, y_b) of the first rot columns turn by pos f_j as in rotary.hip
//
// Memory-bound.  A row is held by 2^k >= d / 8 lanes of a wave, 8 columns each: its mean square is a sum over those lanes, and the partner
// of a pair of halves lies in another one of them.  A wave has a token; its first rows are on their way while it takes the token's sines.
// 16411 tokens, 32 + 8 heads of 128 columns, bf16 (336 MB read and written): 75 us = 4.5 TB/s; 9001 tokens of 48 + 12 + 12 heads of 64 into the
// cache (166 MB): 33 - 36 us = 4.6 - 5.0.  (A workgroup per token, its rows dealt over the threads whatever their kind: 97 and 38.)
#include "heads.h"

#include <algorithm>

namespace tpla {

constexpr int HR_THREADS = 256;
constexpr int HR_BATCH = 4;        // groups of rows of a wave on their way together (16411 tokens, 40 heads of 128 columns: 2 78 us, 3 75.4, 4 75.2, 6 76.3)
constexpr int HR_FILL = 8;         // tokens per compute unit from which on a wave takes a whole token (16411 tokens, a batch of rows per wave: 85 us)

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
  // Past the caches: what a call writes is read by another kernel, and lines kept for it push out what this one still reads (16411 tokens: 81 us with ordinary
  // stores, 75 so; 9001 tokens into the cache 50 and 36).
  __device__ __forceinline__ void store(float* p) const {
    __builtin_nontemporal_store(a, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(b, reinterpret_cast<f32x4*>(p) + 1);
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
  __device__ __forceinline__ void store(bf16_t* p) const { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, a), reinterpret_cast<u32x4*>(p)); }
};

// What a row's columns are multiplied with: y' = y cos + z sin, z the partner's column (the sign of sin is the place in the pair).
struct Turn8 {
  float c[8], s[8];
};

// A wave takes `each` groups of rows of one token, `parts` waves the whole token: first its H heads of queries, then its H_kv of keys, then with slots
// its H_kv of values.  A group is 64 / LPR rows of one kind (LPR lanes hold a row), so that what tells the kinds apart is the same for the whole wave.  LDS:
// [wave][rot / 2] (cos, sin), amplitude included; each wave takes its own, no barrier.  WHOLE: columns in eights are turned alike: rot / 2 a multiple of 8,
// or pairs side by side with rot one.
template <typename T, int LPR, bool WHOLE>
__global__ void __launch_bounds__(HR_THREADS) head_rows_kernel(HeadRowsArgs a, int parts, int each) {
  extern __shared__ float2 all_turns[];
  constexpr int RPW = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = lane % LPR, j = lane / LPR, c = 8 * part, pairs = a.rot / 2;
  const unsigned task = blockIdx.x * (HR_THREADS / 64) + wave;
  const int64_t t = task / (unsigned)parts;
  if (t >= a.T) return;
  float2* const turns = all_turns + wave * pairs;
  const int nq = a.q ? a.H : 0, nk = a.k ? a.H_kv : 0, nv = a.slots ? a.H_kv : 0;
  const int gq = (nq + RPW - 1) / RPW, gk = gq + (nk + RPW - 1) / RPW, gv = gk + (nv + RPW - 1) / RPW;
  const int g0 = (int)(task - (unsigned)t * (unsigned)parts) * each, g1 = min(g0 + each, gv);
  const bool half = a.layout == TPLA_ROTARY_HALF;

  struct Rows {
    const T* src;              // of the group's first row
    int64_t hs;
    int first, n, width;       // the group's first row among those of its kind, and how many of those there are
  };
  auto rows_of = [&](int g) {
    if (g < gq) return Rows{static_cast<const T*>(a.q) + t * a.q_ts + g * RPW * a.q_hs, a.q_hs, g * RPW, nq, a.d_k};
    if (g < gk) return Rows{static_cast<const T*>(a.k) + t * a.k_ts + (g - gq) * RPW * a.k_hs, a.k_hs, (g - gq) * RPW, nk, a.d_k};
    return Rows{static_cast<const T*>(a.v) + t * a.v_ts + (g - gk) * RPW * a.v_hs, a.v_hs, (g - gk) * RPW, nv, a.d_v};
  };
  Piece8<T> x[HR_BATCH], wq, wk;
  auto request = [&](int first) {
#pragma unroll
    for (int k = 0; k < HR_BATCH; ++k)
      if (first + k < g1) {
        const Rows r = rows_of(first + k);
        if (r.first + j < r.n && c < r.width) x[k].load(r.src + (j * r.hs + c));
      }
  };
  request(g0);
  {
    float one[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) one[e] = 1.f;
    wq.set(one);
    wk.set(one);
  }
  if (a.q_weight && c < a.d_k) wq.load(static_cast<const T*>(a.q_weight) + c);
  if (a.k_weight && c < a.d_k) wk.load(static_cast<const T*>(a.k_weight) + c);
  for (int p = lane; p < pairs; p += 64) {
    const double turn = (double)a.positions[t] * (a.freq[p] * 0.15915494309189533577);
    float s, co;
    sincospif((float)(2.0 * (turn - rint(turn))), &s, &co);
    turns[p] = make_float2(co * a.amplitude, s * a.amplitude);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // (LDS operations of a wave complete in order)
  __builtin_amdgcn_wave_barrier();
  const int slot = a.slots ? a.slots[t] : 0;
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
  for (int first = g0; first < g1; first += HR_BATCH) {
#pragma unroll
    for (int k = 0; k < HR_BATCH; ++k) {
      const int g = first + k;
      if (g >= g1) continue;
      const Rows r = rows_of(g);
      const bool inside = r.first + j < r.n && c < r.width;
      if (g < gk) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = 0.f;
        if (inside) x[k].get(y);
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
          if (g < gq)
            wq.get(w);
          else
            wk.get(w);
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
          for (int e = 0; e < 8; ++e) {                // columns c + e -+ pairs: one of 8 values of some lane
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
        x[k].set(y);
      }
      if (!inside) continue;
      if (g < gq) {
        x[k].store(static_cast<T*>(a.q_out) + t * a.qo_ts + r.first * a.qo_hs + (j * a.qo_hs + c));
      } else if (!a.slots) {
        x[k].store(static_cast<T*>(a.k_out) + t * a.ko_ts + r.first * a.ko_hs + (j * a.ko_hs + c));
      } else if (slot >= 0) {
        T* pool = static_cast<T*>(g < gk ? a.k_out : a.v_pool);
        const int64_t row = ((int64_t)page * a.H_kv + r.first) * a.page_tokens + at;
        x[k].store(pool + row * r.width + ((int64_t)j * a.page_tokens * r.width + c));
      }
    }
    if (first + HR_BATCH < g1) request(first + HR_BATCH);
  }
}

template <typename T, bool WHOLE>
static auto head_rows_kernel_of(int lpr) -> void (*)(HeadRowsArgs, int, int) {
  return lpr == 4 ? head_rows_kernel<T, 4, WHOLE> : lpr == 8 ? head_rows_kernel<T, 8, WHOLE> : lpr == 16 ? head_rows_kernel<T, 16, WHOLE> : head_rows_kernel<T, 32, WHOLE>;
}

static int launch_head_rows_tokens(const HeadRowsArgs& a, int dtype, hipStream_t st) {
  const int widest = a.slots && a.d_v > a.d_k ? a.d_v : a.d_k, lpr = widest <= 32 ? 4 : widest <= 64 ? 8 : widest <= 128 ? 16 : 32;
  const int rpw = 64 / lpr, kinds_kv = (a.k ? 1 : 0) + (a.slots ? 1 : 0);
  const int groups = (a.q ? (a.H + rpw - 1) / rpw : 0) + kinds_kv * ((a.H_kv + rpw - 1) / rpw);
  // a wave takes a whole token, sines and all, or where there are few tokens, a batch of its rows
  const int each = a.T >= HR_FILL * device_cu_count() ? groups : std::min(groups, HR_BATCH), parts = (groups + each - 1) / each;
  const int64_t waves = a.T * parts;
  const dim3 grid((unsigned)((waves + HR_THREADS / 64 - 1) / (HR_THREADS / 64)));
  const bool whole = a.rot % (a.layout == TPLA_ROTARY_HALF ? 16 : 8) == 0;
  void (*fn)(HeadRowsArgs, int, int) = dtype == TPLA_F32 ? (whole ? head_rows_kernel_of<float, true>(lpr) : head_rows_kernel_of<float, false>(lpr))
                                                    : (whole ? head_rows_kernel_of<bf16_t, true>(lpr) : head_rows_kernel_of<bf16_t, false>(lpr));
  hipLaunchKernelGGL(fn, grid, dim3(HR_THREADS), (HR_THREADS / 64) * std::max(1, a.rot / 2) * sizeof(float2), st, a, parts, each);
  return check_launch("head_rows_kernel");
}

// A launch holds fewer than 2^32 threads along a dimension: longer calls go in parts.
int launch_head_rows(HeadRowsArgs a, int dtype, hipStream_t st) {
  constexpr int64_t MOST = (int64_t)1 << 20;
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
