// Rotary positions: pairs (x, y) of a row turn by pos f_j,
//   x' = (x cos a - y sin a) amplitude,  y' = (x sin a + y cos a) amplitude,
// interleaved pairs (2 j, 2 j + 1) or halves (j, j + rot / 2); columns from rot on are copied.
// The angle is formed in turns in double, whole turns are dropped there, and sine and cosine are taken in float: a position
// of a million turns the fastest pair by 2^-24 as exactly as position 1.  Memory-bound: a workgroup takes the sines of a few
// tokens once, for all their heads.
#include "tpla_internal.h"

#include <algorithm>

namespace tpla {

constexpr int RO_THREADS = 256;
constexpr int RO_BATCH = 4;        // rows per thread on their way together

template <int BYTES>
struct Word;
template <>
struct Word<2> { typedef unsigned short type; };
template <>
struct Word<4> { typedef unsigned type; };
template <>
struct Word<8> { typedef unsigned long long type; };
template <>
struct Word<16> { typedef f32x4 type; };

template <typename T, int W>
struct alignas(W * sizeof(T) < 16 ? W * sizeof(T) : 16) Columns {
  T v[W];
  // Past the caches: what a call writes is read by another kernel, on other compute units, and lines kept for it push out what this
  // one still reads (20011 tokens, 64 heads: 80 us with ordinary stores, 62 so, 5.3 TB/s read and written; 2048 tokens 10.8 and 7.8).
  __device__ __forceinline__ void stream_to(T* dst) const {
    constexpr int BYTES = alignof(Columns), N = sizeof(v) / BYTES;
    typedef typename Word<BYTES>::type Piece;
    Piece piece[N];
    __builtin_memcpy(piece, v, sizeof(v));
#pragma unroll
    for (int i = 0; i < N; ++i) __builtin_nontemporal_store(piece[i], reinterpret_cast<Piece*>(dst) + i);
  }
};

// What a thread does to one row: W columns, and of halves' rotated columns their W partners.  Pairs side by side and halves of whole eights: W = 8;
// halves of an even number of columns 2, of an odd number 1 (64 heads, 4096 tokens, 60 of 64 columns rotated, bf16: 25.2 us with 1, 16.1 with 2).
template <typename T, int W>
struct RowPart {
  Columns<T, W> p, q;
  __device__ __forceinline__ void load(const RotaryArgs& a, const T* src, int at, bool two) {
    p = *reinterpret_cast<const Columns<T, W>*>(src + at);
    if (two) q = *reinterpret_cast<const Columns<T, W>*>(src + at + a.rot / 2);
  }
  // turn: (cos, sin) of this token's pairs
  __device__ __forceinline__ void store(const RotaryArgs& a, T* dst, int at, bool two, const float2* turn) {
    if (two) {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float2 cs = turn[at + e];
        const float x = (float)p.v[e], y = (float)q.v[e];
        p.v[e] = (T)(x * cs.x - y * cs.y);
        q.v[e] = (T)(x * cs.y + y * cs.x);
      }
      q.stream_to(dst + at + a.rot / 2);
    } else if (W == 8 && a.layout == TPLA_ROTARY_INTERLEAVED) {
#pragma unroll
      for (int e = 0; e + 1 < W; e += 2)
        if (at + e < a.rot) {
          const float2 cs = turn[(at + e) / 2];
          const float x = (float)p.v[e], y = (float)p.v[e + 1];
          p.v[e] = (T)(x * cs.x - y * cs.y);
          p.v[e + 1] = (T)(x * cs.y + y * cs.x);
        }
    }
    p.stream_to(dst + at);
  }
};

// grid: (blocks of tokens, blocks of heads).  LDS: [tokens][rot / 2] pairs of (cos, sin), amplitude included.  A thread keeps its part of a row and
// takes rows lanes_per_row threads apart, RO_BATCH of them on their way together; the keys are one more head.
template <typename T, int W>
__global__ void __launch_bounds__(RO_THREADS) rotary_kernel(RotaryArgs a) {
  extern __shared__ float2 turns[];
  const int pairs = a.rot / 2, tid = threadIdx.x;
  const long long t0 = (long long)blockIdx.x * a.block_tokens;
  const int nt = (int)min((long long)a.block_tokens, a.T - t0);
  for (int x = tid; x < nt * pairs; x += RO_THREADS) {
    const double turn = (double)a.positions[t0 + x / pairs] * (a.freq[x % pairs] * 0.15915494309189533577);
    float s, c;
    sincospif((float)(2.0 * (turn - rint(turn))), &s, &c);
    if (a.inverse) s = -s;
    turns[x] = make_float2(c * a.amplitude, s * a.amplitude);
  }
  __syncthreads();
  const bool half = a.layout == TPLA_ROTARY_HALF;
  // parts of a row: rotated ones (halves: of the first half), then what is copied
  const int lead = half ? pairs / W : a.d_r / W, parts = half ? lead + (a.d_r - a.rot) / W : lead;
  const int at_once = max(1, RO_THREADS / parts);
  const int heads = (a.q ? a.H : 0) + (a.k ? 1 : 0);
  const int h0 = blockIdx.y * a.block_heads, nh = min(a.block_heads, heads - h0), rows = nt * nh;
  for (int part = tid % parts; part < parts; part += RO_THREADS) {       // (once, unless a row has more parts than there are threads)
    const int first = tid / parts;
    if (first >= at_once) continue;
    const bool two = half && part < lead;
    const int at = part < lead ? W * part : a.rot + W * (part - lead);
    // row = token * nh + head, walked without divisions
    const int dt = at_once / nh, dh = at_once % nh;
    int tt = first / nh, h = first % nh;
    for (int row = first; row < rows; row += RO_BATCH * at_once) {
      RowPart<T, W> x[RO_BATCH];
      T* dst[RO_BATCH];
      int tok[RO_BATCH];
#pragma unroll
      for (int k = 0; k < RO_BATCH; ++k) {
        dst[k] = nullptr;
        if (row + k * at_once < rows) {
          const long long t = t0 + tt;
          const bool key = a.k && h0 + h == heads - 1;
          const T* src = key ? static_cast<const T*>(a.k) + t * a.k_ts : static_cast<const T*>(a.q) + t * a.q_ts + (h0 + h) * a.q_hs;
          dst[k] = key ? static_cast<T*>(a.k_out) + t * a.ko_ts : static_cast<T*>(a.q_out) + t * a.qo_ts + (h0 + h) * a.qo_hs;
          tok[k] = tt;
          x[k].load(a, src, at, two);
        }
        tt += dt;
        h += dh;
        if (h >= nh) {
          h -= nh;
          ++tt;
        }
      }
#pragma unroll
      for (int k = 0; k < RO_BATCH; ++k)
        if (dst[k]) x[k].store(a, dst[k], at, two, turns + tok[k] * pairs);
    }
  }
}

static int launch_rotary_tokens(RotaryArgs a, int dtype, hipStream_t st) {
  const bool half = a.layout == TPLA_ROTARY_HALF;
  const int w = !half || a.rot % 16 == 0 ? 8 : a.rot % 4 == 0 ? 2 : 1;
  const int heads = (a.q ? a.H : 0) + (a.k ? 1 : 0);
  // sines shared by the heads of a token; two tokens in a workgroup fill its threads, more leave some compute units behind
  // (4 tokens: 63 us for 20011 tokens and 9.0 for 2048; 2: 62 and 7.8; 1: 69 and 8.1)
  a.block_tokens = a.T >= 4 * device_cu_count() ? 2 : 1;
  a.block_heads = a.T >= device_cu_count() ? heads : (heads + 3) / 4;
  const dim3 grid((unsigned)((a.T + a.block_tokens - 1) / a.block_tokens), (unsigned)((heads + a.block_heads - 1) / a.block_heads));
  const size_t lds = (size_t)a.block_tokens * (a.rot / 2) * sizeof(float2);
  void (*fn)(RotaryArgs);
  if (dtype == TPLA_F32)
    fn = w == 8 ? rotary_kernel<float, 8> : w == 2 ? rotary_kernel<float, 2> : rotary_kernel<float, 1>;
  else
    fn = w == 8 ? rotary_kernel<bf16_t, 8> : w == 2 ? rotary_kernel<bf16_t, 2> : rotary_kernel<bf16_t, 1>;
  hipLaunchKernelGGL(fn, grid, dim3(RO_THREADS), lds, st, a);
  return check_launch("rotary_kernel");
}

// A launch holds fewer than 2^32 threads along a dimension, and a workgroup of 256 may have one token: longer calls go in parts.
int launch_rotary(RotaryArgs a, int dtype, hipStream_t st) {
  constexpr int64_t MOST = (int64_t)1 << 23;
  const int64_t T = a.T, esz = dtype == TPLA_F32 ? 4 : 2;
  const auto ahead = [](const void* p, int64_t bytes) { return p ? static_cast<const char*>(p) + bytes : nullptr; };
  const auto out_ahead = [](void* p, int64_t bytes) { return p ? static_cast<char*>(p) + bytes : nullptr; };
  for (int64_t t = 0; t < T; t += MOST) {
    RotaryArgs part = a;
    part.T = std::min(MOST, T - t);
    part.positions = a.positions + t;
    part.q = ahead(a.q, t * a.q_ts * esz);
    part.k = ahead(a.k, t * a.k_ts * esz);
    part.q_out = out_ahead(a.q_out, t * a.qo_ts * esz);
    part.k_out = out_ahead(a.k_out, t * a.ko_ts * esz);
    const int rc = launch_rotary_tokens(part, dtype, st);
    if (rc) return rc;
  }
  return TPLA_OK;
}

}  // namespace tpla
