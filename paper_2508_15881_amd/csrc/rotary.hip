// Rotary positions: pairs (x, y) of a row turn by pos f_j,
//   x' = (x cos a - y sin a) amplitude,  y' = (x sin a + y cos a) amplitude,
// interleaved pairs (2 j, 2 j + 1) or halves (j, j + rot / 2); columns from rot on are copied.
// The angle is formed in turns in double, whole turns are dropped there, and sine and cosine are taken in float: a position
// of a million turns the fastest pair by 2^-24 as exactly as position 1.  Memory-bound: a workgroup takes the sines of a few
// tokens once, for all their heads.
#include "tpla_internal.h"

namespace tpla {

constexpr int RO_THREADS = 256;

template <typename T>
struct alignas(16) Eight {
  T v[8];
};

// grid: (token blocks, head blocks).  LDS: [tokens][rot / 2] pairs of (cos, sin), amplitude included.
// VEC: a thread takes 8 columns (and, for halves, their 8 partners); otherwise one pair or one copied column.
template <typename T, bool VEC>
__global__ void __launch_bounds__(RO_THREADS) rotary_kernel(RotaryArgs a) {
  extern __shared__ float2 turn[];
  const int pairs = a.rot / 2, tid = threadIdx.x;
  const long long t0 = (long long)blockIdx.x * a.block_tokens;
  const int nt = (int)min((long long)a.block_tokens, a.T - t0);
  for (int x = tid; x < nt * pairs; x += RO_THREADS) {
    const double turns = (double)a.positions[t0 + x / pairs] * (a.freq[x % pairs] * 0.15915494309189533577);
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    if (a.inverse) s = -s;
    turn[x] = make_float2(c * a.amplitude, s * a.amplitude);
  }
  __syncthreads();
  const int heads = (a.q ? a.H : 0) + (a.k ? 1 : 0);
  const int h0 = blockIdx.y * a.block_heads, nh = min(a.block_heads, heads - h0);
  const bool half = a.layout == TPLA_ROTARY_HALF;
  // work per row: VEC: pieces of 8 columns, of the rotated ones of halves the first half's only
  const int lead = VEC ? (half ? pairs / 8 : 0) : pairs;
  const int per_row = VEC ? lead + (half ? (a.d_r - a.rot) / 8 : a.d_r / 8) : pairs + (a.d_r - a.rot);
  for (int x = tid; x < nt * nh * per_row; x += RO_THREADS) {
    const int w = x % per_row, row = x / per_row, h = h0 + row % nh, tt = row / nh;
    const long long t = t0 + tt;
    const bool key = h == heads - 1 && a.k;
    const T* src = static_cast<const T*>(key ? a.k : a.q) + (key ? t * a.k_ts : t * a.q_ts + h * a.q_hs);
    T* dst = static_cast<T*>(key ? a.k_out : a.q_out) + (key ? t * a.ko_ts : t * a.qo_ts + h * a.qo_hs);
    const float2* tr = turn + tt * pairs;
    if constexpr (VEC) {
      if (half && w < lead) {
        const Eight<T> p = *reinterpret_cast<const Eight<T>*>(src + 8 * w), q = *reinterpret_cast<const Eight<T>*>(src + pairs + 8 * w);
        Eight<T> u, v;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 cs = tr[8 * w + e];
          const float p0 = (float)p.v[e], q0 = (float)q.v[e];
          u.v[e] = (T)(p0 * cs.x - q0 * cs.y);
          v.v[e] = (T)(p0 * cs.y + q0 * cs.x);
        }
        *reinterpret_cast<Eight<T>*>(dst + 8 * w) = u;
        *reinterpret_cast<Eight<T>*>(dst + pairs + 8 * w) = v;
      } else {
        const int c0 = half ? a.rot + 8 * (w - lead) : 8 * w;
        Eight<T> p = *reinterpret_cast<const Eight<T>*>(src + c0);
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          if (c0 + e < a.rot && !half) {
            const float2 cs = tr[(c0 + e) / 2];
            const float p0 = (float)p.v[e], q0 = (float)p.v[e + 1];
            p.v[e] = (T)(p0 * cs.x - q0 * cs.y);
            p.v[e + 1] = (T)(p0 * cs.y + q0 * cs.x);
          }
        *reinterpret_cast<Eight<T>*>(dst + c0) = p;
      }
    } else {
      if (w < pairs) {
        const int i = half ? w : 2 * w, j = half ? w + pairs : 2 * w + 1;
        const float2 cs = tr[w];
        const float p0 = (float)src[i], q0 = (float)src[j];
        dst[i] = (T)(p0 * cs.x - q0 * cs.y);
        dst[j] = (T)(p0 * cs.y + q0 * cs.x);
      } else {
        dst[pairs + w] = src[pairs + w];
      }
    }
  }
}

int launch_rotary(RotaryArgs a, int dtype, hipStream_t st) {
  const bool half = a.layout == TPLA_ROTARY_HALF;
  const bool vec = !half || a.rot % 16 == 0;
  const int heads = (a.q ? a.H : 0) + (a.k ? 1 : 0);
  a.block_tokens = a.T >= 4 * device_cu_count() ? 8 : 1;
  while (a.block_tokens > 1 && (size_t)a.block_tokens * (a.rot / 2) * sizeof(float2) > 48 * 1024) a.block_tokens /= 2;
  a.block_heads = a.T >= device_cu_count() ? heads : (heads + 3) / 4;
  const dim3 grid((unsigned)((a.T + a.block_tokens - 1) / a.block_tokens), (unsigned)((heads + a.block_heads - 1) / a.block_heads));
  const size_t lds = (size_t)a.block_tokens * (a.rot / 2) * sizeof(float2);
  void (*fn)(RotaryArgs) = dtype == TPLA_F32 ? (vec ? rotary_kernel<float, true> : rotary_kernel<float, false>)
                                             : (vec ? rotary_kernel<bf16_t, true> : rotary_kernel<bf16_t, false>);
  hipLaunchKernelGGL(fn, grid, dim3(RO_THREADS), lds, st, a);
  return check_launch("rotary_kernel");
}

}  // namespace tpla
