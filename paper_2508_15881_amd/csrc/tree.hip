// Attention of drafted tokens over the paged latent slices (tpla_decode_shard(s)_tree): the general kernel, for every width
// and type, and the merge of partial results of both kernels.
//
// Row r = t H + h of a (slice, sequence): s_k = scale (q_lat . c_k + q_pe . k_pe_k) over the committed tokens k < L and the
// drafts k = L + j whose bit j of mask[b, t] is set; o = sum softmax(s)_k c_k, lse = log sum exp(s).  One pass with the running
// maximum and sum.  A row that sees nothing has sum 0: o = 0, lse = -inf.
#include "split_merge.h"

namespace tpla {

constexpr int TG_ROWS = 8;          // rows per workgroup: two per wave
constexpr int TG_DIMS = 1024;       // widest slice

// A wave's own LDS writes are in place before what follows reads them (LDS operations of a wave complete in order).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// grid: (items, splits).  A wave takes two rows; per 64 tokens a lane scores one token for both, then the lanes hold columns.
// Masked tokens are not multiplied by zero but left out: their rows may hold anything.
template <typename T>
__global__ void __launch_bounds__(256) tree_generic_kernel(TreeArgs a) {
  extern __shared__ float sm[];                     // q [8][dl + d_r], weights [4][2][64]
  const int w = a.dl + a.d_r, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float* weights = sm + TG_ROWS * w + wave * 128;
  const int item = blockIdx.x, v = item / a.p.blocks, rb = item % a.p.blocks, i = v / a.B, b = v % a.B;
  const TreeLens len = tree_lens(a, b);
  const int rows = len.n * a.H, all_rows = a.T * a.H, r0 = rb * TG_ROWS;
  const int k0 = blockIdx.y * a.p.split_tokens, k1 = min(len.keys, k0 + a.p.split_tokens);
  const bool alive = r0 < rows && k0 < k1;          // the same in the whole workgroup
  const T* q_lat = static_cast<const T*>(a.q_lat) + (size_t)v * all_rows * a.dl;
  const T* q_pe = static_cast<const T*>(a.q_pe) + (size_t)b * all_rows * a.d_r;
  const T* pool = static_cast<const T*>(i == 0 ? a.pools[0] : i == 1 ? a.pools[1] : i == 2 ? a.pools[2] : i == 3 ? a.pools[3] :
                                        i == 4 ? a.pools[4] : i == 5 ? a.pools[5] : i == 6 ? a.pools[6] : a.pools[7]);
  if (alive)
    for (int x = tid; x < TG_ROWS * w; x += 256) {
      const int r = min(r0 + x / w, rows - 1), c = x % w;
      sm[x] = c < a.dl ? (float)q_lat[(size_t)r * a.dl + c] : (float)q_pe[(size_t)r * a.d_r + c - a.dl];
    }
  __syncthreads();
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float acc[2][TG_DIMS / 64];
#pragma unroll
  for (int d = 0; d < TG_DIMS / 64; ++d) acc[0][d] = acc[1][d] = 0.f;
  const int rw = r0 + 2 * wave;                     // this wave's rows: rw, rw + 1
  if (alive && rw < rows) {
    unsigned long long bits[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) bits[e] = a.mask[(size_t)b * a.T + min(rw + e, rows - 1) / a.H];
    const float* q = sm + 2 * wave * w;
    for (int t0 = k0; t0 < k1; t0 += 64) {
      const int t = min(t0 + lane, k1 - 1), nt = min(64, k1 - t0);
      const int page = a.block_table[(size_t)b * a.max_pages + t / a.page_tokens];
      const T* row = pool + ((size_t)page * a.page_tokens + t % a.page_tokens) * w;
      float s[2] = {0.f, 0.f};
      for (int c = 0; c < w; c += 8) {
        const Vec8 x = load8_cached(row + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s[0] = fmaf(x.v[e], q[c + e], s[0]);
          s[1] = fmaf(x.v[e], q[w + c + e], s[1]);
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = t0 + lane - len.L;
        const bool sees = lane < nt && (j < 0 || ((bits[e] >> j) & 1));
        const float x = sees ? s[e] * a.scale_log2 : -INFINITY;
        const float m_new = fmaxf(m[e], wave_max(x));
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = exp2f(m[e] - ref), p = exp2f(x - ref);
        l[e] = fmaf(l[e], alpha, wave_sum(p));
        m[e] = m_new;
#pragma unroll
        for (int d = 0; d < TG_DIMS / 64; ++d) acc[e][d] *= alpha;
        weights[64 * e + lane] = p;
      }
      wave_lds_order();
      const size_t row_at = row - pool;
      for (int k = 0; k < nt; ++k) {
        const float p0 = weights[k], p1 = weights[64 + k];
        const size_t at = ((size_t)__builtin_amdgcn_readlane((int)(row_at >> 32), k) << 32) | (unsigned)__builtin_amdgcn_readlane((int)row_at, k);
#pragma unroll
        for (int d = 0; d < TG_DIMS / 64; ++d)
          if (64 * d + lane < a.dl) {
            const float x = (float)pool[at + 64 * d + lane];
            if (p0 != 0.f) acc[0][d] = fmaf(p0, x, acc[0][d]);
            if (p1 != 0.f) acc[1][d] = fmaf(p1, x, acc[1][d]);
          }
      }
      wave_lds_order();
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = rw + e;
    if (r >= all_rows) continue;
    const size_t out = (size_t)v * all_rows + r;
    if (a.p.n_splits == 1) {
      const float inv = l[e] != 0.f ? 1.0f / l[e] : 0.f;
#pragma unroll
      for (int d = 0; d < TG_DIMS / 64; ++d)
        if (64 * d + lane < a.dl) a.o_lat[out * a.dl + 64 * d + lane] = r < rows ? acc[e][d] * inv : 0.f;
      if (a.lse && lane == 0) a.lse[out] = r < rows ? merge_lse(m[e], l[e]) : -INFINITY;
    } else {
      const size_t slot = ((size_t)item * a.p.n_splits + blockIdx.y) * TG_ROWS + (2 * wave + e);
#pragma unroll
      for (int d = 0; d < TG_DIMS / 64; ++d)
        if (64 * d + lane < a.dl) a.part_acc[slot * a.dl + 64 * d + lane] = acc[e][d];
      if (lane == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * slot) = make_float2(m[e], r < rows ? l[e] : 0.f);
    }
  }
}

int launch_tree_generic(const TreeArgs& a, int dtype, hipStream_t st) {
  const dim3 grid((unsigned)(a.n_shards * a.B * a.p.blocks), (unsigned)a.p.n_splits);
  const size_t lds = ((size_t)TG_ROWS * (a.dl + a.d_r) + 4 * 128) * sizeof(float);
  if (dtype == TPLA_F32)
    hipLaunchKernelGGL(tree_generic_kernel<float>, grid, dim3(256), lds, st, a);
  else
    hipLaunchKernelGGL(tree_generic_kernel<bf16_t>, grid, dim3(256), lds, st, a);
  return check_launch("tree_generic_kernel");
}

// Merge: a workgroup takes 8 rows of one item, a wave two of them one after the other.  Per row the lanes hold the references and
// weights of 64 slots at a time, and the slots' rows are added in ascending order, MERGE_LOADS on their way together (each is a round trip
// to memory).  Rows of drafts that do not exist get zeros and -inf here.  grid: (groups of 8 rows of a (slice, sequence), (slice, sequence)).
constexpr int MERGE_ROWS = 8, MERGE_LOADS = 8;
__global__ void __launch_bounds__(256) tree_merge_kernel(TreeArgs a) {
  const int v = blockIdx.y, b = v % a.B, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int all_rows = a.T * a.H, r0 = blockIdx.x * MERGE_ROWS;
  const int item = v * a.p.blocks + r0 / a.p.block;             // whole groups of 8 lie in one
  int first, next, step, n;
  if (a.p.mfma) {
    const int w0 = a.plan[3 * item];                            // (of an item without rows: whatever lies there, not used)
    n = a.plan[3 * item + 1];
    first = 2 * w0 + a.plan[3 * item + 2];
    next = 2 * (w0 + 1);
    step = 2;
  } else {
    first = item * a.p.n_splits;
    next = first + 1;
    step = 1;
    n = a.p.n_splits;
  }
  const int rows = tree_lens(a, b).n * a.H;
  for (int e = wave; e < MERGE_ROWS; e += 4) {
    const int r = r0 + e;
    if (r >= all_rows) break;
    float* out = a.o_lat + ((size_t)v * all_rows + r) * a.dl;
    if (r >= rows) {
      for (int c = 4 * lane; c < a.dl; c += 256) *reinterpret_cast<f32x4*>(out + c) = f32x4{0.f, 0.f, 0.f, 0.f};
      if (a.lse && lane == 0) a.lse[(size_t)v * all_rows + r] = -INFINITY;
      continue;
    }
    if (n == 1 && a.p.mfma) continue;                           // written by the workgroup that had it whole
    const size_t local = r % a.p.block;
    auto slot = [&](int s) { return (size_t)(s == 0 ? first : next + (s - 1) * step) * a.p.block + local; };
    float M = -INFINITY, l = 0.f;
    for (int s0 = 0; s0 < n; s0 += 64) M = fmaxf(M, wave_max(s0 + lane < n ? a.part_ml[2 * slot(s0 + lane)] : -INFINITY));
    const float ref = M == -INFINITY ? 0.f : M;
    for (int c0 = 0; c0 < a.dl; c0 += 256) {
      const int c = min(c0 + 4 * lane, a.dl - 4);
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      for (int s0 = 0; s0 < n; s0 += 64) {
        float2 ml = make_float2(-INFINITY, 0.f);
        if (s0 + lane < n) ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * slot(s0 + lane));
        const float w = exp2f(ml.x - ref);
        if (c0 == 0) l += wave_sum(ml.y * w);
        const int here = min(64, n - s0);
        for (int s = 0; s < here; s += MERGE_LOADS) {
          f32x4 p[MERGE_LOADS];
#pragma unroll
          for (int k = 0; k < MERGE_LOADS; ++k) p[k] = *reinterpret_cast<const f32x4*>(a.part_acc + slot(s0 + min(s + k, here - 1)) * a.dl + c);
#pragma unroll
          for (int k = 0; k < MERGE_LOADS; ++k)
            if (s + k < here) x += p[k] * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), s + k));
        }
      }
      const float inv = l != 0.f ? 1.0f / l : 0.f;
      if (c0 + 4 * lane < a.dl) *reinterpret_cast<f32x4*>(out + c) = x * inv;
    }
    if (a.lse && lane == 0) a.lse[(size_t)v * all_rows + r] = merge_lse(M, l);
  }
}

int launch_tree_merge(const TreeArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)((a.T * a.H + MERGE_ROWS - 1) / MERGE_ROWS), (unsigned)(a.n_shards * a.B)), dim3(256), 0, st, a);
  return check_launch("tree_merge_kernel");
}

}  // namespace tpla
