// Attention of drafted tokens over the paged latent slices (tpla_decode_shard(s)_tree): the general kernel, for every width
// and type, and the merge of partial results of both kernels.
//
// Row r = t H + h of a (slice, sequence): s_k = scale (q_lat . c_k + q_pe . k_pe_k) over the committed tokens k < L and the
// drafts k = L + j whose bit j of mask[b, t] is set; o = sum softmax(s)_k c_k, lse = log sum exp(s).  One pass with the running
// maximum and sum.  A row that sees nothing has sum 0: o = 0, lse = -inf.
#include "split_merge.h"

namespace tpla {

constexpr int TG_DIMS = 1024;       // widest slice
constexpr int TG_LDS = 64 * 1024;
constexpr int TG_TOKENS = 4;        // tokens per lane whose products are on their way together; 8 groups of them are 32 tokens
constexpr int TG_BATCH = 8;         // pieces of 8 per thread on their way together

// A wave's own LDS writes are in place before what follows reads them (LDS operations of a wave complete in order).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ unsigned long long tree_seen(const TreeArgs& a, const TreeLens& len, int b, int t) {      // (all lanes of the wave)
  return drafts_seen(a, b, t, len.L, len.keys, drafts_there(draft_entry(a, b, (len.L + (int)(threadIdx.x & 63)) / a.page_tokens)));
}

// LDS of the general kernel, in floats: queries [rows][w], weights [tokens][rows], rows [stage][w + 4] (an odd number of 16-byte pieces: the
// lanes of a column spread over the banks).
__host__ __device__ constexpr int tg_floats(int w, int rows, int tokens, int stage) { return rows * w + tokens * rows + stage * (w + 4); }

// grid: (items of 4 RW rows, splits).  The rows of `stage` tokens are staged as floats, as many as LDS holds: short contexts are two round trips to
// memory and not two for every 64 tokens.  Of these a wave scores `tokens` (a power of two up to 64 that divides stage) at a time for its RW rows,
// 64 / tokens lanes per token, then its lanes hold columns.  Masked tokens are not multiplied by zero but left out: their rows
// may hold anything (a token that is seen with weight 0 is not: 0 * inf).  DC: columns per lane.
template <typename T, int DC, int RW>
__global__ void __launch_bounds__(256) tree_generic_kernel(TreeArgs a, int tokens, int stage) {
  extern __shared__ __align__(16) float sm[];
  constexpr int ROWS = 4 * RW;
  typedef float Weights __attribute__((ext_vector_type(RW)));
  const int w = a.dl + a.d_r, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* weights = sm + ROWS * w;
  float* staged = weights + tokens * ROWS;
  const int item = blockIdx.x, v = item / a.p.blocks, rb = item % a.p.blocks, i = v / a.B, b = v % a.B;
  const TreeLens len = tree_lens(a, b);
  const int rows = len.n * a.H, all_rows = a.T * a.H, r0 = rb * ROWS;
  const int k0 = blockIdx.y * a.p.split_tokens, k1 = min(len.keys, k0 + a.p.split_tokens);
  const bool alive = r0 < rows && k0 < k1;          // the same in the whole workgroup
  const T* q_lat = static_cast<const T*>(a.q_lat) + (size_t)v * all_rows * a.dl;
  const T* q_pe = static_cast<const T*>(a.q_pe) + (size_t)b * all_rows * a.d_r;
  const T* pool = static_cast<const T*>(tree_pool(a, i));
  const int rw = r0 + RW * wave;                    // this wave's rows: rw .. rw + RW - 1
  float m[RW], l[RW], acc[RW][DC];
#pragma unroll
  for (int e = 0; e < RW; ++e) {
    m[e] = -INFINITY;
    l[e] = 0.f;
#pragma unroll
    for (int d = 0; d < DC; ++d) acc[e][d] = 0.f;
  }
  if (alive) {
    for (int x = tid; x < ROWS * w / 8; x += 256) {
      const int r = min(r0 + 8 * x / w, rows - 1), c = 8 * x % w;
      const Vec8 q = c < a.dl ? load8_cached(q_lat + (size_t)r * a.dl + c) : load8_cached(q_pe + (size_t)r * a.d_r + c - a.dl);
#pragma unroll
      for (int e = 0; e < 8; ++e) sm[8 * x + e] = q.v[e];
    }
    const unsigned long long there = drafts_there(draft_entry(a, b, (len.L + lane) / a.page_tokens));
    unsigned long long bits[RW];
#pragma unroll
    for (int e = 0; e < RW; ++e) bits[e] = a.mask[(size_t)b * a.T + min(rw + e, rows - 1) / a.H] & there;
    const float* q = sm + RW * wave * w;
    float* mine = weights + wave * tokens * RW;     // [tokens][RW]
    const int parts = 64 / tokens, tok = lane % tokens, part = lane / tokens;
    // narrow slices: groups of lanes take different tokens
    const int cols = a.dl > 32 || tokens < 64 ? 64 : a.dl > 16 ? 32 : a.dl > 8 ? 16 : 8, groups = 64 / cols;
    const int col = lane % cols, group = lane / cols;
    for (int s0 = k0; s0 < k1; s0 += stage) {
      __syncthreads();                              // the rows before these are no longer read
      const int pieces = w / 8, here = min(stage, (k1 - s0 + tokens - 1) / tokens * tokens), all = here * pieces;
      for (int x0 = tid; x0 < all; x0 += 256 * TG_BATCH) {
        int at[TG_BATCH];
        size_t row[TG_BATCH];
#pragma unroll
        for (int e = 0; e < TG_BATCH; ++e) {
          const int x = min(x0 + 256 * e, all - 1), k = x / pieces, t = min(s0 + k, k1 - 1), p = t / a.page_tokens;
          at[e] = k * (w + 4) + 8 * (x - k * pieces);
          row[e] = ((size_t)max(a.block_table[(size_t)b * a.max_pages + p], 0) * a.page_tokens + (t - p * a.page_tokens)) * w + 8 * (x - k * pieces);
        }
        Vec8 r[TG_BATCH];
#pragma unroll
        for (int e = 0; e < TG_BATCH; ++e) r[e] = load8_cached(pool + row[e]);
#pragma unroll
        for (int e = 0; e < TG_BATCH; ++e)
          if (x0 + 256 * e < all) {
            *reinterpret_cast<f32x4*>(staged + at[e]) = f32x4{r[e].v[0], r[e].v[1], r[e].v[2], r[e].v[3]};
            *reinterpret_cast<f32x4*>(staged + at[e] + 4) = f32x4{r[e].v[4], r[e].v[5], r[e].v[6], r[e].v[7]};
          }
      }
      __syncthreads();
      if (rw >= rows) continue;
      for (int t0 = s0; t0 < s0 + here; t0 += tokens) {
        const float* tile = staged + (t0 - s0) * (w + 4);
        float s[RW];
#pragma unroll
        for (int e = 0; e < RW; ++e) s[e] = 0.f;
        for (int c = 4 * part; c < w; c += 4 * parts) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(tile + tok * (w + 4) + c);
#pragma unroll
          for (int e = 0; e < RW; ++e) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(q + e * w + c);
#pragma unroll
            for (int z = 0; z < 4; ++z) s[e] = fmaf(x[z], y[z], s[e]);
          }
        }
        const int t = t0 + tok, j = t - len.L;
#pragma unroll
        for (int e = 0; e < RW; ++e) {
          for (int d = tokens; d < 64; d <<= 1) s[e] += __shfl_xor(s[e], d);
          const bool sees = t < k1 && (j < 0 || ((bits[e] >> (j & 63)) & 1));
          const float x = sees ? s[e] * a.scale_log2 : -INFINITY;
          const float m_new = fmaxf(m[e], wave_max(x));
          const float ref = m_new == -INFINITY ? 0.f : m_new;
          const float alpha = exp2f(m[e] - ref), p = sees ? exp2f(x - ref) : -0.f;       // -0: not seen, which 0 (a score of -inf) is
          l[e] = fmaf(l[e], alpha, wave_sum(part == 0 ? p : 0.f));
          m[e] = m_new;
#pragma unroll
          for (int d = 0; d < DC; ++d) acc[e][d] *= alpha;
          if (part == 0) mine[tok * RW + e] = p;
        }
        wave_lds_order();
        // (tokens past the end are not seen; of committed ones nothing is masked)
        const int plain = min(len.L, k1) - t0;
        for (int k = 0; k < tokens; k += TG_TOKENS * groups) {
          Weights p[TG_TOKENS];
          float x[TG_TOKENS][DC];
#pragma unroll
          for (int u = 0; u < TG_TOKENS; ++u) {
            const int kk = k + u * groups + group;
            p[u] = *reinterpret_cast<const Weights*>(mine + kk * RW);
#pragma unroll
            for (int d = 0; d < DC; ++d) x[u][d] = tile[kk * (w + 4) + min(64 * d + col, w - 1)];
          }
          if (k + TG_TOKENS * groups <= plain) {
#pragma unroll
            for (int u = 0; u < TG_TOKENS; ++u)
#pragma unroll
              for (int d = 0; d < DC; ++d)
#pragma unroll
                for (int e = 0; e < RW; ++e) acc[e][d] = fmaf(p[u][e], x[u][d], acc[e][d]);
          } else {
#pragma unroll
            for (int u = 0; u < TG_TOKENS; ++u)
#pragma unroll
              for (int d = 0; d < DC; ++d)
#pragma unroll
                for (int e = 0; e < RW; ++e) acc[e][d] = __float_as_uint(p[u][e]) != 0x80000000u ? fmaf(p[u][e], x[u][d], acc[e][d]) : acc[e][d];
          }
        }
        wave_lds_order();
      }
    }
#pragma unroll
    for (int e = 0; e < RW; ++e)
      for (int d = cols; d < 64; d <<= 1) acc[e][0] += __shfl_xor(acc[e][0], d);
  }
#pragma unroll
  for (int e = 0; e < RW; ++e) {
    const int r = rw + e;
    if (r >= all_rows) continue;
    const size_t out = (size_t)v * all_rows + r;
    if (a.p.n_splits == 1) {
      if (l[e] == 0.f && r < rows && (len.L > 0 || tree_seen(a, len, b, r / a.H) != 0)) l[e] = __builtin_nanf("");
      const float inv = l[e] != 0.f ? 1.0f / l[e] : 0.f;
#pragma unroll
      for (int d = 0; d < DC; ++d)
        if (64 * d + lane < a.dl) a.o_lat[out * a.dl + 64 * d + lane] = r < rows ? acc[e][d] * inv : 0.f;
      if (a.lse && lane == 0) a.lse[out] = r < rows ? merge_lse(m[e], l[e]) : -INFINITY;
    } else if (r < rows) {
      const size_t slot = ((size_t)item * a.p.n_splits + blockIdx.y) * ROWS + (RW * wave + e);
#pragma unroll
      for (int d = 0; d < DC; ++d)
        if (64 * d + lane < a.dl) a.part_acc[slot * a.dl + 64 * d + lane] = acc[e][d];
      if (lane == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * slot) = make_float2(m[e], l[e]);
    }
  }
}

template <typename T, int RW>
static int launch_generic(const TreeArgs& a, hipStream_t st) {
  const int w = a.dl + a.d_r, rows = 4 * RW;
  int tokens = 64;
  while (tokens > 4 && tg_floats(w, rows, tokens, tokens) * 4 > TG_LDS) tokens /= 2;
  int stage = tokens;
  while (stage < 256 && stage < a.p.split_tokens && tg_floats(w, rows, tokens, 2 * stage) * 4 <= TG_LDS) stage *= 2;
  const size_t lds = (size_t)tg_floats(w, rows, tokens, stage) * 4;
  void (*fn)(TreeArgs, int, int) = a.dl <= 64 ? tree_generic_kernel<T, 1, RW> : a.dl <= 256 ? tree_generic_kernel<T, 4, RW> : tree_generic_kernel<T, TG_DIMS / 64, RW>;
  const int rc = allow_lds(reinterpret_cast<const void*>(fn), 160 * 1024, "tree_generic_kernel");
  if (rc) return rc;
  const dim3 grid((unsigned)(a.n_shards * a.B * a.p.blocks), (unsigned)a.p.n_splits);
  hipLaunchKernelGGL(fn, grid, dim3(256), lds, st, a, tokens, stage);
  return check_launch("tree_generic_kernel");
}

int launch_tree_generic(const TreeArgs& a, int dtype, hipStream_t st) {
  if (a.p.block == 4) return dtype == TPLA_F32 ? launch_generic<float, 1>(a, st) : launch_generic<bf16_t, 1>(a, st);
  return dtype == TPLA_F32 ? launch_generic<float, 4>(a, st) : launch_generic<bf16_t, 4>(a, st);
}

// Merge: a wave takes one row after another of an item, MERGE_LOADS slots' rows on their way together, the first of them requested with their references
// (each is a round trip to memory); the lanes hold the references and weights of 64 slots at a time, and the rows are added in ascending order.  Rows of
// drafts that do not exist get zeros and -inf here.  grid: (groups of `group` rows, a multiple of 4 that divides 16, of a (slice, sequence), (slice,
// sequence)).  Where the matrix kernels put zeros in the place of drafts' values that are not finite (a negative sum, or -1 partial results of an
// item that one workgroup had whole), rows that see such a draft get NaN in its column, whatever its weight: 0 * inf where its score is -inf.
constexpr int MERGE_LOADS = 8;
__global__ void __launch_bounds__(256) tree_merge_kernel(TreeArgs a, int group) {
  const int v = blockIdx.y, b = v % a.B, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int all_rows = a.T * a.H, r0 = blockIdx.x * group;
  const int item = v * a.p.blocks + r0 / a.p.block;             // a group lies in one
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
  unsigned cleaned = 0, empty = 0;                              // rows of the group
  for (int e = wave; e < group; e += 4) {
    const int r = r0 + e;
    if (r >= all_rows) break;
    float* out = a.o_lat + ((size_t)v * all_rows + r) * a.dl;
    if (r >= rows) {
      for (int c = 4 * lane; c < a.dl; c += 256) *reinterpret_cast<f32x4*>(out + c) = f32x4{0.f, 0.f, 0.f, 0.f};
      if (a.lse && lane == 0) a.lse[(size_t)v * all_rows + r] = -INFINITY;
      continue;
    }
    if (n <= 1 && a.p.mfma) {                                   // written by the workgroup that had it whole
      if (n < 0) cleaned |= 1u << e;
      continue;
    }
    const size_t local = r % a.p.block;
    auto slot = [&](int s) { return (size_t)(s == 0 ? first : next + (s - 1) * step) * a.p.block + local; };
    auto request = [&](f32x4 (&p)[MERGE_LOADS], int s0, int c) {
#pragma unroll
      for (int k = 0; k < MERGE_LOADS; ++k) p[k] = *reinterpret_cast<const f32x4*>(a.part_acc + slot(min(s0 + k, n - 1)) * a.dl + c);
    };
    f32x4 p[MERGE_LOADS];
    request(p, 0, min(4 * lane, a.dl - 4));
    float2 ml = make_float2(-INFINITY, 0.f);                    // of slot `lane`
    if (lane < n) ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * slot(lane));
    float M = wave_max(ml.x);
    for (int s0 = 64; s0 < n; s0 += 64) M = fmaxf(M, wave_max(s0 + lane < n ? a.part_ml[2 * slot(s0 + lane)] : -INFINITY));
    const float ref = M == -INFINITY ? 0.f : M;
    float l = 0.f;
    for (int c0 = 0; c0 < a.dl; c0 += 256) {
      const int c = min(c0 + 4 * lane, a.dl - 4);
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      for (int s0 = 0; s0 < n; s0 += 64) {
        float2 q = ml;
        if (s0 > 0) {
          q = make_float2(-INFINITY, 0.f);
          if (s0 + lane < n) q = *reinterpret_cast<const float2*>(a.part_ml + 2 * slot(s0 + lane));
        }
        const float w = exp2f(q.x - ref);
        if (c0 == 0) {
          l += wave_sum(fabsf(q.y) * w);
          if (__any(__float_as_int(q.y) < 0)) cleaned |= 1u << e;
        }
        const int here = min(64, n - s0);
        for (int s = 0; s < here; s += MERGE_LOADS) {
          if (c0 + s0 + s > 0) request(p, s0 + s, c);
#pragma unroll
          for (int k = 0; k < MERGE_LOADS; ++k)
            if (s + k < here) x += p[k] * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), s + k));
        }
      }
      const float inv = l != 0.f ? 1.0f / l : 0.f;
      if (c0 + 4 * lane < a.dl) *reinterpret_cast<f32x4*>(out + c) = x * inv;
    }
    if (a.lse && lane == 0) a.lse[(size_t)v * all_rows + r] = merge_lse(M, l);
    if (l == 0.f) empty |= 1u << e;
  }
  // ---- rare: rows of the matrix kernels whose drafts' values were cleaned, and rows without a weight ----
  if (!a.p.mfma) cleaned = 0;
  for (unsigned left = cleaned | empty; left; left &= left - 1) {
    const int e = __builtin_ctz(left), r = r0 + e;
    const TreeLens len = tree_lens(a, b);
    unsigned long long seen = tree_seen(a, len, b, r / a.H);
    float* out = a.o_lat + ((size_t)v * all_rows + r) * a.dl;   // (a lane's columns are those it wrote above)
    const float nan = __builtin_nanf("");
    if (((empty >> e) & 1) && (seen != 0 || len.L > 0)) {       // every score -inf: 0 / 0
      for (int c = 4 * lane; c < a.dl; c += 256) *reinterpret_cast<f32x4*>(out + c) = f32x4{nan, nan, nan, nan};
      if (a.lse && lane == 0) a.lse[(size_t)v * all_rows + r] = nan;
    } else if ((cleaned >> e) & 1) {                            // a value that is not finite, whatever its weight (0 * inf where its score is -inf)
      for (; seen; seen &= seen - 1) {
        const int k = len.L + __builtin_ctzll(seen), p = k / a.page_tokens;
        const unsigned short* row = static_cast<const unsigned short*>(tree_pool(a, v / a.B)) +
                                    ((size_t)a.block_table[(size_t)b * a.max_pages + p] * a.page_tokens + (k - p * a.page_tokens)) * (a.dl + a.d_r);
        for (int c = 4 * lane; c < a.dl; c += 256)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if ((row[c + x] & 0x7F80) == 0x7F80) out[c + x] = nan;
      }
    }
  }
}

int launch_tree_merge(const TreeArgs& a, hipStream_t st) {
  // one row per wave while that leaves no more than some workgroups per compute unit
  const int rows = a.T * a.H, n_v = a.n_shards * a.B;
  int group = 4;
  while (group < 16 && group < a.p.block && (long long)((rows + group - 1) / group) * n_v > 16LL * device_cu_count()) group *= 2;
  hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)((rows + group - 1) / group), (unsigned)n_v), dim3(256), 0, st, a, group);
  return check_launch("tree_merge_kernel");
}

}  // namespace tpla
