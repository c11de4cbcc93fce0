// Layers with a key and a value per group of query heads: what the translation units of tpla_norm_rotary_heads, tpla_append_heads,
// tpla_decode_heads and tpla_prefill_heads share.
#pragma once
#include "tpla_internal.h"

namespace tpla {

// ---- rows: see heads_rows.hip.  Strides in elements; q or k may be nullptr. ----
struct HeadRowsArgs {
  const double* freq;
  const int32_t* positions;
  const void *q, *k, *v, *q_weight, *k_weight;
  void *q_out, *k_out;         // k_out: rows, or with slots the pool
  void* v_pool;
  const int32_t* slots;        // nullptr: k_out is dense rows and there is no v
  int64_t T, q_ts, q_hs, qo_ts, qo_hs, k_ts, k_hs, ko_ts, ko_hs, v_ts, v_hs;
  int H, H_kv, d_k, d_v, page_tokens, rot, layout;
  float amplitude, eps;        // eps < 0: no norm
};
int launch_head_rows(HeadRowsArgs a, int dtype, hipStream_t st);

// ---- attention ----
struct HeadsArgs {
  const void *q, *k_pool, *v_pool;
  const int32_t *table, *lens, *cu;      // cu nullptr: decode, one row of q per sequence, lens count it; lens nullptr: 0
  void* o;
  float *lse, *part_acc, *part_ml;       // partial results: [slot][rows of an item], of d_v columns and of (reference, sum)
  int B, H, H_kv, G, d_k, d_v, page_tokens, max_pages, o_dtype;
  int T, max_new, n_splits;
  int tiles;                             // of rows: decode per (sequence, head of keys), prefill an upper bound for all sequences, per head of keys
  int32_t* plan;                         // ranges: where the merge finds an item's parts, three ints per item; prompts: tokens of a part
  int n_wg;                              // ranges: workgroups, each with a range (0: a workgroup per item); prompts: what the chip holds
  float scale_log2;
};

enum HeadsKernel { HEADS_GENERAL, HEADS_RANGES, HEADS_PROMPTS };
struct HeadsPlan {
  HeadsKernel kernel;
  int n_wg;                    // HeadsArgs::n_wg
  int64_t slots;               // partial results, of `rows` rows each
  int rows;                    // rows of an item
  int tiles;                   // HeadsArgs::tiles
  int64_t items;               // work items (upper bound)
  int n_splits;                // general: parts of an item; prompts: 1, or rounds of parts that there are slots for
  size_t workspace;            // bytes
};
// max_new = 0: decode
HeadsPlan general_heads_plan(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages);
size_t general_heads_room(const tpla_heads_t& sh, int64_t T, int32_t max_pages);      // the most that a prefill of up to T tokens needs
int launch_general_heads(const HeadsArgs& a, const HeadsPlan& p, int dtype, hipStream_t st);
// bf16, d_k = d_v of 64 or 128, pages of a multiple of 16 tokens, at most 32 rows per head of keys: see heads_ranges.hip
bool heads_mfma_supported(const tpla_heads_t& sh);
bool heads_ranges_fit(const tpla_heads_t& sh, int32_t max_new);
HeadsPlan heads_ranges_plan(const tpla_heads_t& sh, int32_t max_new, int32_t max_pages);
size_t heads_ranges_room(const tpla_heads_t& sh, int32_t max_new, int32_t max_pages);
int launch_heads_ranges(const HeadsArgs& a, const HeadsPlan& p, hipStream_t st);
// the same types, any number of rows: see heads_prompts.hip
HeadsPlan heads_prompts_plan(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages);
size_t heads_prompts_room(const tpla_heads_t& sh, int64_t T, int32_t max_pages);
int launch_heads_prompts(const HeadsArgs& a, const HeadsPlan& p, hipStream_t st);

// A work item: `rows` rows of one head of keys of one sequence.  Row r of a (sequence, head) is its new token r / G, query head r % G of the group.
struct HeadsItem {
  int b, kvh, row0, rows;      // rows of the sequence in all; row0 < rows
  int first;                   // row of q and o of its first new token
  int L, keys;                 // tokens before the new ones, tokens that exist
  // Tokens that row r sees (negative pages apart): L + r / G + 1 of those that exist.
  __device__ __forceinline__ int sees(int r, int G) const { return r / G + 1 < keys - L ? L + r / G + 1 : keys; }
};

__device__ __forceinline__ int wave_prefix(int v) {      // inclusive sum over the wave
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

__device__ __forceinline__ int heads_cap(const HeadsArgs& a) { return a.max_pages * a.page_tokens; }      // (the host: below 2^31)
// New tokens of sequence b and the first of their rows.
__device__ __forceinline__ int heads_new(const HeadsArgs& a, int b, int& first) {
  if (!a.cu) {
    first = b;
    return 1;
  }
  first = min(max(a.cu[b], 0), a.T);
  return min(min(max(a.cu[b + 1], first), a.T) - first, a.max_new);
}
__device__ __forceinline__ void heads_lens(const HeadsArgs& a, int b, int n, HeadsItem& it) {
  const int cap = heads_cap(a), len = a.lens ? min(max(a.lens[b], 0), cap) : 0;
  it.L = a.cu ? len : len - 1;                             // (decode of an empty sequence: -1, its row sees 0 tokens)
  it.keys = a.cu ? min(len + min(n, cap - len), cap) : len;
}
// Item `idx` of the grid; false: there is none (the grid is an upper bound).  All lanes of a wave take part.  ROWS: rows of an item.
// Heads of keys are the slower index of a prefill: the row tiles that read the same keys follow each other.
template <int ROWS>
__device__ __forceinline__ bool heads_item(const HeadsArgs& a, int idx, HeadsItem& it) {
  if (!a.cu) {
    const int tile = idx % a.tiles, v = idx / a.tiles;
    it.kvh = v % a.H_kv;
    it.b = v / a.H_kv;
    it.row0 = tile * ROWS;
    it.rows = a.G;
    it.first = it.b;
    heads_lens(a, it.b, 1, it);
    return true;
  }
  const int lane = threadIdx.x & 63;
  it.kvh = idx / a.tiles;
  int tile = idx % a.tiles;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int b = b0 + lane;
    int first = 0;
    const int n = b < a.B ? heads_new(a, b, first) : 0;
    const int tiles = (n * a.G + ROWS - 1) / ROWS, incl = wave_prefix(tiles);
    const unsigned long long past = __ballot(incl > tile);
    if (past == 0) {
      tile -= __builtin_amdgcn_readlane(incl, 63);
      continue;
    }
    const int src = __builtin_ctzll(past);
    it.b = b0 + src;
    tile -= __builtin_amdgcn_readlane(incl - tiles, src);
    const int mine = __builtin_amdgcn_readlane(n, src);
    it.first = __builtin_amdgcn_readlane(first, src);
    it.rows = mine * a.G;
    it.row0 = tile * ROWS;
    heads_lens(a, it.b, mine, it);
    return true;
  }
  return false;
}

// Tokens of a part of an item that sees `keys` of them: equal for all but the last, at least HEADS_SPLIT_MIN.
constexpr int HEADS_SPLIT_MIN = 128;
__host__ __device__ __forceinline__ int heads_split_tokens(int keys, int n_splits, int unit) {
  const int per = ((keys + n_splits - 1) / n_splits + unit - 1) / unit * unit;
  return per < HEADS_SPLIT_MIN ? HEADS_SPLIT_MIN : per;
}
__host__ __device__ __forceinline__ int heads_parts(int keys, int per) { return keys > 0 ? (keys - 1) / per + 1 : 1; }

__device__ __forceinline__ void store4(void* o, size_t at, int dtype, f32x4 x) {
  if (dtype == TPLA_F32) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(o) + at) = x;
  } else {
    const bf16x4 y = {(bf16_t)x[0], (bf16_t)x[1], (bf16_t)x[2], (bf16_t)x[3]};
    *reinterpret_cast<bf16x4*>(static_cast<bf16_t*>(o) + at) = y;
  }
}

// A row's reference and sum at the end of a part of its tokens.  One that sees tokens but no score above -inf: the sum becomes NaN (0 / 0),
// which counts where no other part has such a score.  One with a score that is NaN and none above -inf: the reference becomes +inf, so that
// the NaN counts whatever the other parts hold.
__device__ __forceinline__ void heads_close(float& m, float& l, bool seen) {
  if (m != -INFINITY) return;
  if (l != l)
    m = INFINITY;
  else if (seen)
    l = __builtin_nanf("");
}
// Parts (reference, sum) joined one after the other, with `top` their largest reference: the factor of the part's columns.
__device__ __forceinline__ float heads_join(float top, float2 part, float& l) {
  if (top == -INFINITY) {
    l += part.y;
    return 0.f;
  }
  if (part.x == -INFINITY) return 0.f;
  const float by = __builtin_amdgcn_exp2f(part.x - top);
  l = fmaf(part.y, by, l);
  return by;
}
__device__ __forceinline__ float heads_inverse(float l) { return l == 0.f ? 0.f : 1.0f / l; }
__device__ __forceinline__ float heads_lse(float m, float l) {
  return m == -INFINITY ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

}  // namespace tpla
