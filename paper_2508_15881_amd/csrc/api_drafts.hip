// C ABI entry points of the speculative decode step: argument validation, planning and dispatch.  No kernel is launched when
// validation fails.
#include <math.h>
#include "tpla_internal.h"

namespace tpla {

static int check_table(const tpla_shape_t* sh, int32_t max_pages) {
  if (max_pages < 1) return fail(TPLA_ERR_SHAPE, "max_pages_per_seq=%d", max_pages);
  if ((int64_t)max_pages * sh->page_tokens > (int64_t)2147483647)
    return fail(TPLA_ERR_SHAPE, "max_pages_per_seq * page_tokens overflows int32");
  return TPLA_OK;
}

static int check_drafts(int32_t T) {
  if (T < 1 || T > TPLA_MAX_DRAFTS) return fail(TPLA_ERR_SHAPE, "T=%d is not in 1 .. %d", T, TPLA_MAX_DRAFTS);
  return TPLA_OK;
}

static TreePlan plan_tree(const tpla_shape_t& sh, int n_shards, int T, int max_pages) {
  TreePlan p;
  if (tree_mfma_supported(sh)) {
    tree_mfma_plan(sh, n_shards, T, max_pages, &p);
    return p;
  }
  p.mfma = 0;
  p.n_wg = 0;
  p.teams = 0;
  // Four rows per wave read LDS a third as often; one row per wave where that leaves compute units idle (two sequences of 128 tokens, 20
  // rows, 32 columns: 17.9 us with four, 11.6 with one).
  p.block = (double)n_shards * sh.B * ((T * sh.H + 15) / 16) >= device_cu_count() ? 16 : 4;
  p.blocks = (T * sh.H + p.block - 1) / p.block;
  // enough workgroups to fill the chip, not below 256 tokens each
  const double items = (double)n_shards * sh.B * p.blocks, tokens = (double)max_pages * sh.page_tokens;
  int n = (int)fmin(fmax(4.0 * device_cu_count() / items, 1.0), fmax(tokens / 256.0, 1.0));
  const int64_t per = ((int64_t)max_pages * sh.page_tokens + n - 1) / n;
  p.split_tokens = (int)((per + 63) / 64 * 64 > 2147483584LL ? 2147483584LL : (per + 63) / 64 * 64);
  p.n_splits = (int)(((int64_t)max_pages * sh.page_tokens + p.split_tokens - 1) / p.split_tokens);
  return p;
}

static size_t tree_slots(const tpla_shape_t& sh, int n_shards, const TreePlan& p) {
  if (p.mfma) return 2 * (size_t)p.n_wg;
  return p.n_splits == 1 ? 0 : (size_t)n_shards * sh.B * p.blocks * p.n_splits;
}
static size_t tree_workspace(const tpla_shape_t& sh, int n_shards, const TreePlan& p) {
  size_t bytes = tree_slots(sh, n_shards, p) * p.block * (sh.d_c / sh.g + 2) * sizeof(float);
  if (p.mfma) bytes += (size_t)n_shards * sh.B * p.blocks * 3 * sizeof(int32_t);
  return bytes < 16 ? 16 : (bytes + 15) / 16 * 16;
}

// The shape and what follows from T: limits of the index arithmetic included.
static int check_tree(const tpla_shape_t* sh, int n_shards, int32_t T, int32_t max_pages, TreePlan* p) {
  int rc = check_shape(sh);
  if (rc || (rc = check_drafts(T)) || (rc = check_table(sh, max_pages))) return rc;
  const int dl = sh->d_c / sh->g;
  if ((int64_t)sh->B * T * sh->H > (int64_t)2147483647 / 2 || (int64_t)n_shards * sh->B > 65535 || sh->H > 65535)
    return fail(TPLA_ERR_UNSUPPORTED, "B * T * H (or n_shards * B, or H) too large");
  if (!tree_mfma_supported(*sh) && (dl > 1024 || dl + sh->d_r > 1984))
    return fail(TPLA_ERR_UNSUPPORTED, "d_c/g=%d above 1024, or d_c/g + d_r=%d above 1984", dl, dl + sh->d_r);
  // token and page numbers stay int in the kernels: a split, a tile, the lanes of a wave or two chunks of page ids past the end included
  if ((int64_t)max_pages * sh->page_tokens > ((int64_t)1 << 31) - (1 << 17))
    return fail(TPLA_ERR_UNSUPPORTED, "max_pages_per_seq * page_tokens above 2^31 - 2^17");
  *p = plan_tree(*sh, n_shards, T, max_pages);
  const double tiles = ((double)max_pages * sh->page_tokens + 31) / 32, items = (double)n_shards * sh->B * p->blocks;
  // (general: a workgroup of 256 threads per item, fewer than 2^32 in a launch)
  if (p->mfma ? items * (tiles + 8) >= 2147483647.0 : items >= 16777216.0 || items * p->n_splits >= 2147483647.0 || p->n_splits > 65535)
    return fail(TPLA_ERR_UNSUPPORTED, "n_shards * B * row blocks * max_pages_per_seq too large");
  return TPLA_OK;
}

static int tree_common(const tpla_shape_t* shape, int n_shards, int32_t T, const void* q_lat, const void* q_pe,
                       const void* const* pools, const int32_t* block_table, int32_t max_pages, const int32_t* seq_lens,
                       const int32_t* draft_lens, const uint64_t* mask, void* workspace, size_t workspace_bytes, float* o_lat,
                       float* lse, void* stream) {
  TreePlan p;
  int rc = check_tree(shape, n_shards, T, max_pages, &p);
  if (rc) return rc;
  if (!q_lat || !q_pe || !pools || !block_table || !seq_lens || !mask || !workspace || !o_lat)
    return fail(TPLA_ERR_NULL, "a required pointer is NULL");
  for (int i = 0; i < n_shards; ++i) {
    if (!pools[i]) return fail(TPLA_ERR_NULL, "cache pool %d is NULL", i);
    if (!aligned16(pools[i])) return fail(TPLA_ERR_ALIGN, "cache pool %d is not 16-byte aligned", i);
  }
  if (!aligned16(q_lat) || !aligned16(q_pe) || !aligned16(block_table) || !aligned16(seq_lens) || !aligned16(draft_lens) ||
      !aligned16(mask) || !aligned16(workspace) || !aligned16(o_lat) || !aligned16(lse))
    return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  const size_t need = tree_workspace(*shape, n_shards, p);
  if (workspace_bytes < need) return fail(TPLA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);

  TreeArgs a;
  a.q_lat = q_lat;
  a.q_pe = q_pe;
  for (int i = 0; i < TPLA_MAX_G; ++i) a.pools[i] = i < n_shards ? pools[i] : nullptr;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.draft_lens = draft_lens;
  a.mask = reinterpret_cast<const unsigned long long*>(mask);
  a.dl = shape->d_c / shape->g;
  const size_t part_rows = tree_slots(*shape, n_shards, p) * p.block;
  a.part_acc = static_cast<float*>(workspace);
  a.part_ml = a.part_acc + part_rows * a.dl;
  a.plan = reinterpret_cast<int32_t*>(a.part_ml + part_rows * 2);
  a.o_lat = o_lat;
  a.lse = lse;
  a.n_shards = n_shards;
  a.B = shape->B;
  a.T = T;
  a.H = shape->H;
  a.d_r = shape->d_r;
  a.page_tokens = shape->page_tokens;
  a.max_pages = max_pages;
  a.p = p;
  a.scale_log2 = shape->sm_scale * 1.4426950408889634f;
  hipStream_t st = (hipStream_t)stream;
  if (p.mfma) {
    if ((rc = launch_tree_mfma(a, st))) return rc;
  } else {
    if ((rc = launch_tree_generic(a, shape->dtype, st))) return rc;
    if (p.n_splits == 1) return TPLA_OK;
  }
  return launch_tree_merge(a, st);
}

}  // namespace tpla

using namespace tpla;

extern "C" {
#pragma GCC visibility push(default)

int tpla_extend_sequences(const tpla_shape_t* shape, const int32_t* seq_lens, const int32_t* add_lens, int32_t row_tokens,
                          const int32_t* depths, const int32_t* free_pages, int32_t n_free, const int32_t* pages_held,
                          int32_t* pages_held_out, int32_t* block_table, int32_t max_pages_per_seq, int32_t* cu_tokens,
                          int32_t* slots, int32_t* positions, int64_t n_tokens, int32_t* counts, void* stream) {
  int rc = check_shape(shape);
  if (rc || (rc = check_table(shape, max_pages_per_seq))) return rc;
  if (!seq_lens || !add_lens || !pages_held || !pages_held_out || !block_table || !cu_tokens || !counts)
    return fail(TPLA_ERR_NULL, "a required pointer is NULL");
  if (row_tokens < 0 || n_free < 0 || n_tokens < 0 || n_tokens > (int64_t)2147483647)
    return fail(TPLA_ERR_SHAPE, "row_tokens=%d n_free=%d n_tokens=%lld", row_tokens, n_free, (long long)n_tokens);
  if (row_tokens > 0 && n_tokens != (int64_t)shape->B * row_tokens)
    return fail(TPLA_ERR_SHAPE, "n_tokens=%lld is not B * row_tokens=%lld", (long long)n_tokens, (long long)shape->B * row_tokens);
  if (depths && row_tokens == 0) return fail(TPLA_ERR_SHAPE, "depths need rows (row_tokens > 0)");
  if (n_free > 0 && !free_pages) return fail(TPLA_ERR_NULL, "free_pages is NULL");
  if (n_tokens > 0 && (!slots || !positions)) return fail(TPLA_ERR_NULL, "slots/positions is NULL");
  if (!aligned16(seq_lens) || !aligned16(add_lens) || !aligned16(depths) || !aligned16(free_pages) || !aligned16(pages_held) ||
      !aligned16(pages_held_out) || !aligned16(block_table) || !aligned16(cu_tokens) || !aligned16(slots) || !aligned16(positions) ||
      !aligned16(counts))
    return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  ExtendArgs a{seq_lens, add_lens, depths, free_pages, pages_held, pages_held_out, block_table, cu_tokens, slots, positions, counts,
               shape->B, shape->page_tokens, max_pages_per_seq, row_tokens, n_free, (int32_t)n_tokens};
  return launch_extend_sequences(a, (hipStream_t)stream);
}

int tpla_rotary_frequencies(int32_t rot_dim, double base, double factor, int32_t original_positions, double beta_fast,
                            double beta_slow, double* freq) {
  if (!freq) return fail(TPLA_ERR_NULL, "freq is NULL");
  if (rot_dim < 2 || rot_dim % 2) return fail(TPLA_ERR_SHAPE, "rot_dim=%d must be even and at least 2", rot_dim);
  if (!(base > 1.0) || !isfinite(base) || !(factor >= 1.0) || !isfinite(factor) || original_positions < 0)
    return fail(TPLA_ERR_SHAPE, "base=%g factor=%g original_positions=%d", base, factor, original_positions);
  if (original_positions > 0 && !(beta_slow > 0.0 && beta_fast > beta_slow && isfinite(beta_fast)))
    return fail(TPLA_ERR_SHAPE, "beta_fast=%g beta_slow=%g", beta_fast, beta_slow);
  const double two_pi = 6.283185307179586476925;
  double low = 0.0, high = 0.0;
  if (original_positions > 0) {
    // the pair (a real number) that turns `turns` times over the original positions
    auto at = [&](double turns) { return rot_dim * log(original_positions / (two_pi * turns)) / (2.0 * log(base)); };
    low = fmax(floor(at(beta_fast)), 0.0);
    high = fmin(ceil(at(beta_slow)), rot_dim - 1.0);
  }
  for (int j = 0; j < rot_dim / 2; ++j) {
    const double f = pow(base, -2.0 * j / rot_dim);
    double slow = 1.0;
    // (pair 0 turns most: where it does so at most beta_slow times, the ramp ends ahead of it)
    if (original_positions > two_pi * beta_slow) slow = fmin(fmax((j - low) / fmax(high - low, 1e-3), 0.0), 1.0);
    freq[j] = f * (1.0 - slow) + f / factor * slow;
  }
  return TPLA_OK;
}

int tpla_apply_rotary(const tpla_shape_t* shape, int32_t layout, int32_t inverse, int32_t rot_dim, const double* freq,
                      float amplitude, const int32_t* positions, int64_t T, const void* q, int64_t q_token_stride,
                      int64_t q_head_stride, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, const void* k,
                      int64_t k_token_stride, void* k_out, int64_t k_out_token_stride, void* stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if (layout != TPLA_ROTARY_INTERLEAVED && layout != TPLA_ROTARY_HALF) return fail(TPLA_ERR_SHAPE, "unknown rotary layout %d", layout);
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > shape->d_r)
    return fail(TPLA_ERR_SHAPE, "rot_dim=%d must be even and in 2 .. d_r=%d", rot_dim, shape->d_r);
  if (T < 0 || T > (int64_t)2147483647) return fail(TPLA_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if (!isfinite(amplitude)) return fail(TPLA_ERR_SHAPE, "amplitude is not finite");
  if (rot_dim > 8192) return fail(TPLA_ERR_UNSUPPORTED, "rot_dim=%d above 8192", rot_dim);
  if (T == 0) return TPLA_OK;                        // (tensors of no tokens may have no address)
  if (!freq || !positions) return fail(TPLA_ERR_NULL, "freq/positions is NULL");
  if (!q != !q_out || !k != !k_out || (!q && !k)) return fail(TPLA_ERR_NULL, "q and q_out, or k and k_out, or both pairs are needed");
  const int esz = shape->dtype == TPLA_F32 ? 4 : 2;
  // the stride of a dimension of size 1, and those of a pair that is not there, mean nothing
  if (T == 1) q_token_stride = q_out_token_stride = k_token_stride = k_out_token_stride = 0;
  if (shape->H == 1) q_head_stride = q_out_head_stride = 0;
  if (!q) q_token_stride = q_head_stride = q_out_token_stride = q_out_head_stride = 0;
  if (!k) k_token_stride = k_out_token_stride = 0;
  const int64_t strides[] = {q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride, k_token_stride, k_out_token_stride};
  for (int64_t s : strides) {
    if (s < 0) return fail(TPLA_ERR_SHAPE, "a stride is negative");
    if (s % (16 / esz)) return fail(TPLA_ERR_ALIGN, "strides must be whole 16 bytes");
  }
  if (rows_beyond_memory(T, q_token_stride, shape->H, q_head_stride, esz) || rows_beyond_memory(T, q_out_token_stride, shape->H, q_out_head_stride, esz) ||
      rows_beyond_memory(T, k_token_stride, 1, 0, esz) || rows_beyond_memory(T, k_out_token_stride, 1, 0, esz))
    return fail(TPLA_ERR_SHAPE, "strides reach beyond any memory");
  // an output whose rows share memory would be written twice
  if (q && rows_share(T, q_out_token_stride, shape->H, q_out_head_stride, shape->d_r))
    return fail(TPLA_ERR_SHAPE, "rows of q_out overlap");
  if (k && T > 1 && k_out_token_stride < shape->d_r) return fail(TPLA_ERR_SHAPE, "rows of k_out overlap");
  if ((q && q == q_out && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride)) ||
      (k && k == k_out && k_token_stride != k_out_token_stride))
    return fail(TPLA_ERR_SHAPE, "in place needs equal strides");
  if (!aligned16(freq) || !aligned16(positions) || !aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(k_out))
    return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  RotaryArgs a;
  a.freq = freq;
  a.positions = positions;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.T = T;
  a.q_ts = q_token_stride;
  a.q_hs = q_head_stride;
  a.qo_ts = q_out_token_stride;
  a.qo_hs = q_out_head_stride;
  a.k_ts = k_token_stride;
  a.ko_ts = k_out_token_stride;
  a.H = shape->H;
  a.d_r = shape->d_r;
  a.rot = rot_dim;
  a.layout = layout;
  a.inverse = inverse ? 1 : 0;
  a.amplitude = amplitude;
  return launch_rotary(a, shape->dtype, (hipStream_t)stream);
}

size_t tpla_workspace_bytes_tree(const tpla_shape_t* shape, int32_t T, int32_t max_pages_per_seq) {
  TreePlan one, all;
  if (check_tree(shape, 1, T, max_pages_per_seq, &one) || check_tree(shape, shape->g, T, max_pages_per_seq, &all)) return 0;
  const size_t a = tree_workspace(*shape, 1, one), b = tree_workspace(*shape, shape->g, all);
  return a > b ? a : b;
}

int tpla_decode_shard_tree(const tpla_shape_t* shape, int32_t T, const void* q_lat_i, const void* q_pe, const void* shard_pool,
                           const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens,
                           const int32_t* draft_lens, const uint64_t* tree_mask, void* workspace, size_t workspace_bytes,
                           float* o_lat_i, float* lse_i, void* stream) {
  return tree_common(shape, 1, T, q_lat_i, q_pe, &shard_pool, block_table, max_pages_per_seq, seq_lens, draft_lens, tree_mask,
                     workspace, workspace_bytes, o_lat_i, lse_i, stream);
}

int tpla_decode_shards_tree(const tpla_shape_t* shape, int32_t T, const void* q_lat, const void* q_pe,
                            const void* const* shard_pools, const int32_t* block_table, int32_t max_pages_per_seq,
                            const int32_t* seq_lens, const int32_t* draft_lens, const uint64_t* tree_mask, void* workspace,
                            size_t workspace_bytes, float* o_lat, float* lse, void* stream) {
  const int rc = check_shape(shape);
  if (rc) return rc;
  return tree_common(shape, shape->g, T, q_lat, q_pe, shard_pools, block_table, max_pages_per_seq, seq_lens, draft_lens, tree_mask,
                     workspace, workspace_bytes, o_lat, lse, stream);
}

int tpla_decode_shards_tree_combine(const tpla_shape_t* shape, int32_t T, const void* q_lat, const void* q_pe,
                                    const void* const* shard_pools, const int32_t* block_table, int32_t max_pages_per_seq,
                                    const int32_t* seq_lens, const int32_t* draft_lens, const uint64_t* tree_mask,
                                    void* workspace, size_t workspace_bytes, const void* W_UV_t, void* o, int32_t o_dtype,
                                    float* o_lat, float* lse, void* stream) {
  int rc = check_shape(shape);
  if (rc) return rc;
  if (!W_UV_t || !o) return fail(TPLA_ERR_NULL, "W_UV_t/o is NULL");
  if (o_dtype != TPLA_F32 && o_dtype != TPLA_BF16) return fail(TPLA_ERR_DTYPE, "o_dtype %d is neither TPLA_F32 nor TPLA_BF16", o_dtype);
  if (!aligned16(W_UV_t) || !aligned16(o)) return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  TreePlan p;
  if ((rc = check_tree(shape, shape->g, T, max_pages_per_seq, &p))) return rc;
  tpla_shape_t rows = *shape;
  rows.B = shape->B * T;                             // (check_tree: no overflow)
  if (!combine_mfma_supported(rows) && (rc = check_combine_grid(rows))) return rc;
  rc = tree_common(shape, shape->g, T, q_lat, q_pe, shard_pools, block_table, max_pages_per_seq, seq_lens, draft_lens, tree_mask,
                   workspace, workspace_bytes, o_lat, lse, stream);
  if (rc) return rc;
  return tpla_combine_shards_to(&rows, o_lat, W_UV_t, o, o_dtype, stream);
}

int tpla_commit_drafts(const tpla_shape_t* shape, int32_t T, const int32_t* accepted, const int32_t* n_accepted,
                       const int32_t* seq_lens, const int32_t* block_table, int32_t max_pages_per_seq,
                       void* const* shard_pools, int32_t* new_lens, void* stream) {
  int rc = check_shape(shape);
  if (rc || (rc = check_drafts(T)) || (rc = check_table(shape, max_pages_per_seq))) return rc;
  if (shape->B >= 1 << 22) return fail(TPLA_ERR_UNSUPPORTED, "B=%d above 2^22 - 1", shape->B);       // (1024 threads each, fewer than 2^32 in a launch)
  if (!accepted || !n_accepted || !seq_lens || !block_table || !shard_pools || !new_lens)
    return fail(TPLA_ERR_NULL, "a required pointer is NULL");
  CommitArgs a;
  for (int i = 0; i < TPLA_MAX_G; ++i) a.pools.p[i] = nullptr;
  for (int i = 0; i < shape->g; ++i) {
    if (!shard_pools[i]) return fail(TPLA_ERR_NULL, "shard_pools[%d] is NULL", i);
    if (!aligned16(shard_pools[i])) return fail(TPLA_ERR_ALIGN, "shard_pools[%d] not 16-byte aligned", i);
    a.pools.p[i] = shard_pools[i];
  }
  if (!aligned16(accepted) || !aligned16(n_accepted) || !aligned16(seq_lens) || !aligned16(block_table) || !aligned16(new_lens))
    return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  a.accepted = accepted;
  a.n_accepted = n_accepted;
  a.seq_lens = seq_lens;
  a.block_table = block_table;
  a.new_lens = new_lens;
  a.T = T;
  a.n_shards = shape->g;
  a.page_tokens = shape->page_tokens;
  a.max_pages = max_pages_per_seq;
  a.row_bytes = (shape->d_c / shape->g + shape->d_r) * (shape->dtype == TPLA_F32 ? 4 : 2);
  a.B = shape->B;
  return launch_commit_drafts(a, (hipStream_t)stream);
}

#pragma GCC visibility pop
}  // extern "C"
