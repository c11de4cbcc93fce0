// C ABI entry points of layers with grouped heads: argument validation, planning and dispatch.  No kernel is launched when validation fails.
#include <math.h>
#include "heads.h"

namespace tpla {

static int check_heads(const tpla_heads_t* sh) {
  if (!sh) return fail(TPLA_ERR_NULL, "shape is NULL");
  if (sh->dtype != TPLA_F32 && sh->dtype != TPLA_BF16) return fail(TPLA_ERR_DTYPE, "dtype %d is neither TPLA_F32 nor TPLA_BF16", sh->dtype);
  if (sh->B < 1 || sh->H < 1 || sh->H_kv < 1 || sh->d_k < 1 || sh->d_v < 1 || sh->page_tokens < 1)
    return fail(TPLA_ERR_SHAPE, "every dimension must be positive (B=%d H=%d H_kv=%d d_k=%d d_v=%d page_tokens=%d)", sh->B, sh->H, sh->H_kv,
                sh->d_k, sh->d_v, sh->page_tokens);
  if (sh->H % sh->H_kv) return fail(TPLA_ERR_SHAPE, "H=%d is not divisible by H_kv=%d", sh->H, sh->H_kv);
  if (sh->d_k % 8 || sh->d_v % 8) return fail(TPLA_ERR_SHAPE, "d_k=%d and d_v=%d must be multiples of 8 (16-byte row pieces)", sh->d_k, sh->d_v);
  if (!(sh->sm_scale > 0.0f) || !isfinite(sh->sm_scale)) return fail(TPLA_ERR_SHAPE, "sm_scale must be positive and finite");
  if (sh->d_k > 256 || sh->d_v > 256) return fail(TPLA_ERR_UNSUPPORTED, "d_k=%d d_v=%d above 256", sh->d_k, sh->d_v);
  if (sh->H > 65535) return fail(TPLA_ERR_UNSUPPORTED, "H=%d above 65535", sh->H);
  if ((int64_t)sh->H_kv * sh->page_tokens > (int64_t)2147483647) return fail(TPLA_ERR_UNSUPPORTED, "H_kv * page_tokens too large");
  return TPLA_OK;
}

static int check_heads_table(const tpla_heads_t* sh, int32_t max_pages) {
  if (max_pages < 1) return fail(TPLA_ERR_SHAPE, "max_pages_per_seq=%d", max_pages);
  // token numbers stay int in the kernels, a split or a few tiles past the end included
  if ((int64_t)max_pages * sh->page_tokens > ((int64_t)1 << 31) - (1 << 17))
    return fail(TPLA_ERR_UNSUPPORTED, "max_pages_per_seq * page_tokens above 2^31 - 2^17");
  return TPLA_OK;
}

// ---- rows ----
struct RowsOf {
  const char* name;
  const void* p;
  int64_t *ts, *hs;
  int heads, width;
  bool written;
};

static int check_rows(int64_t T, int esz, const RowsOf* rows, int n) {
  for (int i = 0; i < n; ++i) {
    const RowsOf& r = rows[i];
    // the stride of a dimension of size 1, and those of rows that are not there, mean nothing
    if (!r.p || T == 1) *r.ts = 0;
    if (!r.p || r.heads == 1) *r.hs = 0;
    if (!r.p) continue;
    if (*r.ts < 0 || *r.hs < 0) return fail(TPLA_ERR_SHAPE, "a stride of %s is negative", r.name);
    if (*r.ts % (16 / esz) || *r.hs % (16 / esz)) return fail(TPLA_ERR_ALIGN, "strides of %s must be whole 16 bytes", r.name);
    if (rows_beyond_memory(T, *r.ts, r.heads, *r.hs, esz)) return fail(TPLA_ERR_SHAPE, "strides of %s reach beyond any memory", r.name);
    if (!aligned16(r.p)) return fail(TPLA_ERR_ALIGN, "%s is not 16-byte aligned", r.name);
    // an output whose rows share memory would be written twice
    if (r.written && rows_share(T, *r.ts, r.heads, *r.hs, r.width)) return fail(TPLA_ERR_SHAPE, "rows of %s overlap", r.name);
  }
  return TPLA_OK;
}

static int check_turn(const tpla_heads_t* sh, int32_t layout, int32_t rot_dim, const double* freq, float amplitude, const void* q_weight,
                      const void* k_weight, float norm_eps, const int32_t* positions, int64_t T) {
  if (layout != TPLA_ROTARY_INTERLEAVED && layout != TPLA_ROTARY_HALF) return fail(TPLA_ERR_SHAPE, "unknown rotary layout %d", layout);
  if (rot_dim < 0 || rot_dim % 2 || rot_dim > sh->d_k)
    return fail(TPLA_ERR_SHAPE, "rot_dim=%d must be even and in 0 .. d_k=%d", rot_dim, sh->d_k);
  if (T < 0 || T > (int64_t)2147483647) return fail(TPLA_ERR_SHAPE, "T=%lld out of range", (long long)T);
  if (!isfinite(amplitude)) return fail(TPLA_ERR_SHAPE, "amplitude is not finite");
  if (!isfinite(norm_eps)) return fail(TPLA_ERR_SHAPE, "norm_eps is not finite");
  if (norm_eps < 0.0f && (q_weight || k_weight)) return fail(TPLA_ERR_SHAPE, "weights without a norm (norm_eps < 0)");
  if (T == 0) return TPLA_OK;                        // (tensors of no tokens may have no address)
  if (rot_dim > 0 && (!freq || !positions)) return fail(TPLA_ERR_NULL, "freq/positions is NULL");
  if (!aligned16(freq) || !aligned16(positions) || !aligned16(q_weight) || !aligned16(k_weight))
    return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  return TPLA_OK;
}

static HeadRowsArgs rows_args(const tpla_heads_t* sh, int32_t layout, int32_t rot_dim, const double* freq, float amplitude, const void* q_weight,
                              const void* k_weight, float norm_eps, const int32_t* positions, int64_t T) {
  HeadRowsArgs a{};
  a.freq = freq;
  a.positions = positions;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.T = T;
  a.H = sh->H;
  a.H_kv = sh->H_kv;
  a.d_k = sh->d_k;
  a.d_v = sh->d_v;
  a.page_tokens = sh->page_tokens;
  a.rot = rot_dim;
  a.layout = layout;
  a.amplitude = amplitude;
  a.eps = norm_eps;
  return a;
}

// ---- attention ----
static HeadsPlan plan_heads(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages) {
  if (heads_mfma_supported(sh)) return heads_ranges_fit(sh, max_new) ? heads_ranges_plan(sh, max_new, max_pages) : heads_prompts_plan(sh, T, max_new, max_pages);
  return general_heads_plan(sh, T, max_new, max_pages);
}

// What a prefill of up to T tokens, up to max_new of a sequence, needs at most, whichever kernel and split its own numbers lead to.
static size_t prefill_room(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages) {
  if (!heads_mfma_supported(sh)) return general_heads_room(sh, T, max_pages);
  const size_t few = heads_ranges_room(sh, max_new, max_pages), many = heads_prompts_room(sh, T, max_pages);
  return few > many ? few : many;
}

// rows: of q (decode: B, prefill: T); max_new: 0 for decode, cut to T
static int check_attention(const tpla_heads_t* sh, int64_t rows, int32_t* max_new, int32_t max_pages, HeadsPlan* p) {
  int rc = check_heads(sh);
  if (rc || (rc = check_heads_table(sh, max_pages))) return rc;
  if (rows >= (int64_t)1 << 28) return fail(TPLA_ERR_UNSUPPORTED, "T=%lld above 2^28 - 1", (long long)rows);
  if (*max_new > rows) *max_new = (int32_t)rows;
  if (rows * sh->H >= (int64_t)1 << 28) return fail(TPLA_ERR_UNSUPPORTED, "rows * H = %lld above 2^28 - 1", (long long)rows * sh->H);
  if (sh->B >= 1 << 22) return fail(TPLA_ERR_UNSUPPORTED, "B=%d above 2^22 - 1", sh->B);
  *p = plan_heads(*sh, rows, *max_new, max_pages);
  if (p->kernel == HEADS_RANGES && p->n_wg > 0 && (double)p->items * (((double)max_pages * sh->page_tokens + 31) / 32 + 8) >= 2147483647.0)
    return fail(TPLA_ERR_UNSUPPORTED, "sequences * heads of keys * max_pages_per_seq too large");
  if (p->items >= (int64_t)1 << 23) return fail(TPLA_ERR_UNSUPPORTED, "%lld work items are more than a launch has", (long long)p->items);
  return TPLA_OK;
}

static int attention(const tpla_heads_t* sh, const HeadsPlan& p, const void* q, const void* k_pool, const void* v_pool,
                     const int32_t* table, int32_t max_pages, const int32_t* lens, const int32_t* cu, int64_t T, int32_t max_new,
                     void* workspace, size_t workspace_bytes, void* o, int32_t o_dtype, float* lse, void* stream) {
  if (o_dtype != TPLA_F32 && o_dtype != TPLA_BF16) return fail(TPLA_ERR_DTYPE, "o_dtype %d is neither TPLA_F32 nor TPLA_BF16", o_dtype);
  if (!q || !k_pool || !v_pool || !table || !o || (p.workspace > 0 && !workspace)) return fail(TPLA_ERR_NULL, "a required pointer is NULL");
  if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(table) || !aligned16(lens) || !aligned16(cu) ||
      !aligned16(workspace) || !aligned16(o) || !aligned16(lse))
    return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  if (workspace_bytes < p.workspace) return fail(TPLA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, p.workspace);
  HeadsArgs a{};
  a.q = q;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.table = table;
  a.lens = lens;
  a.cu = cu;
  a.o = o;
  a.lse = lse;
  a.part_acc = static_cast<float*>(workspace);
  a.part_ml = a.part_acc ? a.part_acc + (size_t)p.slots * p.rows * sh->d_v : nullptr;
  a.plan = a.part_acc ? reinterpret_cast<int32_t*>(a.part_ml + (size_t)p.slots * p.rows * 2) : nullptr;
  a.n_wg = p.n_wg;
  a.B = sh->B;
  a.H = sh->H;
  a.H_kv = sh->H_kv;
  a.G = sh->H / sh->H_kv;
  a.d_k = sh->d_k;
  a.d_v = sh->d_v;
  a.page_tokens = sh->page_tokens;
  a.max_pages = max_pages;
  a.o_dtype = o_dtype;
  a.T = (int)T;
  a.max_new = max_new;
  a.n_splits = p.n_splits;
  a.tiles = p.tiles;
  a.scale_log2 = sh->sm_scale * 1.4426950408889634f;
  if (p.kernel == HEADS_PROMPTS) return launch_heads_prompts(a, p, (hipStream_t)stream);
  if (p.kernel == HEADS_RANGES) return launch_heads_ranges(a, p, (hipStream_t)stream);
  return launch_general_heads(a, p, sh->dtype, (hipStream_t)stream);
}

}  // namespace tpla

using namespace tpla;

extern "C" {
#pragma GCC visibility push(default)

int tpla_norm_rotary_heads(const tpla_heads_t* shape, int32_t layout, int32_t rot_dim, const double* freq, float amplitude,
                           const void* q_weight, const void* k_weight, float norm_eps, const int32_t* positions, int64_t T,
                           const void* q, int64_t q_token_stride, int64_t q_head_stride, void* q_out, int64_t q_out_token_stride,
                           int64_t q_out_head_stride, const void* k, int64_t k_token_stride, int64_t k_head_stride, void* k_out,
                           int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
  int rc = check_heads(shape);
  if (rc || (rc = check_turn(shape, layout, rot_dim, freq, amplitude, q_weight, k_weight, norm_eps, positions, T)) || T == 0) return rc;
  if (!q != !q_out || !k != !k_out || (!q && !k)) return fail(TPLA_ERR_NULL, "q and q_out, or k and k_out, or both pairs are needed");
  const RowsOf rows[] = {{"q", q, &q_token_stride, &q_head_stride, shape->H, shape->d_k, false},
                         {"q_out", q_out, &q_out_token_stride, &q_out_head_stride, shape->H, shape->d_k, true},
                         {"k", k, &k_token_stride, &k_head_stride, shape->H_kv, shape->d_k, false},
                         {"k_out", k_out, &k_out_token_stride, &k_out_head_stride, shape->H_kv, shape->d_k, true}};
  if ((rc = check_rows(T, shape->dtype == TPLA_F32 ? 4 : 2, rows, 4))) return rc;
  if ((q && q == q_out && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride)) ||
      (k && k == k_out && (k_token_stride != k_out_token_stride || k_head_stride != k_out_head_stride)))
    return fail(TPLA_ERR_SHAPE, "in place needs equal strides");
  HeadRowsArgs a = rows_args(shape, layout, rot_dim, freq, amplitude, q_weight, k_weight, norm_eps, positions, T);
  a.q = q;
  a.q_ts = q_token_stride;
  a.q_hs = q_head_stride;
  a.q_out = q_out;
  a.qo_ts = q_out_token_stride;
  a.qo_hs = q_out_head_stride;
  a.k = k;
  a.k_ts = k_token_stride;
  a.k_hs = k_head_stride;
  a.k_out = k_out;
  a.ko_ts = k_out_token_stride;
  a.ko_hs = k_out_head_stride;
  return launch_head_rows(a, shape->dtype, (hipStream_t)stream);
}

int tpla_append_heads(const tpla_heads_t* shape, int32_t layout, int32_t rot_dim, const double* freq, float amplitude,
                      const void* q_weight, const void* k_weight, float norm_eps, const int32_t* positions, int64_t T,
                      const void* q, int64_t q_token_stride, int64_t q_head_stride, void* q_out, int64_t q_out_token_stride,
                      int64_t q_out_head_stride, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                      int64_t v_token_stride, int64_t v_head_stride, const int32_t* slots, void* k_pool, void* v_pool, void* stream) {
  int rc = check_heads(shape);
  if (rc || (rc = check_turn(shape, layout, rot_dim, freq, amplitude, q_weight, k_weight, norm_eps, positions, T)) || T == 0) return rc;
  if (!q != !q_out) return fail(TPLA_ERR_NULL, "q without q_out, or q_out without q");
  if (!k || !v || !slots || !k_pool || !v_pool) return fail(TPLA_ERR_NULL, "a required pointer is NULL");
  const RowsOf rows[] = {{"q", q, &q_token_stride, &q_head_stride, shape->H, shape->d_k, false},
                         {"q_out", q_out, &q_out_token_stride, &q_out_head_stride, shape->H, shape->d_k, true},
                         {"k", k, &k_token_stride, &k_head_stride, shape->H_kv, shape->d_k, false},
                         {"v", v, &v_token_stride, &v_head_stride, shape->H_kv, shape->d_v, false}};
  if ((rc = check_rows(T, shape->dtype == TPLA_F32 ? 4 : 2, rows, 4))) return rc;
  if (q && q == q_out && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride))
    return fail(TPLA_ERR_SHAPE, "in place needs equal strides");
  if (!aligned16(slots) || !aligned16(k_pool) || !aligned16(v_pool)) return fail(TPLA_ERR_ALIGN, "pointers must be 16-byte aligned");
  HeadRowsArgs a = rows_args(shape, layout, rot_dim, freq, amplitude, q_weight, k_weight, norm_eps, positions, T);
  a.q = q;
  a.q_ts = q_token_stride;
  a.q_hs = q_head_stride;
  a.q_out = q_out;
  a.qo_ts = q_out_token_stride;
  a.qo_hs = q_out_head_stride;
  a.k = k;
  a.k_ts = k_token_stride;
  a.k_hs = k_head_stride;
  a.k_out = k_pool;
  a.v = v;
  a.v_ts = v_token_stride;
  a.v_hs = v_head_stride;
  a.v_pool = v_pool;
  a.slots = slots;
  return launch_head_rows(a, shape->dtype, (hipStream_t)stream);
}

size_t tpla_workspace_bytes_heads(const tpla_heads_t* shape, int32_t max_pages_per_seq) {
  HeadsPlan p;
  int32_t none = 0;
  if (check_attention(shape, shape ? shape->B : 0, &none, max_pages_per_seq, &p)) return 0;
  return p.workspace < 16 ? 16 : p.workspace;
}

int tpla_decode_heads(const tpla_heads_t* shape, const void* q, const void* k_pool, const void* v_pool, const int32_t* block_table,
                      int32_t max_pages_per_seq, const int32_t* seq_lens, void* workspace, size_t workspace_bytes, void* o,
                      int32_t o_dtype, float* lse, void* stream) {
  HeadsPlan p;
  int32_t none = 0;
  const int rc = check_attention(shape, shape ? shape->B : 0, &none, max_pages_per_seq, &p);
  if (rc) return rc;
  if (!seq_lens) return fail(TPLA_ERR_NULL, "seq_lens is NULL");
  return attention(shape, p, q, k_pool, v_pool, block_table, max_pages_per_seq, seq_lens, nullptr, shape->B, 1, workspace, workspace_bytes, o,
                   o_dtype, lse, stream);
}

size_t tpla_workspace_bytes_prefill_heads(const tpla_heads_t* shape, int64_t T, int32_t max_new, int32_t max_pages_per_seq) {
  HeadsPlan p;
  if (T < 1 || max_new < 1 || check_attention(shape, T, &max_new, max_pages_per_seq, &p)) return 0;
  return prefill_room(*shape, T, max_new, max_pages_per_seq);
}

int tpla_prefill_heads(const tpla_heads_t* shape, const void* q, const void* k_pool, const void* v_pool, const int32_t* block_table,
                       int32_t max_pages_per_seq, const int32_t* seq_lens, const int32_t* cu_seqlens, int64_t T, int32_t max_new,
                       void* workspace, size_t workspace_bytes, void* o, int32_t o_dtype, float* lse, void* stream) {
  HeadsPlan p;
  if (T < 0 || max_new < 0 || (T > 0 && max_new == 0)) return fail(TPLA_ERR_SHAPE, "T=%lld max_new=%d", (long long)T, max_new);
  if (T == 0) {
    const int rc = check_heads(shape);
    return rc ? rc : check_heads_table(shape, max_pages_per_seq);
  }
  const int rc = check_attention(shape, T, &max_new, max_pages_per_seq, &p);
  if (rc) return rc;
  if (!cu_seqlens) return fail(TPLA_ERR_NULL, "cu_seqlens is NULL");
  return attention(shape, p, q, k_pool, v_pool, block_table, max_pages_per_seq, seq_lens, cu_seqlens, T, max_new, workspace, workspace_bytes, o,
                   o_dtype, lse, stream);
}

#pragma GCC visibility pop
}  // extern "C"
