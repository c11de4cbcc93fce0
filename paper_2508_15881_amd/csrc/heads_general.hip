// Attention of grouped heads over paged keys and values, the general kernel: every type, width and page size, prompts and single tokens.
//
//   s_t = scale (q . k_t),   o = sum_t softmax(s)_t v_t   over the tokens that a row sees, in one pass with the running maximum and sum
//
// in float on the matrix instructions: tokens are the M dimension of the scores, rows (new token, query head of the group) the N dimension,
//   S^T[token, row] = K[token, :] . Q[row, :],   O^T[dim, row] += V^T[dim, token] . P^T[token, row]
// so a lane holds one row of a block of 16 and the weights stay in the registers that the scores came in.  Widths are padded with zeros to
// NB blocks of 16 columns.  Bound by the float matrix instructions for long prompts (4000 tokens, 32 heads on 8, 128 columns: 1780 us = 74 TFLOP/s), by a round
// trip to memory, the way through LDS and two barriers per tile otherwise (three sequences of up to 70 tokens 9.6 us).
#include "heads.h"

namespace tpla {

constexpr int HG_JOIN_TOK = 64, HG_ROWS_TOK = 32;      // tokens staged at once
constexpr int HG_SPLIT = 512;                           // tokens of a block-table row from which on it pays to split them

// JOIN: the four waves have the same 16 rows and a quarter of the staged tokens each, and join at the end: few rows.  Otherwise 16 rows each.
template <int NB, bool JOIN>
struct GeneralTile {
  static constexpr int W = 16 * NB, PITCH = W + 4;     // an odd number of 16-byte pieces: the rows of a column spread over the banks
  static constexpr int TOK = JOIN ? HG_JOIN_TOK : HG_ROWS_TOK;
  static constexpr int ROWS = JOIN ? 16 : 64;
  static constexpr int BLOCKS = JOIN ? 1 : TOK / 16;   // of 16 tokens per wave
  static constexpr int PIECES = TOK * (W / 8);         // of 8 columns, of keys and of values
  static constexpr int PER_THREAD = (PIECES + 255) / 256;
  static constexpr int LDS = 2 * TOK * PITCH * 4 + 2 * TOK * 8 + 16;
  static_assert(!JOIN || 4 * 16 * (W + 4) <= 2 * TOK * PITCH, "the join uses the staged rows' place");
};

template <typename T, int NB, bool JOIN>
__global__ void __launch_bounds__(256) heads_general_kernel(HeadsArgs a) {
  using Tile = GeneralTile<NB, JOIN>;
  constexpr int PITCH = Tile::PITCH, TOK = Tile::TOK, BLOCKS = Tile::BLOCKS;
  extern __shared__ __align__(16) float sm[];
  float* const sk = sm;
  float* const sv = sm + TOK * PITCH;
  long long* const rows_at = reinterpret_cast<long long*>(sv + TOK * PITCH);      // [2][TOK]: row of the pools that a token is, -1: none
  volatile int* const odd = reinterpret_cast<int*>(rows_at + 2 * TOK);            // [2] whether some staged value is not finite, tile by tile in turn
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j16 = lane & 15, q4 = lane >> 4;
  HeadsItem it;
  if (!heads_item<Tile::ROWS>(a, blockIdx.x, it)) return;
  const int last = min(it.row0 + Tile::ROWS, it.rows) - 1;
  const int keys = max(it.sees(last, a.G), 0), least = it.sees(it.row0, a.G);      // most and fewest tokens that a row of the item sees
  const int per = heads_split_tokens(keys, a.n_splits, TOK);
  const int parts = heads_parts(keys, per), split = blockIdx.y;
  if (split >= parts) return;
  const int k0 = split * per, k1 = min(keys, k0 + per);

  const int row = it.row0 + (JOIN ? 0 : 16 * wave) + j16;
  const bool alive = row < it.rows;
  const int mine = min(row, it.rows - 1), sees = alive ? it.sees(mine, a.G) : 0;
  const size_t out_row = (size_t)(it.first + mine / a.G) * a.H + it.kvh * a.G + mine % a.G;
  f32x4 q[NB], acc[NB];
#pragma unroll
  for (int s = 0; s < NB; ++s) {
    acc[s] = q[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int c = 16 * s + 4 * q4;
    if (c < a.d_k) {
      const T* src = static_cast<const T*>(a.q) + out_row * a.d_k + c;
#pragma unroll
      for (int e = 0; e < 4; ++e) q[s][e] = load_as_f32(src + e);
    }
  }
  float m = -INFINITY, l = 0.f;
  bool seen = false;
  const int32_t* table = a.table + (size_t)it.b * a.max_pages;
  // Where the tokens of a tile are is found a tile ahead: one round trip to memory per tile and not two.
  auto find_rows = [&](int t0, int which) {
    if (tid >= TOK) return;
    const int t = t0 + tid, page = t < k1 ? table[t / a.page_tokens] : -1;
    rows_at[which * TOK + tid] = page < 0 ? -1 : ((long long)page * a.H_kv + it.kvh) * a.page_tokens + t % a.page_tokens;
  };
  if (tid < 2) odd[tid] = 0;
  find_rows(k0, 0);
  __syncthreads();

  for (int t0 = k0, which = 0; t0 < k1; t0 += TOK, which ^= 1) {
    const bool some_masked = t0 + TOK > least;
    const long long* const at = rows_at + which * TOK;
    // (columns from d on are zeros, and so are tokens that are none)
    Vec8 x[2][Tile::PER_THREAD];
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int k = 0; k < Tile::PER_THREAD; ++k) {
        const int p = tid + 256 * k, tok = p / (Tile::W / 8), c = 8 * (p % (Tile::W / 8)), d = part ? a.d_v : a.d_k;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[part][k].v[e] = 0.f;
        if (p < Tile::PIECES && c < d) {
          const long long row = at[tok];
          if (row >= 0) x[part][k] = load8_cached(static_cast<const T*>(part ? a.v_pool : a.k_pool) + row * d + c);
        }
      }
    find_rows(t0 + TOK, which ^ 1);
#pragma unroll
    for (int part = 0; part < 2; ++part)
#pragma unroll
      for (int k = 0; k < Tile::PER_THREAD; ++k) {
        const int p = tid + 256 * k, tok = p / (Tile::W / 8), c = 8 * (p % (Tile::W / 8));
        if (p >= Tile::PIECES) continue;
        const Vec8& r = x[part][k];
        if (part && some_masked) {
          bool fine = true;
#pragma unroll
          for (int e = 0; e < 8; ++e) fine = fine && __builtin_isfinite(r.v[e]);
          if (!fine) odd[which] = 1;
        }
        float* dst = (part ? sv : sk) + tok * PITCH + c;
        *reinterpret_cast<f32x4*>(dst) = f32x4{r.v[0], r.v[1], r.v[2], r.v[3]};
        *reinterpret_cast<f32x4*>(dst + 4) = f32x4{r.v[4], r.v[5], r.v[6], r.v[7]};
      }
    __syncthreads();
    const int tok0 = JOIN ? 16 * wave : 0;
    f32x4 s[BLOCKS];
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < BLOCKS; ++n) {
      s[n] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float* src = sk + (tok0 + 16 * n + j16) * PITCH + 4 * q4;
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const f32x4 k = *reinterpret_cast<const f32x4*>(src + 16 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[c][e], s[n], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int tok = tok0 + 16 * n + 4 * q4 + i;
        const bool vis = at[tok] >= 0 && t0 + tok < sees;
        seen = seen || vis;
        s[n][i] = vis ? s[n][i] * a.scale_log2 : -INFINITY;
        top = fmaxf(top, s[n][i]);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - ref);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(s[n][i] - ref);
        l += s[n][i];
      }
#pragma unroll
    for (int c = 0; c < NB; ++c) acc[c] *= alpha;
    if (!odd[which]) {
#pragma unroll
      for (int n = 0; n < BLOCKS; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* src = sv + (tok0 + 16 * n + 4 * q4 + i) * PITCH + j16;
#pragma unroll
          for (int c = 0; c < NB; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(src[16 * c], s[n][i], acc[c], 0, 0, 0);
        }
    } else {
      // Some rows do not see some of these values, and a weight of zero does not silence what is not finite: one token at a time, kept by
      // the rows that see it.
      for (int tok = tok0; tok < tok0 + 16 * BLOCKS; ++tok) {
        const int n = (tok - tok0) >> 4, i = tok & 3;
        const bool holds = q4 == ((tok >> 2) & 3), vis = at[tok] >= 0 && t0 + tok < sees;
        float p = 0.f;
#pragma unroll
        for (int nn = 0; nn < BLOCKS; ++nn)
#pragma unroll
          for (int ii = 0; ii < 4; ++ii)
            if (nn == n && ii == i && holds) p = s[nn][ii];
        const float* src = sv + tok * PITCH + j16;
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x4f32(holds ? src[16 * c] : 0.f, p, acc[c], 0, 0, 0);
          acc[c] = vis ? x : acc[c];
        }
      }
    }
    __syncthreads();                                   // the tile is read
    if (tid == 0) odd[which] = 0;                      // (set again two tiles on: the barrier of the next lies between)
  }

  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  int any = seen;
  any |= __shfl_xor(any, 16);
  any |= __shfl_xor(any, 32);
  heads_close(m, l, any);
  if constexpr (JOIN) {
    // the waves' references and sums, then their columns, through LDS
    float2* ml = reinterpret_cast<float2*>(sm);
    if (q4 == 0) ml[wave * 16 + j16] = make_float2(m, l);
    __syncthreads();
    float M = -INFINITY, total = 0.f;
    float2 all[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      all[w] = ml[w * 16 + j16];
      M = fmaxf(M, all[w].x);
    }
    float mine_by = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float by = heads_join(M, all[w], total);
      mine_by = w == wave ? by : mine_by;
    }
    const bool none = m == -INFINITY;                  // (nothing of this wave counts)
    __syncthreads();
    float* x = sm + wave * 16 * (Tile::W + 4) + j16 * (Tile::W + 4) + 4 * q4;
#pragma unroll
    for (int c = 0; c < NB; ++c) *reinterpret_cast<f32x4*>(x + 16 * c) = none ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[c] * mine_by;
    __syncthreads();
    m = M;
    l = total;
    if (wave > 0) return;
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) acc[c] += *reinterpret_cast<const f32x4*>(x + w * 16 * (Tile::W + 4) + 16 * c);
    }
  }
  if (!alive) return;
  if (parts == 1) {
    const float inv = heads_inverse(l);
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int at = 16 * c + 4 * q4;
      if (at < a.d_v) store4(a.o, out_row * a.d_v + at, a.o_dtype, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[c] * inv);
    }
    if (a.lse && q4 == 0) a.lse[out_row] = heads_lse(m, l);
  } else {
    const size_t slot = ((size_t)blockIdx.x * a.n_splits + split) * Tile::ROWS + (row - it.row0);
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      const int at = 16 * c + 4 * q4;
      if (at < a.d_v) *reinterpret_cast<f32x4*>(a.part_acc + slot * a.d_v + at) = acc[c];
    }
    if (q4 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * slot) = make_float2(m, l);
  }
}

// grid: (items, groups of 256 quads of columns).  The parts of an item, in their order; a thread holds four columns of a row.
template <int ROWS, int UNIT>
__global__ void __launch_bounds__(256) heads_merge_kernel(HeadsArgs a) {
  HeadsItem it;
  if (!heads_item<ROWS>(a, blockIdx.x, it)) return;
  const int last = min(it.row0 + ROWS, it.rows) - 1, keys = max(it.sees(last, a.G), 0);
  const int per = heads_split_tokens(keys, a.n_splits, UNIT), parts = heads_parts(keys, per);
  if (parts == 1) return;
  const int quads = a.d_v / 4, x = blockIdx.y * 256 + threadIdx.x;
  if (x < (last - it.row0 + 1) * quads) {
    const int r = x / quads, c = 4 * (x % quads), row = it.row0 + r;
    const size_t slot0 = (size_t)blockIdx.x * a.n_splits * ROWS + r;
    const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
    float M = -INFINITY, l = 0.f;
    for (int s = 0; s < parts; ++s) M = fmaxf(M, ml[slot0 + (size_t)s * ROWS].x);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < parts; ++s) {
      const float2 v = ml[slot0 + (size_t)s * ROWS];
      const float by = heads_join(M, v, l);
      if (v.x != -INFINITY) acc += *reinterpret_cast<const f32x4*>(a.part_acc + (slot0 + (size_t)s * ROWS) * a.d_v + c) * by;
    }
    const size_t out_row = (size_t)(it.first + row / a.G) * a.H + it.kvh * a.G + row % a.G;
    const float inv = heads_inverse(l);
    store4(a.o, out_row * a.d_v + c, a.o_dtype, l == 0.f ? acc : acc * inv);
    if (a.lse && c == 0) a.lse[out_row] = heads_lse(M, l);
  }
}

// Rows of an item: 16, which the four waves share, for few rows to a head of keys and where items of 64 would leave compute units idle (three prompts of up to
// 300 tokens, six heads, 96 columns, float: 34.8 us with 64, split and merged, 18.2 with 16); the rows of a sequence in items of 64 read the keys a quarter as often.
static int general_rows(const tpla_heads_t& sh, int64_t T, int32_t max_new) {
  const int64_t G = sh.H / sh.H_kv;
  if (G * (max_new > 0 ? max_new : 1) <= 16) return 16;
  const int64_t items = max_new > 0 ? (T * G / 64 + sh.B) * sh.H_kv : (G + 63) / 64 * sh.H_kv * sh.B;
  return items < device_cu_count() ? 16 : 64;
}

HeadsPlan general_heads_plan(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages) {
  HeadsPlan p;
  p.kernel = HEADS_GENERAL;
  p.n_wg = 0;
  const int G = sh.H / sh.H_kv;
  p.rows = general_rows(sh, T, max_new);
  const int64_t tiles = max_new > 0 ? T * G / p.rows + sh.B : (G + p.rows - 1) / p.rows;
  p.items = tiles * sh.H_kv * (max_new > 0 ? 1 : sh.B);
  p.tiles = (int)(tiles < 2147483647 ? tiles : 2147483647);
  const int64_t tokens = (int64_t)max_pages * sh.page_tokens, want = (4 * (int64_t)device_cu_count() + p.items - 1) / p.items;
  const int64_t most = (tokens + HG_SPLIT - 1) / HG_SPLIT;
  p.n_splits = (int)(want < 1 ? 1 : want < most ? want : most);
  p.slots = p.n_splits > 1 ? p.items * p.n_splits : 0;
  p.workspace = (size_t)p.slots * p.rows * (sh.d_v + 2) * sizeof(float);
  return p;
}

// items * n_splits is below 4 compute units' worth of items and one more split of each, and there are fewer items than that wherever they are split.
size_t general_heads_room(const tpla_heads_t& sh, int64_t T, int32_t max_pages) {
  if ((int64_t)max_pages * sh.page_tokens <= HG_SPLIT) return 0;
  const int64_t fill = 4 * (int64_t)device_cu_count();
  size_t most = 0;
  for (int rows = 16; rows <= 64; rows *= 4) {
    const int64_t items = (T * (sh.H / sh.H_kv) / rows + sh.B) * sh.H_kv, slots = (items < fill ? items : fill) + fill;
    const size_t bytes = (size_t)slots * rows * (sh.d_v + 2) * sizeof(float);
    most = bytes > most ? bytes : most;
  }
  return most;
}

template <typename T, bool JOIN>
static int launch_general(const HeadsArgs& a, const HeadsPlan& p, hipStream_t st) {
  const int nb = ((a.d_k > a.d_v ? a.d_k : a.d_v) + 15) / 16;
  void (*fn)(HeadsArgs) = nullptr;
  int lds = 0;
#define TPLA_WIDTH(N)                                   \
  if (!fn && nb <= N) {                                 \
    fn = heads_general_kernel<T, N, JOIN>;              \
    lds = GeneralTile<N, JOIN>::LDS;                    \
  }
  TPLA_WIDTH(2)
  TPLA_WIDTH(4)
  TPLA_WIDTH(6)
  TPLA_WIDTH(8)
  TPLA_WIDTH(12)
  TPLA_WIDTH(16)
#undef TPLA_WIDTH
  if (!fn) return fail(TPLA_ERR_UNSUPPORTED, "d_k=%d d_v=%d above 256", a.d_k, a.d_v);
  const int rc = allow_lds(reinterpret_cast<const void*>(fn), lds, "heads_general_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3((unsigned)p.items, (unsigned)p.n_splits), dim3(256), lds, st, a);
  return check_launch("heads_general_kernel");
}

int launch_general_heads(const HeadsArgs& a, const HeadsPlan& p, int dtype, hipStream_t st) {
  const bool join = p.rows == 16;
  int rc = dtype == TPLA_F32 ? (join ? launch_general<float, true>(a, p, st) : launch_general<float, false>(a, p, st))
                             : (join ? launch_general<bf16_t, true>(a, p, st) : launch_general<bf16_t, false>(a, p, st));
  if (rc || p.n_splits == 1) return rc;
  void (*fn)(HeadsArgs) = join ? heads_merge_kernel<16, HG_JOIN_TOK> : heads_merge_kernel<64, HG_ROWS_TOK>;
  hipLaunchKernelGGL(fn, dim3((unsigned)p.items, (unsigned)((p.rows * (a.d_v / 4) + 255) / 256)), dim3(256), 0, st, a);
  return check_launch("heads_merge_kernel");
}

}  // namespace tpla
