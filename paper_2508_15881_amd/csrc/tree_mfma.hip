// Attention of drafted tokens on the matrix cores: bf16, slices of 64, 128, 256 or 512 columns, 64 of RoPE key.
//
// The T H rows of a (slice, sequence) all read the same cache rows, so the rows are the MFMA N dimension and a tile of 32 tokens
// is shared by everything the workgroup holds:
//   S^T[token, row] = K[token, :] . Q[row, :]           M = tokens (LDS), N = rows (Q in registers for the whole item)
//   O^T[dim, row]  += V^T[dim, token] . P^T[token, row]  V = the first dl columns of the same LDS rows, read transposed
// A workgroup is 4 waves of RB blocks of 16 rows.  Every wave reads the whole tile from LDS, and a fragment it reads feeds RB
// MFMAs: RB decides how far LDS (128 bytes a clock) keeps up with the matrix cores.
//
// All 32-token tiles of all items (slice, sequence, row block) are laid end to end and cut into equal ranges, one per workgroup;
// an item that lies in one range is written at once, the others leave partial results for the merge (tree.hip).
#include "lds_tile.h"

#include <algorithm>

namespace tpla {

constexpr int TR_TOK = 32;           // tokens per tile
constexpr int TR_NW = 4;
// Page ids in LDS: chunks of 256 in a ring of 4.  A chunk is a whole number of tiles, at least 8, whatever the page size.  The
// first tile of a chunk to be requested requests the ids of the next one: at most NSTAGE - 1 tiles are requested between two
// barriers, so what is overwritten (three chunks back) is read by nobody, and the ids have arrived when 8 tiles later the
// first of them is read (the wait for the tile after the request covers them).
constexpr int TR_IDS = 256, TR_ID_RING = 4 * TR_IDS;

template <int DL>
struct TreeTile {
  static constexpr int RC = (DL + 64) / 8;             // 16-byte pieces per row
  static constexpr int BYTES = TR_TOK * RC * 16;
  static constexpr int CPT = TR_TOK * RC / 64 / TR_NW;  // direct-to-LDS loads per wave and tile
  // Tiles in flight or in use; at most 8 (see TR_IDS).
  static constexpr int NSTAGE = 150 * 1024 / BYTES < 8 ? 150 * 1024 / BYTES : 8;
  static constexpr int LDS = NSTAGE * BYTES + TR_ID_RING * 4;
  static_assert(TR_TOK * RC % (64 * TR_NW) == 0, "every wave issues the same number of loads");
};

__host__ __device__ __forceinline__ int tree_start(int n_wg, int units, int w) { return (int)((double)w * (double)units / (double)n_wg); }
// The last workgroup whose range begins at or before unit u.  Exact: the products stay below 2^53 and a quotient that is not a
// whole number is further from one than its rounding.
__host__ __device__ __forceinline__ int tree_owner(int n_wg, int units, int u) {
  return (int)((((double)u + 1.0) * (double)n_wg - 1.0) / (double)units);
}

__device__ __forceinline__ int tree_prefix(int v) {      // inclusive sum over the wave
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}
// Units (tiles) of sequence b: row blocks x tiles; none without drafts.
__device__ __forceinline__ int tree_units(const TreeArgs& a, int b, int* tiles) {
  if (b >= a.B) return *tiles = 0;
  const TreeLens len = tree_lens(a, b);
  *tiles = len.n > 0 ? max((len.keys + TR_TOK - 1) / TR_TOK, 1) : 0;
  return *tiles * ((len.n * a.H + a.p.block - 1) / a.p.block);
}

template <int DL, int RB>
__global__ void __launch_bounds__(TR_NW * 64, 1) tree_mfma_kernel(TreeArgs a) {
  using Tile = TreeTile<DL>;
  constexpr int RC = Tile::RC, CPT = Tile::CPT, NSTAGE = Tile::NSTAGE;
  constexpr int KS = (DL + 64) / 32, DB = DL / 16;
  constexpr int KRING = 8, VRING = 4;
  extern __shared__ u32x4 smem[];
  const unsigned lds_base = lds_at(reinterpret_cast<const char*>(smem));
  const unsigned lds_ids = lds_base + NSTAGE * Tile::BYTES;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j16 = lane & 15, q4 = lane >> 4;

  // ---- this workgroup's range of units ----
  int per_slice = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int tiles;
    per_slice += __builtin_amdgcn_readlane(tree_prefix(tree_units(a, b0 + lane, &tiles)), 63);
  }
  const int units = per_slice * a.n_shards;
  const int n_wg = max(1, min(a.p.n_wg, units / a.p.split_tokens));     // no shorter ranges than pay
  const int w = n_wg % 8 == 0 ? (blockIdx.x & 7) * (n_wg >> 3) + (blockIdx.x >> 3) : blockIdx.x;
  if ((int)blockIdx.x >= n_wg || units == 0) return;
  int pos = tree_start(n_wg, units, w);
  const int range0 = pos, end = tree_start(n_wg, units, w + 1);

  // ---- per-lane LDS offsets (as in the prefill kernel) ----
  const int xk = swz(j16);
  unsigned k_off[2];
  k_off[0] = (unsigned)((j16 * RC + (q4 ^ xk)) * 16);
  k_off[1] = (unsigned)((j16 * RC + ((4 | q4) ^ xk)) * 16);
  const int v_tok = 4 * q4 + (j16 >> 2), xv = swz(v_tok), cb = (j16 & 3) >> 1;
  unsigned v_off[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) v_off[d] = (unsigned)((v_tok * RC + (((d << 1) | cb) ^ xv)) * 16 + (j16 & 1) * 8);
  int ld_tok[CPT], ld_byte[CPT];
#pragma unroll
  for (int j = 0; j < CPT; ++j) {
    const int x = (wave + j * TR_NW) * 64 + lane;
    ld_tok[j] = x / RC;
    ld_byte[j] = ((x % RC) ^ swz(ld_tok[j])) * 16;
  }
  const int pt = a.page_tokens, shift = (pt & (pt - 1)) == 0 ? __builtin_ctz(pt) : -1;
  auto page_of = [&](int t) { return shift >= 0 ? t >> shift : t / pt; };

  while (pos < end) {
    // ---- the item of unit `pos` ----
    const int i = pos / per_slice, rem = pos - i * per_slice;
    int b = 0, before = 0, tiles = 1;
    for (int b0 = 0, base = 0; b0 < a.B; b0 += 64) {
      int t_b;
      const int u = tree_units(a, b0 + lane, &t_b), incl = tree_prefix(u) + base;
      const unsigned long long past = __ballot(incl > rem);
      if (past) {
        const int src = __builtin_ctzll(past);
        b = b0 + src;
        before = __builtin_amdgcn_readlane(incl - u, src);
        tiles = __builtin_amdgcn_readlane(t_b, src);
        break;
      }
      base = __builtin_amdgcn_readlane(incl, 63);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    const int rb = (rem - before) / tiles, t0 = rem - before - rb * tiles, t1 = min(tiles, t0 + (end - pos));
    const TreeLens len = tree_lens(a, b);
    const int L = __builtin_amdgcn_readfirstlane(len.L), keys = __builtin_amdgcn_readfirstlane(len.keys);
    const int rows = __builtin_amdgcn_readfirstlane(len.n) * a.H;
    const int v = i * a.B + b, item = v * a.p.blocks + rb;
    const int row0 = rb * a.p.block + wave * (16 * RB);          // this wave's first row
    const bool alive = row0 < rows;
    const int all_rows = a.T * a.H;
    const char* pool = static_cast<const char*>(i == 0 ? a.pools[0] : i == 1 ? a.pools[1] : i == 2 ? a.pools[2] : i == 3 ? a.pools[3] :
                                                i == 4 ? a.pools[4] : i == 5 ? a.pools[5] : i == 6 ? a.pools[6] : a.pools[7]);
    const int32_t* table = a.block_table + (size_t)b * a.max_pages;

    // ---- page ids and tiles on their way ----
    int chunk = page_of(t0 * TR_TOK) / TR_IDS;
    auto request_ids = [&](int c) {
      const int p = min(c * TR_IDS + wave * 64 + lane, a.max_pages - 1);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(table + p),
                                       (__attribute__((address_space(3))) void*)(reinterpret_cast<char*>(smem) + NSTAGE * Tile::BYTES +
                                                                                 ((c & 3) * TR_IDS + wave * 64) * 4), 4, 0, 0);
    };
    auto issue = [&](int t) {
      const int c = __builtin_amdgcn_readfirstlane(page_of(t * TR_TOK)) / TR_IDS;
      int page[CPT], off[CPT];
#pragma unroll
      for (int j = 0; j < CPT; ++j) {
        const int k = min(t * TR_TOK + ld_tok[j], keys - 1), p = page_of(k);
        off[j] = k - p * pt;
        const unsigned at = lds_ids + (unsigned)(p & (TR_ID_RING - 1)) * 4;
        asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(page[j]) : "v"(at) : "memory");
      }
      char* dst = reinterpret_cast<char*>(smem) + (t % NSTAGE) * Tile::BYTES;
#pragma unroll
      for (int j = 0; j < CPT; ++j) {
        const char* src = pool + ((size_t)page[j] * pt + off[j]) * (RC * 16) + ld_byte[j];
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                         (__attribute__((address_space(3))) void*)(dst + (wave + j * TR_NW) * 1024), 16, 0, 0);
      }
      if (c != chunk) {
        chunk = c;
        request_ids(c + 1);
      }
    };
    lds_barrier();                                   // the item before this one no longer reads LDS
    request_ids(chunk);
    request_ids(chunk + 1);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __builtin_amdgcn_s_barrier();
    for (int t = t0; t < t1 && t < t0 + NSTAGE - 1; ++t) issue(t);

    // ---- queries as B operands: block r, lane holds row row0 + 16 r + j16 ----
    bf16x8 q[RB][KS];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const int row = min(row0 + 16 * r + j16, rows - 1);
      const bf16_t* ql = static_cast<const bf16_t*>(a.q_lat) + ((size_t)v * all_rows + row) * DL;
      const bf16_t* qp = static_cast<const bf16_t*>(a.q_pe) + ((size_t)b * all_rows + row) * 64;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int k0 = ks * 32 + q4 * 8;
        q[r][ks] = *reinterpret_cast<const bf16x8*>(ks * 32 < DL ? ql + k0 : qp + (k0 - DL));
      }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[r][ks]));   // complete before the loop

    f32x4 acc[RB][DB];
    float m_run[RB], l_run[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      m_run[r] = -INFINITY;
      l_run[r] = 0.f;
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    for (int t = t0; t < t1; ++t) {
      if (t + NSTAGE - 2 < t1)
        __builtin_amdgcn_s_waitcnt(vmcnt_imm((NSTAGE - 2) * CPT));
      else
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __builtin_amdgcn_s_barrier();                  // tile t visible to all waves, tile t - 1 no longer read
      if (t + NSTAGE - 1 < t1) issue(t + NSTAGE - 1);
      const unsigned tile = lds_base + (unsigned)((t % NSTAGE) * Tile::BYTES);
      const bool tail = (t + 1) * TR_TOK > L;        // drafts, or past the end

      f32x4 s[RB][2];
      if (alive) {
#pragma unroll
        for (int r = 0; r < RB; ++r) s[r][0] = s[r][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int NQ = KS * 2;                   // K fragments, in order (ks, tb)
        bf16x8 kf[KRING];
        const unsigned ka[2] = {tile + k_off[0], tile + k_off[1]};
        static_for<KRING>([&](auto ic) {
          constexpr int x = decltype(ic)::value, ks = x / 2, tb = x % 2;
          lds_read_b128<(ks >> 1) * 128 + tb * (16 * RC * 16)>(kf[x], ka[ks & 1]);
        });
        static_for<NQ>([&](auto ic) {
          constexpr int x = decltype(ic)::value, ks = x / 2, tb = x % 2;
          constexpr int ahead = (NQ - 1 - x) < KRING - 1 ? (NQ - 1 - x) : KRING - 1;
          lds_wait<ahead>(kf[x % KRING]);
#pragma unroll
          for (int r = 0; r < RB; ++r) s[r][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[x % KRING], q[r][ks], s[r][tb], 0, 0, 0);
          if constexpr (x + KRING < NQ) {
            constexpr int ks2 = (x + KRING) / 2, tb2 = (x + KRING) % 2;
            lds_read_b128<(ks2 >> 1) * 128 + tb2 * (16 * RC * 16)>(kf[x % KRING], ka[ks2 & 1]);
          }
        });
      }
      if (tail) {
        // Values of drafts are masked per row, and a weight of zero does not silence an infinity or a NaN: what is not finite
        // becomes zero here, behind the scores.  A row that sees such a draft has it in its score already.
        lds_barrier();
        for (int x = tid; x < TR_TOK * RC; x += TR_NW * 64) {
          const int tok = x / RC, c = (x % RC) ^ swz(tok);
          if (c >= DL / 8 || t * TR_TOK + tok < L) continue;
          u32x4* at = smem + (t % NSTAGE) * (TR_TOK * RC) + x;
          u32x4 u = *at;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((u[e] & 0x7F80u) == 0x7F80u) u[e] &= 0xFFFF0000u;
            if ((u[e] & 0x7F800000u) == 0x7F800000u) u[e] &= 0xFFFFu;
          }
          *at = u;
        }
        lds_barrier();
      }
      if (!alive) continue;

      // the first V fragments start now: their LDS latency passes under the softmax arithmetic
      u32x2 vlo[VRING], vhi[VRING];
      unsigned va[4];
#pragma unroll
      for (int d = 0; d < 4; ++d) va[d] = tile + v_off[d];
      static_for<VRING>([&](auto ic) {
        constexpr int d = decltype(ic)::value;
        lds_read_tr_b64<(d >> 2) * 128>(vlo[d], va[d & 3]);
        lds_read_tr_b64<(d >> 2) * 128 + 16 * RC * 16>(vhi[d], va[d & 3]);
      });

      // ---- online softmax: lane = one row per block, tokens 32 t + 16 tb + 4 q4 + e ----
      bf16x8 pb[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        if (tail) {
          const int row = min(row0 + 16 * r + j16, rows - 1);
          const unsigned long long bits = a.mask[(size_t)b * a.T + row / a.H];
#pragma unroll
          for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = t * TR_TOK + 16 * tb + 4 * q4 + e, j = k - L;
              if (j >= 0 && (k >= keys || !((bits >> (j & 63)) & 1))) s[r][tb][e] = -INFINITY;
            }
        }
        float mx = s[r][0][0];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[r][tb][e]);
        mx *= a.scale_log2;
        if (__any(mx > m_run[r] + LAZY)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float m_new = fmaxf(m_run[r], mx);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[r] - m_new);   // 0 the first time
          l_run[r] *= alpha;
          m_run[r] = m_new;
#pragma unroll
          for (int d = 0; d < DB; ++d) acc[r][d] *= alpha;
        }
        const float ref = m_run[r] == -INFINITY ? 0.f : m_run[r];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[r][tb][e], a.scale_log2, -ref));
            l_run[r] += p;
            // weights go into the second product in bf16, at most 2^-9 off each; their sum is that of the unrounded ones, so
            // that lse has float accuracy
            pb[r][4 * tb + e] = (bf16_t)p;
          }
      }

      // ---- O^T += V^T P^T ----
      static_for<DB>([&](auto ic) {
        constexpr int d = decltype(ic)::value;
        constexpr int ahead = (DB - 1 - d) < VRING - 1 ? (DB - 1 - d) : VRING - 1;
        lds_wait<2 * ahead>(vlo[d % VRING], vhi[d % VRING]);
        const u32x4 v4 = {vlo[d % VRING][0], vlo[d % VRING][1], vhi[d % VRING][0], vhi[d % VRING][1]};
#pragma unroll
        for (int r = 0; r < RB; ++r)
          acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v4), pb[r], acc[r][d], 0, 0, 0);
        if constexpr (d + VRING < DB) {
          constexpr int d2 = d + VRING;
          lds_read_tr_b64<(d2 >> 2) * 128>(vlo[d % VRING], va[d2 & 3]);
          lds_read_tr_b64<(d2 >> 2) * 128 + 16 * RC * 16>(vhi[d % VRING], va[d2 & 3]);
        }
      });
    }

    // ---- the item's result, or a partial one ----
    const bool whole = t0 == 0 && t1 == tiles;
    const int slot = 2 * w + (pos == range0 ? 0 : 1);
    if (t0 == 0 && tid == 0) {
      const int last = tree_owner(n_wg, units, pos + tiles - 1);
      a.plan[3 * item] = w;
      a.plan[3 * item + 1] = last - w + 1;
      a.plan[3 * item + 2] = pos == range0 ? 0 : 1;
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const int local = wave * (16 * RB) + 16 * r + j16, row = row0 + 16 * r + j16;
      float l = l_run[r];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (!alive || row >= rows) continue;
      const float inv = whole ? (l != 0.f ? 1.0f / l : 0.f) : 1.f;
      float* out = whole ? a.o_lat + ((size_t)v * all_rows + row) * DL : a.part_acc + ((size_t)slot * a.p.block + local) * DL;
#pragma unroll
      for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(out + 16 * d + 4 * q4) = acc[r][d] * inv;
      if (q4 == 0) {
        if (!whole)
          *reinterpret_cast<float2*>(a.part_ml + 2 * ((size_t)slot * a.p.block + local)) = make_float2(m_run[r], l);
        else if (a.lse)
          a.lse[(size_t)v * all_rows + row] = l != 0.f ? (m_run[r] + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
    }
    pos += t1 - t0;
  }
}

bool tree_mfma_supported(const tpla_shape_t& sh) {
  const int dl = sh.d_c / sh.g;
  return sh.dtype == TPLA_BF16 && sh.d_r == 64 && (dl == 64 || dl == 128 || dl == 256 || dl == 512);
}

// Blocks of 16 rows per wave.
static int row_blocks(int dl, int rows) {
  const int most = dl == 512 ? 1 : dl == 64 ? 4 : 2;
  int best = 1;
  double least = 1e30;
  for (int rb = 1; rb <= most; ++rb) {
    if (rb == 3) continue;
    const double t = (double)((rows + 64 * rb - 1) / (64 * rb)) * (1.0 + 0.35 * rb);
    if (t < least) {
      least = t;
      best = rb;
    }
  }
  return best;
}

void tree_mfma_plan(const tpla_shape_t& sh, int n_shards, int T, int max_pages, TreePlan* p) {
  const int dl = sh.d_c / sh.g;
  p->mfma = 1;
  p->block = 64 * row_blocks(dl, T * sh.H);
  p->blocks = (T * sh.H + p->block - 1) / p->block;
  const double tiles = ((double)max_pages * sh.page_tokens + TR_TOK - 1) / TR_TOK;
  const double most = (double)n_shards * sh.B * p->blocks * std::max(tiles, 1.0);
  p->n_wg = (int)std::min((double)device_cu_count(), most);
  p->n_splits = 1;
  p->split_tokens = 8;         // fewest tiles of a range
}

template <int DL, int RB>
static int launch_tree(const TreeArgs& a, hipStream_t st) {
  const auto fn = tree_mfma_kernel<DL, RB>;
  const int rc = allow_lds(reinterpret_cast<const void*>(fn), TreeTile<DL>::LDS, "tree_mfma_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3(a.p.n_wg), dim3(TR_NW * 64), TreeTile<DL>::LDS, st, a);
  return check_launch("tree_mfma_kernel");
}

int launch_tree_mfma(const TreeArgs& a, hipStream_t st) {
  switch (a.dl * 8 + a.p.block / 64) {
    case 64 * 8 + 1: return launch_tree<64, 1>(a, st);
    case 64 * 8 + 2: return launch_tree<64, 2>(a, st);
    case 64 * 8 + 4: return launch_tree<64, 4>(a, st);
    case 128 * 8 + 1: return launch_tree<128, 1>(a, st);
    case 128 * 8 + 2: return launch_tree<128, 2>(a, st);
    case 256 * 8 + 1: return launch_tree<256, 1>(a, st);
    case 256 * 8 + 2: return launch_tree<256, 2>(a, st);
    case 512 * 8 + 1: return launch_tree<512, 1>(a, st);
  }
  return fail(TPLA_ERR_UNSUPPORTED, "no kernel for slices of %d columns in blocks of %d rows", a.dl, a.p.block);
}

}  // namespace tpla
