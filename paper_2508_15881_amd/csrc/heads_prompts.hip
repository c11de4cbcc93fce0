// Causal attention of prompts, or parts of prompts behind cached tokens, over paged keys and values of grouped heads, on the bf16 matrix
// instructions.
//
//   S^T[token, row] = K[token, :] . Q[row, :],   O^T[dim, row] += V^T[dim, token] . P^T[token, row]
//
// The rows of a head of keys are its (new token, query head of the group) pairs, token by token, so that a workgroup's 128 rows are few tokens:
// they share every tile of keys and values, and only the last tiles are cut by the diagonal.  A wave has 32 of them as two blocks of 16; tiles
// go through a ring of four in LDS that direct loads fill.  A lane holds one row per block: the running maximum and sum need two
// exchanges between lanes, and the weights stay in the registers that the scores came in.
#include "heads_tile.h"

#include <algorithm>

namespace tpla {

constexpr int HP_NW = 4, HP_QB = 2, HP_ROWS = HP_NW * HP_QB * 16;
constexpr int HP_NSTAGE = 4;
constexpr int HP_TILE = 8192;            // bytes of keys, and of values, of a tile
constexpr int HP_CPT = HP_TILE / 1024 / HP_NW;   // direct loads per wave, of keys and of values
constexpr int HP_IDS = 1024;             // page ids held at once
constexpr int HP_ODD = HP_NSTAGE * 2 * HP_TILE + HP_IDS * 4;
constexpr int HP_LDS = HP_ODD + (HP_NSTAGE + 1) * 4;
constexpr int HP_CHUNK_MIN = 512;        // tokens of a part of an item at least

// One part of an item: tokens [k0, k1).
struct PromptUnit {
  HeadsItem it;
  int k0, k1, parts, slot;               // slot: that of part 0; part p lies `step` p behind
  int step;
};

// The parts of all items are as long as each other: with few items, what all of them read is divided over a.n_wg workgroups.
struct PromptSeq {
  HeadsItem it;
  int tiles;
};
__device__ __forceinline__ PromptSeq prompt_seq(const HeadsArgs& a, int b) {
  PromptSeq s{};
  if (b >= a.B) return s;
  int first;
  const int n = heads_new(a, b, first);
  s.it.b = b;
  s.it.first = first;
  s.it.rows = n * a.G;
  heads_lens(a, b, n, s.it);
  s.tiles = (s.it.rows + HP_ROWS - 1) / HP_ROWS;
  return s;
}
// Heads of keys are the fastest index: workgroups go to the XCDs in turn, so each XCD's L2 holds the keys and values of few heads.  PARTS: the work
// of an item is split; then tiles follow, then parts.  Otherwise the tiles of a sequence go from its last (most keys) to its first.
// `first_part`: the unit is an item's part 0 and idx counts items alone (the merge).
template <bool PARTS>
__device__ __forceinline__ bool prompt_unit(const HeadsArgs& a, int idx, bool items_only, PromptUnit& u) {
  const int lane = threadIdx.x & 63;
  const int kvh = idx % a.H_kv;
  int at = idx / a.H_kv, before = 0;
  const PromptSeq front = prompt_seq(a, lane);
  int chunk = 0x7fffffff;
  if constexpr (PARTS) {
    double work = (double)front.tiles * front.it.keys;
    for (int b0 = 64; b0 < a.B; b0 += 64) {
      const PromptSeq s = prompt_seq(a, b0 + lane);
      work += (double)s.tiles * s.it.keys;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) work += __shfl_xor(work, d);
    const double per = ceil(work * a.H_kv / a.n_wg);       // (whole numbers below 2^53)
    chunk = __builtin_amdgcn_readfirstlane(per < 1073741824.0 ? max(((int)per + 63) / 64 * 64, HP_CHUNK_MIN) : 0x7fffffff);
  }
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const PromptSeq s = b0 == 0 ? front : prompt_seq(a, b0 + lane);
    const int parts = PARTS ? heads_parts(s.it.keys, chunk) : 1;
    const int units = s.tiles * parts, incl = wave_prefix(units);
    const int count = items_only ? s.tiles : units, count_incl = items_only ? wave_prefix(count) : incl;
    const unsigned long long past = __ballot(count_incl > at);
    if (past == 0) {
      at -= __builtin_amdgcn_readlane(count_incl, 63);
      before += __builtin_amdgcn_readlane(incl, 63);
      continue;
    }
    const int src = __builtin_ctzll(past);
    at -= __builtin_amdgcn_readlane(count_incl - count, src);
    before += __builtin_amdgcn_readlane(incl - units, src);
    const int tiles = __builtin_amdgcn_readlane(s.tiles, src);
    u.it.b = b0 + src;
    u.it.kvh = kvh;
    u.it.first = __builtin_amdgcn_readlane(s.it.first, src);
    u.it.rows = __builtin_amdgcn_readlane(s.it.rows, src);
    u.it.L = __builtin_amdgcn_readlane(s.it.L, src);
    u.it.keys = __builtin_amdgcn_readlane(s.it.keys, src);
    const int part = PARTS ? at / tiles : 0, tile = PARTS ? at - part * tiles : tiles - 1 - at;
    u.it.row0 = tile * HP_ROWS;
    const int keys = max(u.it.sees(min(u.it.row0 + HP_ROWS, u.it.rows) - 1, a.G), 0);
    u.parts = PARTS ? heads_parts(keys, chunk) : 1;
    u.slot = (before + tile) * a.H_kv + kvh;
    u.step = tiles * a.H_kv;
    if (part >= u.parts) return false;
    u.k0 = PARTS ? part * chunk : 0;                   // (part < parts: below keys)
    u.k1 = keys - u.k0 > chunk ? u.k0 + chunk : keys;
    u.slot += part * u.step;
    return true;
  }
  return false;
}

template <int D, bool PARTS>
__global__ void __launch_bounds__(HP_NW * 64, 2) heads_prompts_kernel(HeadsArgs a) {
  constexpr int RC = D / 8, TOK = HP_TILE / (2 * D), TB = TOK / 16, KS = D / 32, DB = D / 16, QB = HP_QB;
  constexpr int LOAD_TOK = 64 / RC;
  static_assert(QB * DB <= 16, "the accumulators are a0 to a63");
  extern __shared__ u32x4 smem[];
  char* const lds = reinterpret_cast<char*>(smem);
  int* const ids = reinterpret_cast<int*>(lds + HP_NSTAGE * 2 * HP_TILE);
  int* const odd_tile = reinterpret_cast<int*>(lds + HP_ODD);      // 1 + the last tile of each place that holds values that are not finite
  int* const first_hole = odd_tile + HP_NSTAGE;                     // first page of those in ids that is missing
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j16 = lane & 15, q4 = lane >> 4;
  PromptUnit u;
  if (!prompt_unit<PARTS>(a, blockIdx.x, false, u)) return;
  const HeadsItem it = u.it;
  const int keys = it.keys;
  if (tid < HP_NSTAGE) odd_tile[tid] = 0;

  // ---- per-lane places ----
  unsigned ld_at[HP_CPT], k_at[KS], v_at[DB];
#pragma unroll
  for (int j = 0; j < HP_CPT; ++j) {
    const int tok = (wave + j * HP_NW) * LOAD_TOK + lane / RC;      // the piece of the row that this lane loads, and the row within the load
    ld_at[j] = (unsigned)((lane / RC) * (2 * D) + ((lane % RC) ^ heads_swz<RC>(tok)) * 16);
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_at[ks] = (j16 * RC + ((4 * ks + q4) ^ heads_swz<RC>(j16))) * 16;
  const int v_tok = 4 * q4 + (j16 >> 2);
#pragma unroll
  for (int d = 0; d < DB; ++d) v_at[d] = HP_TILE + (v_tok * RC + ((2 * d + ((j16 & 3) >> 1)) ^ heads_swz<RC>(v_tok))) * 16 + (j16 & 1) * 8;
  const unsigned lds_base = lds_at(lds);

  const int pt = a.page_tokens, shift = (pt & (pt - 1)) == 0 ? __builtin_ctz(pt) : -1;
  auto page_of = [&](int t) { return shift >= 0 ? t >> shift : t / pt; };
  const size_t page_bytes = (size_t)a.H_kv * pt * (2 * D);
  const int32_t* table = a.table + (size_t)it.b * a.max_pages;
  const char* k_head = static_cast<const char*>(a.k_pool) + (size_t)it.kvh * pt * (2 * D);
  const char* v_head = static_cast<const char*>(a.v_pool) + (size_t)it.kvh * pt * (2 * D);
  int id0 = 0;

  // Tile t on its way.  A load's tokens lie in one page (of a multiple of 16 tokens); ids: their pages.
  auto load_tok = [&](int t, int j) { return t * TOK + (wave + j * HP_NW) * LOAD_TOK; };
  auto issue_whole = [&](int t, const int (&id)[HP_CPT]) {
    char* dst = lds + (t % HP_NSTAGE) * (2 * HP_TILE) + wave * 1024;
    size_t at[HP_CPT];
#pragma unroll
    for (int j = 0; j < HP_CPT; ++j) {
      const int tok = load_tok(t, j);
      at[j] = (size_t)(unsigned)max(__builtin_amdgcn_readfirstlane(id[j]), 0) * page_bytes + (size_t)(tok - page_of(tok) * pt) * (2 * D);
    }
#pragma unroll
    for (int j = 0; j < HP_CPT; ++j)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(k_head + at[j] + ld_at[j]),
                                       (__attribute__((address_space(3))) void*)(dst + j * HP_NW * 1024), 16, 0, 0);
#pragma unroll
    for (int j = 0; j < HP_CPT; ++j)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(v_head + at[j] + ld_at[j]),
                                       (__attribute__((address_space(3))) void*)(dst + HP_TILE + j * HP_NW * 1024), 16, 0, 0);
  };
  // Tokens past the end repeat the last one, those of missing pages are page 0's; they are masked, and their values zeroed.
  auto issue = [&](int t) {
    if ((t + 1) * TOK <= keys) {
      int id[HP_CPT];
#pragma unroll
      for (int j = 0; j < HP_CPT; ++j) id[j] = lds_read_page(ids + (page_of(load_tok(t, j)) - id0));
      issue_whole(t, id);
      return;
    }
    char* dst = lds + (t % HP_NSTAGE) * (2 * HP_TILE) + wave * 1024;
#pragma unroll 1
    for (int j = 0; j < HP_CPT; ++j) {
      const int in_tile = (wave + j * HP_NW) * LOAD_TOK + lane / RC, tok = min(t * TOK + in_tile, keys - 1), p = page_of(tok);
      const int id = max(lds_read_page(ids + (p - id0)), 0);
      const size_t at = (size_t)id * page_bytes + (size_t)(tok - p * pt) * (2 * D) + ((lane % RC) ^ heads_swz<RC>(in_tile)) * 16;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(k_head + at),
                                       (__attribute__((address_space(3))) void*)(dst + j * HP_NW * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(v_head + at),
                                       (__attribute__((address_space(3))) void*)(dst + HP_TILE + j * HP_NW * 1024), 16, 0, 0);
    }
  };
  // The tile t is there, its own loads of the next two tiles may be on their way.
  auto arrived = [&](int t, int c1) {
    if (t + 2 < c1)
      loads_wait<2 * 2 * HP_CPT>();
    else if (t + 1 < c1)
      loads_wait<2 * HP_CPT>();
    else
      loads_wait<0>();
  };

  // ---- this wave's rows ----
  const int row_w = it.row0 + wave * (16 * QB);
  int sees[QB];
#pragma unroll
  for (int r = 0; r < QB; ++r) {
    const int row = row_w + 16 * r + j16;
    sees[r] = row < it.rows ? it.sees(row, a.G) : 0;
  }
  auto out_row = [&](int row) { return (size_t)(it.first + row / a.G) * a.H + it.kvh * a.G + row % a.G; };
  const bool alive = row_w < it.rows;
  const int most = alive ? it.sees(min(row_w + 16 * QB, it.rows) - 1, a.G) : 0;                       // tokens that some row of the wave sees
  const int least = it.sees(it.row0, a.G);                                                            // and that all rows of the workgroup see

  bf16x8 q[QB][KS];
  float m[QB], l[QB];
  int seen[QB];
#pragma unroll
  for (int r = 0; r < QB; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
    seen[r] = 0;
  }
  out_keep();
  static_for<QB * DB>([&](auto ic) { out_write<decltype(ic)::value>(f32x4{0.f, 0.f, 0.f, 0.f}); });

  // ---- one tile.  CUT: some of its tokens are not seen by some rows; there: its blocks of 16 tokens that have a page ----
  auto tile_body = [&](int t, int there, auto cut_tag) {
    constexpr bool CUT = decltype(cut_tag)::value;
    const int tok0 = t * TOK;
    const unsigned base = lds_base + (unsigned)((t % HP_NSTAGE) * (2 * HP_TILE));
    f32x4 s[QB][TB];
    {
      constexpr int N = KS * TB, AHEAD = D == 128 ? 8 : 4;
      bf16x8 kf[AHEAD];
      static_for<AHEAD>([&](auto ic) {
        constexpr int x = decltype(ic)::value;
        lds_read_b128<(x % TB) * (16 * RC * 16)>(kf[x], base + k_at[x / TB]);
      });
      static_for<N>([&](auto ic) {
        constexpr int x = decltype(ic)::value, ks = x / TB, n = x % TB;
        lds_wait<(N - 1 - x < AHEAD - 1 ? N - 1 - x : AHEAD - 1)>(kf[x % AHEAD]);
#pragma unroll
        for (int r = 0; r < QB; ++r) {
          if constexpr (ks == 0)
            score_first(s[r][n], kf[x % AHEAD], q[r][ks]);
          else
            score_more(s[r][n], kf[x % AHEAD], q[r][ks]);
        }
        if constexpr (x + AHEAD < N) lds_read_b128<((x + AHEAD) % TB) * (16 * RC * 16)>(kf[x % AHEAD], base + k_at[(x + AHEAD) / TB]);
      });
    }
    // the first values start now, so that their way from LDS passes under the softmax
    constexpr int NV = DB * (TB / 2), VA = 4;
    u32x2 lo[VA], hi[VA];
    auto value = [&](auto yc) {
      constexpr int y = decltype(yc)::value;
      lds_read_tr_b64<(y / DB) * (32 * RC * 16)>(lo[y % VA], base + v_at[y % DB]);
      lds_read_tr_b64<(y / DB) * (32 * RC * 16) + 16 * RC * 16>(hi[y % VA], base + v_at[y % DB]);
    };
    if constexpr (!CUT) static_for<VA>([&](auto ic) { value(ic); });
    out_settle_result();
#pragma unroll
    for (int r = 0; r < QB; ++r)
#pragma unroll
      for (int n = 0; n < TB; ++n) settle_scores(s[r][n]);

    bf16x8 p[QB][TB / 2];
    static_for<QB>([&](auto rc) {
      constexpr int r = decltype(rc)::value;
      if constexpr (CUT) {
#pragma unroll
        for (int n = 0; n < TB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool vis = ((there >> n) & 1) && tok0 + 16 * n + 4 * q4 + i < sees[r];
            seen[r] |= vis;
            if (!vis) s[r][n][i] = -INFINITY;
          }
      }
      float top = s[r][0][0];
#pragma unroll
      for (int n = 0; n < TB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][n][i]);
      top *= a.scale_log2;
      if (__any(top > m[r] + LAZY)) {
        top = fmaxf(top, lane_xor<16>(top, lane));
        top = fmaxf(top, lane_xor<32>(top, lane));
        const float m_new = fmaxf(m[r], top);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[r] - m_new);
        l[r] *= alpha;
        m[r] = m_new;
        out_settle_result();
        static_for<DB>([&](auto dc) { out_scale<r * DB + decltype(dc)::value>(alpha); });
      }
      const float ref = m[r] == -INFINITY ? 0.f : m[r];
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < TB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[r][n][i], a.scale_log2, -ref));
          sum[i] += e;
          p[r][n / 2][4 * (n & 1) + i] = (bf16_t)e;
        }
      l[r] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    });

#pragma unroll
    for (int r = 0; r < QB; ++r)
#pragma unroll
      for (int h = 0; h < TB / 2; ++h) settle_weights(p[r][h]);
    bool odd = false;
    if constexpr (CUT) odd = __builtin_amdgcn_readfirstlane(lds_read_page(odd_tile + t % HP_NSTAGE)) == t + 1;
    if (!odd) {
      if constexpr (CUT) static_for<VA>([&](auto ic) { value(ic); });
      static_for<NV>([&](auto ic) {
        constexpr int x = decltype(ic)::value, d = x % DB, h = x / DB, ahead = NV - 1 - x < VA - 1 ? NV - 1 - x : VA - 1;
        lds_wait<2 * ahead>(lo[x % VA], hi[x % VA]);
        const u32x4 v = {lo[x % VA][0], lo[x % VA][1], hi[x % VA][0], hi[x % VA][1]};
        static_for<QB>([&](auto rc) { out_product<decltype(rc)::value * DB + d>(v, p[decltype(rc)::value][h]); });
        if constexpr (x + VA < NV) value(std::integral_constant<int, x + VA>{});
      });
    } else {
      // A weight of zero does not silence what is not finite: one token at a time, kept by the rows that see it.
      out_settle_result();
#pragma unroll 1
      for (int tok = 0; tok < TOK; ++tok) {
        const unsigned h = tok >> 5;
        const u32x4 keep = keep_token(tok, q4);
        out_keep();
        static_for<DB>([&](auto dc) {
          constexpr int d = decltype(dc)::value;
          u32x2 vlo, vhi;
          lds_read_tr_b64<0>(vlo, base + v_at[d] + h * (32 * RC * 16));
          lds_read_tr_b64<16 * RC * 16>(vhi, base + v_at[d] + h * (32 * RC * 16));
          lds_wait<0>(vlo, vhi);
          bf16x8 v = __builtin_bit_cast(bf16x8, u32x4{vlo[0], vlo[1], vhi[0], vhi[1]} & keep);
          settle_weights(v);
          static_for<QB>([&](auto rc) {
            constexpr int r = decltype(rc)::value;
            u32x4 w = __builtin_bit_cast(u32x4, p[r][0]);
            if constexpr (TB == 4) w = (w & (h - 1u)) | (__builtin_bit_cast(u32x4, p[r][1]) & (0u - h));
            const f32x4 was = out_read<r * DB + d>();
            bf16x8 one = __builtin_bit_cast(bf16x8, w & keep);
            f32x4 x = was;
            settle_scores(x);
            settle_weights(one);
            score_more(x, v, one);
            out_settle_result();
            settle_scores(x);
            const bool vis = ((there >> (tok >> 4)) & 1) && tok0 + tok < sees[r];
            out_write<r * DB + d>(vis ? x : was);
          });
        });
      }
      out_settle_write();
    }
  };

  const int t0 = u.k0 / TOK, t1 = (u.k1 + TOK - 1) / TOK;
  const int id_tiles = (int)min(max((long long)(HP_IDS - 1) * pt / TOK, 1ll), 1ll << 26);           // tiles whose pages fit in ids, wherever in a page they begin
  for (int c0 = t0; c0 < t1; c0 += id_tiles) {
    const int c1 = min(t1, c0 + id_tiles);
    __syncthreads();
    id0 = page_of(c0 * TOK);
    if (tid == 0) *first_hole = 0x7fffffff;
    __syncthreads();
    for (int x = tid; x < HP_IDS; x += HP_NW * 64) {
      const int p = id0 + x;
      if (p < a.max_pages && (long long)p * pt < (long long)min(keys, c1 * TOK)) {
        const int id = table[p];
        ids[x] = id;
        if (id < 0) atomicMin(first_hole, p);
      }
    }
    __syncthreads();
    // tiles that exist whole and that every row of the workgroup sees
    const int hole = __builtin_amdgcn_readfirstlane(*first_hole), plain = hole == 0x7fffffff ? least : min(least, hole * pt);
    const int whole = min(c1, max(c0, plain / TOK));
    for (int t = c0; t < min(c1, c0 + HP_NSTAGE - 1); ++t) issue(t);
    if (c0 == t0) {
#pragma unroll
      for (int r = 0; r < QB; ++r)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          q[r][ks] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16_t*>(a.q) + out_row(min(row_w + 16 * r + j16, it.rows - 1)) * D + 32 * ks + 8 * q4);
#pragma unroll
      for (int r = 0; r < QB; ++r)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[r][ks]));       // complete before the loop
    }
    int t = c0;
    // the page ids of the tile that is requested next, read a tile ahead
    const int last_id = page_of(max(min(keys, c1 * TOK) - 1, 0)) - id0;
    int id[HP_CPT];
#pragma unroll
    for (int j = 0; j < HP_CPT; ++j) id[j] = lds_read_page(ids + min(page_of(load_tok(t + HP_NSTAGE - 1, j)) - id0, last_id));
    for (; t < whole; ++t) {
      out_keep();
      arrived(t, c1);
      __builtin_amdgcn_s_barrier();                    // tile t is there for all waves, tile t - 1 is no longer read
      asm volatile("" ::: "memory");
      const int next = t + HP_NSTAGE - 1;
      if (next < c1) {
        if ((next + 1) * TOK <= keys)
          issue_whole(next, id);
        else
          issue(next);
      }
#pragma unroll
      for (int j = 0; j < HP_CPT; ++j) lds_request_page(id[j], ids + min(page_of(load_tok(next + 1, j)) - id0, last_id));
      if (alive) tile_body(t, 0, std::false_type{});
#pragma unroll
      for (int j = 0; j < HP_CPT; ++j) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(id[j]) : : "memory");      // (long there)
    }
    if (whole > t0) seen[0] = seen[1] = 1;
    for (; t < c1; ++t) {
      out_keep();
      arrived(t, c1);
      const int tok0 = t * TOK;
      int there = 0;
#pragma unroll
      for (int n = 0; n < TB; ++n)
        if (tok0 + 16 * n < keys && __builtin_amdgcn_readfirstlane(lds_read_page(ids + (page_of(tok0 + 16 * n) - id0))) >= 0) there |= 1 << n;
      // what this wave has loaded: rows that are no tokens become zeros; values that are not finite, which some rows may not see
      char* mine = lds + (t % HP_NSTAGE) * (2 * HP_TILE) + HP_TILE + wave * 1024 + lane * 16;
#pragma unroll
      for (int j = 0; j < HP_CPT; ++j) {
        const int in_tile = (wave + j * HP_NW) * LOAD_TOK + lane / RC;
        u32x4* piece = reinterpret_cast<u32x4*>(mine + j * HP_NW * 1024);
        if (tok0 + in_tile >= keys || !((there >> (in_tile >> 4)) & 1)) {
          *piece = u32x4{0u, 0u, 0u, 0u};
        } else {
          const u32x4 v = *piece;
          if (not_finite_pair(v[0]) || not_finite_pair(v[1]) || not_finite_pair(v[2]) || not_finite_pair(v[3])) odd_tile[t % HP_NSTAGE] = t + 1;
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (t + HP_NSTAGE - 1 < c1) issue(t + HP_NSTAGE - 1);
      if (tok0 >= most) continue;                      // (the wave's rows see none of it; the barriers above are still reached)
      tile_body(t, there, std::true_type{});
    }
  }
  if (!alive) return;
  out_settle_result();
  static_for<QB>([&](auto rc) {
    constexpr int r = decltype(rc)::value;
    l[r] += lane_xor<16>(l[r], lane);
    l[r] += lane_xor<32>(l[r], lane);
    int any = seen[r];
    any |= __shfl_xor(any, 16);
    any |= __shfl_xor(any, 32);
    heads_close(m[r], l[r], any);
    int j = j16;
    asm volatile("" : "+v"(j));                        // (made here: nothing of it is kept over the loops)
    const int row = row_w + 16 * r + j;
    const bool written = row < it.rows;
    const float inv = heads_inverse(l[r]);
    const size_t out = out_row(min(row, it.rows - 1));
    const size_t at = (size_t)u.slot * HP_ROWS + (row - it.row0);
    static_for<DB>([&](auto dc) {
      constexpr int d = decltype(dc)::value;
      const f32x4 x = out_read<r * DB + d>();
      if (!written) return;
      if (u.parts == 1)
        store4(a.o, out * D + 16 * d + 4 * q4, a.o_dtype, l[r] == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : x * inv);
      else
        *reinterpret_cast<f32x4*>(a.part_acc + at * D + 16 * d + 4 * q4) = x;
    });
    if (written && q4 == 0) {
      if (u.parts > 1)
        *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m[r], l[r]);
      else if (a.lse)
        a.lse[out] = heads_lse(m[r], l[r]);
    }
  });
}

// grid: (items, groups of 256 / (D / 4) rows).  The parts of a row in their order, a thread for four columns.
template <int D>
__global__ void __launch_bounds__(256) heads_prompts_merge_kernel(HeadsArgs a) {
  constexpr int LPR = D / 4, AT_ONCE = 256 / LPR;
  PromptUnit u;
  if (!prompt_unit<true>(a, blockIdx.x, true, u) || u.parts == 1) return;
  const int r = blockIdx.y * AT_ONCE + threadIdx.x / LPR, c = 4 * (threadIdx.x % LPR), row = u.it.row0 + r;
  if (row >= u.it.rows) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  auto at = [&](int p) { return (size_t)(u.slot + p * u.step) * HP_ROWS + r; };
  float M = -INFINITY, sum = 0.f;
  for (int p = 0; p < u.parts; ++p) M = fmaxf(M, ml[at(p)].x);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < u.parts; ++p) {
    const float2 part = ml[at(p)];
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_acc + at(p) * D + c);
    const float by = heads_join(M, part, sum);
    if (part.x != -INFINITY) o += x * by;
  }
  const size_t out = (size_t)(u.it.first + row / a.G) * a.H + u.it.kvh * a.G + row % a.G;
  const float inv = heads_inverse(sum);
  store4(a.o, out * D + c, a.o_dtype, sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv);
  if (a.lse && c == 0) a.lse[out] = heads_lse(M, sum);
}

static int64_t prompts_items(const tpla_heads_t& sh, int64_t T) { return (T * (sh.H / sh.H_kv) / HP_ROWS + sh.B) * sh.H_kv; }

HeadsPlan heads_prompts_plan(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages) {
  HeadsPlan p;
  p.kernel = HEADS_PROMPTS;
  p.rows = HP_ROWS;
  p.items = prompts_items(sh, T);
  p.tiles = (int)(p.items / sh.H_kv);
  p.n_wg = 2 * device_cu_count();                      // workgroups that the chip holds
  // Split where the items do not fill it twice and there are tokens to split.
  p.n_splits = p.items < 2 * p.n_wg && (int64_t)max_pages * sh.page_tokens > HP_CHUNK_MIN ? 2 : 1;
  p.slots = p.n_splits > 1 ? p.items + p.n_wg : 0;     // (the parts of an item: what it reads over the chunk's length, rounded up)
  p.workspace = (size_t)p.slots * p.rows * (sh.d_v + 2) * sizeof(float);
  return p;
}

size_t heads_prompts_room(const tpla_heads_t& sh, int64_t T, int32_t max_pages) {
  if ((int64_t)max_pages * sh.page_tokens <= HP_CHUNK_MIN) return 0;
  const int64_t n_wg = 2 * device_cu_count();
  return (size_t)(std::min(prompts_items(sh, T), 2 * n_wg) + n_wg) * HP_ROWS * (sh.d_v + 2) * sizeof(float);
}

int launch_heads_prompts(const HeadsArgs& a, const HeadsPlan& p, hipStream_t st) {
  const bool parts = p.n_splits > 1;
  void (*fn)(HeadsArgs) = a.d_k == 128 ? (parts ? heads_prompts_kernel<128, true> : heads_prompts_kernel<128, false>)
                                       : (parts ? heads_prompts_kernel<64, true> : heads_prompts_kernel<64, false>);
  int rc = allow_lds(reinterpret_cast<const void*>(fn), HP_LDS, "heads_prompts_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3((unsigned)(parts ? p.slots : p.items)), dim3(HP_NW * 64), HP_LDS, st, a);
  if ((rc = check_launch("heads_prompts_kernel")) || !parts) return rc;
  const int rows = 256 / (a.d_k / 4);
  hipLaunchKernelGGL(a.d_k == 128 ? heads_prompts_merge_kernel<128> : heads_prompts_merge_kernel<64>, dim3((unsigned)p.items, HP_ROWS / rows), dim3(256), 0,
                     st, a);
  return check_launch("heads_prompts_merge_kernel");
}

}  // namespace tpla
