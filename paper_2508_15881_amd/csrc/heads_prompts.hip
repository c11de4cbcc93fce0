// Causal attention of prompts, or parts of prompts behind cached tokens, over paged keys and values of grouped heads, on the bf16 matrix
// instructions.
//
//   S^T[token, row] = K[token, :] . Q[row, :],   O^T[dim, row] += V^T[dim, token] . P^T[token, row]
//
// The rows of a head of keys are its (new token, query head of the group) pairs, token by token, so that a workgroup's 128 rows are few tokens:
// they share every tile of keys and values, and only the last tiles are cut by the diagonal.  A wave has 32 of them as two blocks of 16; tiles
// go through a ring of four in LDS that direct loads fill.  A lane holds one row per block: the running maximum and sum need two
// exchanges between lanes, and the weights stay in the registers that the scores came in.  Tiles that every row of the workgroup sees whole run
// in a loop of their own, without masks and without a look at the block table.
//
// Bound by vector and matrix instructions that hardly pass at the same time: of a 16384-token prompt (32 heads on 8, 128 columns, 2.2 TFLOP) 1970 - 2210 us on
// different boxes = 1.0 - 1.12 PFLOP/s, the matrix cores are busy 48 % of the time and the vector units 56 %; the socket draws 1375 W of its 1400, the clock is at 2.23 of 2.4 GHz.
// Weights in bf16 for the second product, as in heads_ranges.hip; their sum in float from the unrounded ones (the log-sum-exp is a float's).
// Measured and not kept: exponentials of one block of rows between the matrix instructions of the other, the next tile's keys read ahead (2095 us; with the
// values read once per block 2240, against 2080 in this order at the time); workgroups of 256 rows (2092, 13 packed prompts 148 -> 162 us); fewer instructions
// for the maximum and the reference (1990 -> 2030).
#include "heads_tile.h"

#include <algorithm>

namespace tpla {

constexpr int HP_NW = 4, HP_QB = 2, HP_ROWS = HP_NW * HP_QB * 16;
constexpr int HP_PER_CU = 8 / HP_NW;
constexpr int HP_NSTAGE = 4;
constexpr int HP_TILE = 8192;            // bytes of keys, and of values, of a tile
constexpr int HP_CPT = HP_TILE / 1024 / HP_NW;   // direct loads per wave, of keys and of values
constexpr int HP_IDS = 1024;             // page ids held at once
constexpr int HP_ODD = HP_NSTAGE * 2 * HP_TILE + HP_IDS * 4;
constexpr int HP_LDS = HP_ODD + (HP_NSTAGE + HP_NW) * 4;
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
__device__ __forceinline__ float wave_total(float v) {
  const int lane = threadIdx.x & 63;
  v += lane_xor<1>(v, lane);
  v += lane_xor<2>(v, lane);
  v += lane_xor<4>(v, lane);
  v += lane_xor<8>(v, lane);
  v += lane_xor<16>(v, lane);
  return v + lane_xor<32>(v, lane);
}
__device__ __forceinline__ float wave_most(float v) {
  const int lane = threadIdx.x & 63;
  v = fmaxf(v, lane_xor<1>(v, lane));
  v = fmaxf(v, lane_xor<2>(v, lane));
  v = fmaxf(v, lane_xor<4>(v, lane));
  v = fmaxf(v, lane_xor<8>(v, lane));
  v = fmaxf(v, lane_xor<16>(v, lane));
  return fmaxf(v, lane_xor<32>(v, lane));
}
// Tokens of a part: of a few lengths, the one that ends first by an estimate in tokens (floats: every workgroup comes to the same).  S: workgroups at once.
//   - no split: the longest item, or where there is more than a round of them, the mean of a round's workgroups and half an item;
//   - parts of c tokens: c if they are one round, otherwise the mean and half of a part; and HP_MERGE for the partial results.
// A few parts more than a round take as long as two: two sequences, 16 and 7 tiles of 8512 and 20211 tokens, 8 heads of keys: 536 parts of 4288 tokens 237 us, 480 of
// 5120 200.  One prompt of 2000 tokens, 504 items, 32 heads on 8: unsplit 87 us, in parts of 1024 79; of 4000, 1000 items: stays unsplit.
constexpr float HP_MERGE = 384.f;
__device__ __forceinline__ int prompt_chunk(const HeadsArgs& a, const PromptSeq& front) {
  const int lane = threadIdx.x & 63;
  const float S = (float)a.n_wg, per_token = (float)a.G * (1.f / HP_ROWS);      // tiles per new token
  // of one sequence: tokens that all its tiles read (tile i sees some L + (i + 1) / per_token)
  auto reads = [&](const PromptSeq& s) { return s.tiles * ((float)min(s.it.L, s.it.keys) + 0.5f * (float)(s.it.keys - min(s.it.L, s.it.keys))); };
  float work = reads(front), items = (float)front.tiles, longest = front.tiles > 0 ? (float)front.it.keys : 0.f;
  for (int b0 = 64; b0 < a.B; b0 += 64) {
    const PromptSeq s = prompt_seq(a, b0 + lane);
    work += reads(s);
    items += (float)s.tiles;
    longest = fmaxf(longest, s.tiles > 0 ? (float)s.it.keys : 0.f);
  }
  const float mean = wave_total(work) * (float)a.H_kv / S;
  items = wave_total(items) * (float)a.H_kv;
  longest = wave_most(longest);
  if (!(mean < 1073741824.f) || items == 0.f) return 0x7fffffff;
  float best = items <= S ? longest : fmaxf(longest, mean + 0.5f * mean * S / items);
  int chunk = 0x7fffffff;
#pragma unroll 1
  for (int k = 0; k < 3; ++k) {
    const int c = max(((int)(mean * (1.f + 0.19f * k)) + 63) / 64 * 64, HP_CHUNK_MIN);
    float parts = 0.f, room = 0.f;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      const PromptSeq s = b0 == 0 ? front : prompt_seq(a, b0 + lane);
      // the tiles that see more than p c tokens, over p
      const int all = heads_parts(s.it.keys, c);
      const float first = fminf(floorf((float)s.it.L / (float)c) + 1.f, (float)all);      // parts 0 .. first - 1 are every tile's
      const float n = (float)all - first, gone = n * ((float)c * 0.5f * ((float)all - 1.f + first) - (float)s.it.L) * per_token;
      parts += s.tiles > 0 ? fmaxf((float)s.tiles * (float)all - gone, (float)s.tiles) : 0.f;
      room += (float)s.tiles * (float)all;
    }
    parts = wave_total(parts) * (float)a.H_kv;
    if (wave_total(room) * (float)a.H_kv > (float)a.n_splits * S) continue;      // (below 2^24: exact)
    const float ends = (parts <= S ? (float)c : mean + 0.5f * mean * S / parts) + HP_MERGE;
    if (ends < best) {
      best = ends;
      chunk = c;
    }
  }
  return __builtin_amdgcn_readfirstlane(chunk);
}

// Lane k gets what the sequence with the k-th largest key has in this lane (ties by index): `from` its lane.  Bit by bit from the top: the sequences that
// agree with this lane's so far, those of them that are larger by this bit.
__device__ __forceinline__ int longest_first(int key, int& from) {
  const int lane = threadIdx.x & 63;
  int top = key;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = max(top, __shfl_xor(top, d));
  unsigned long long same = ~0ull;
  int rank = 0;
  for (int bit = 31 - __builtin_clz(__builtin_amdgcn_readfirstlane(top) | 1); bit >= 0; --bit) {
    const bool mine = (key >> bit) & 1;
    const unsigned long long set = __ballot(mine);
    rank += mine ? 0 : __popcll(same & set);
    same &= mine ? set : ~set;
  }
  rank += __popcll(same & ((1ull << lane) - 1));
  from = __builtin_amdgcn_ds_permute(4 * rank, lane);
  return rank;
}

// Heads of keys are the fastest index: workgroups go to the XCDs in turn, so each XCD's L2 holds the keys and values of few heads.  Whole sequences follow,
// longest first (in groups of 64), PARTS: the parts of all tiles one after the other, and the tiles of a sequence from its last (most keys) to its
// first: the grid ends on short items.  (From the first tile to the last, one prompt of 4000 tokens, 32 heads on 8: 202 us; so 176.)
// ITEMS: the unit is an item's part 0 and idx counts items alone (the merge, which finds the chunk in a.plan).
template <bool PARTS, bool ITEMS>
__device__ __forceinline__ bool prompt_unit(const HeadsArgs& a, int idx, PromptUnit& u) {
  const int lane = threadIdx.x & 63;
  const int kvh = idx % a.H_kv;
  int at = idx / a.H_kv, before = 0;
  const PromptSeq front = prompt_seq(a, lane);
  const int chunk = ITEMS ? a.plan[0] : PARTS ? prompt_chunk(a, front) : 0x7fffffff;
  if (PARTS && !ITEMS && blockIdx.x == 0 && threadIdx.x == 0) a.plan[0] = chunk;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const PromptSeq s = b0 == 0 ? front : prompt_seq(a, b0 + lane);
    int tiles = s.tiles, units = s.tiles * (PARTS ? heads_parts(s.it.keys, chunk) : 1), from = lane;
    if (a.B > 1) {
      longest_first((s.it.keys >> 5) + (s.tiles > 0 ? 1 : 0), from);
      tiles = __shfl(tiles, from);
      units = __shfl(units, from);
    }
    const int count = ITEMS ? tiles : units, incl = wave_prefix(units), count_incl = ITEMS ? wave_prefix(count) : incl;
    const unsigned long long past = __ballot(count_incl > at);
    if (past == 0) {
      at -= __builtin_amdgcn_readlane(count_incl, 63);
      before += __builtin_amdgcn_readlane(incl, 63);
      continue;
    }
    const int place = __builtin_ctzll(past), src = __builtin_amdgcn_readlane(from, place);
    at -= __builtin_amdgcn_readlane(count_incl - count, place);
    before += __builtin_amdgcn_readlane(incl - units, place);
    tiles = __builtin_amdgcn_readlane(tiles, place);
    u.it.b = b0 + src;
    u.it.kvh = kvh;
    u.it.first = __builtin_amdgcn_readlane(s.it.first, src);
    u.it.rows = __builtin_amdgcn_readlane(s.it.rows, src);
    u.it.L = __builtin_amdgcn_readlane(s.it.L, src);
    u.it.keys = __builtin_amdgcn_readlane(s.it.keys, src);
    const int part = PARTS ? at / tiles : 0, nth = PARTS ? at - part * tiles : at;
    u.it.row0 = (tiles - 1 - nth) * HP_ROWS;
    const int keys = max(u.it.sees(min(u.it.row0 + HP_ROWS, u.it.rows) - 1, a.G), 0);
    u.parts = PARTS ? heads_parts(keys, chunk) : 1;
    u.slot = (before + nth) * a.H_kv + kvh;
    u.step = tiles * a.H_kv;
    if (part >= u.parts) return false;
    u.k0 = PARTS ? part * chunk : 0;                   // (part < parts: below keys)
    u.k1 = keys - u.k0 > chunk ? u.k0 + chunk : keys;
    u.slot += part * u.step;
    return true;
  }
  return false;
}

// ONE: pages of whole tiles.
template <int D, bool PARTS, bool ONE>
__global__ void __launch_bounds__(HP_NW * 64, 2) heads_prompts_kernel(HeadsArgs a) {
  constexpr int RC = D / 8, TOK = HP_TILE / (2 * D), TB = TOK / 16, KS = D / 32, DB = D / 16, QB = HP_QB;
  constexpr int LOAD_TOK = 64 / RC;
  static_assert(QB * DB <= 16, "accumulators of 64 registers");
  extern __shared__ u32x4 smem[];
  char* const lds = reinterpret_cast<char*>(smem);
  int* const ids = reinterpret_cast<int*>(lds + HP_NSTAGE * 2 * HP_TILE);
  int* const odd_tile = reinterpret_cast<int*>(lds + HP_ODD);      // 1 + the last tile of each place that holds values that are not finite
  int* const first_hole = odd_tile + HP_NSTAGE;                     // of the ids that each wave has read, the first page that is missing
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j16 = lane & 15, q4 = lane >> 4;
  PromptUnit u;
  if (!prompt_unit<PARTS, false>(a, blockIdx.x, u)) return;
  const HeadsItem it = u.it;
  const int keys = it.keys;
  if (tid < HP_NSTAGE) odd_tile[tid] = 0;

  // ---- per-lane places ----
  unsigned ld_at[HP_CPT];
#pragma unroll
  for (int j = 0; j < HP_CPT; ++j) {
    const int tok = (wave + j * HP_NW) * LOAD_TOK + lane / RC;      // the piece of the row that this lane loads, and the row within the load
    ld_at[j] = (unsigned)((ONE ? tok : lane / RC) * (2 * D) + ((lane % RC) ^ heads_swz<RC>(tok)) * 16);
  }
  // Rows begin at whole 128 bytes and places at whole 16 KB, so pieces of a row differ in a few address bits alone: k-step ks of the keys is at ks << 6,
  // block d of the values at d << 5 of the first one's.
  const unsigned k_at = (unsigned)((j16 * RC + (q4 ^ heads_swz<RC>(j16))) * 16);
  const int v_tok = 4 * q4 + (j16 >> 2);
  const unsigned v_at = (unsigned)(HP_TILE + (v_tok * RC + (((j16 & 3) >> 1) ^ heads_swz<RC>(v_tok))) * 16 + (j16 & 1) * 8);
  const unsigned lds_base = lds_at(lds);

  const int pt = a.page_tokens, shift = (pt & (pt - 1)) == 0 ? __builtin_ctz(pt) : -1;
  auto page_of = [&](int t) { return shift >= 0 ? t >> shift : t / pt; };
  const size_t page_bytes = (size_t)a.H_kv * pt * (2 * D);
  const int32_t* table = a.table + (size_t)it.b * a.max_pages;
  const char* k_head = static_cast<const char*>(a.k_pool) + (size_t)it.kvh * pt * (2 * D);
  const char* v_head = static_cast<const char*>(a.v_pool) + (size_t)it.kvh * pt * (2 * D);
  int id0 = 0;

  // Where a load is: its tokens lie in one page (pages are a multiple of 16 tokens), ONE: those of all loads of a tile do.  Walked from tile to tile
  // without divisions.
  constexpr int CURS = ONE ? 1 : HP_CPT;
  auto load_tok = [&](int t, int j) { return t * TOK + (ONE ? 0 : (wave + j * HP_NW) * LOAD_TOK); };
  struct Cursor {
    int page, off;
  };
  Cursor cur[CURS];
  const int step_pages = TOK / pt, step_off = TOK % pt;
  auto seek = [&](int t) {
#pragma unroll
    for (int j = 0; j < CURS; ++j) {
      const int tok = load_tok(t, j);
      cur[j].page = page_of(tok);
      cur[j].off = tok - cur[j].page * pt;
    }
  };
  auto advance = [&]() {
#pragma unroll
    for (int j = 0; j < CURS; ++j) {
      cur[j].page += step_pages;
      cur[j].off += step_off;
      if (cur[j].off >= pt) {
        cur[j].off -= pt;
        ++cur[j].page;
      }
    }
  };
  // Tile t on its way, all of its tokens exist; id: its loads' pages, where the cursors are.
  auto issue_whole = [&](int t, const int (&id)[CURS]) {
    char* dst = lds + (t % HP_NSTAGE) * (2 * HP_TILE) + wave * 1024;
    size_t at[CURS];
#pragma unroll
    for (int j = 0; j < CURS; ++j) at[j] = (unsigned)max(__builtin_amdgcn_readfirstlane(id[j]), 0) * page_bytes + (size_t)(unsigned)cur[j].off * (2 * D);
#pragma unroll
    for (int j = 0; j < HP_CPT; ++j)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(k_head + at[j % CURS] + ld_at[j]),
                                       (__attribute__((address_space(3))) void*)(dst + j * HP_NW * 1024), 16, 0, 0);
#pragma unroll
    for (int j = 0; j < HP_CPT; ++j)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(v_head + at[j % CURS] + ld_at[j]),
                                       (__attribute__((address_space(3))) void*)(dst + HP_TILE + j * HP_NW * 1024), 16, 0, 0);
  };
  // Tokens past the end repeat the last one, those of missing pages are page 0's; they are masked, and their values zeroed.
  auto issue = [&](int t) {
    if ((t + 1) * TOK <= keys) {
      int id[CURS];
#pragma unroll
      for (int j = 0; j < CURS; ++j) id[j] = lds_read_page(ids + (cur[j].page - id0));
      issue_whole(t, id);
      advance();
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
    if (t + HP_NSTAGE - 2 < c1)
      loads_wait<(HP_NSTAGE - 2) * 2 * HP_CPT>();
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
    const bf16_t* src = static_cast<const bf16_t*>(a.q) + out_row(min(row_w + 16 * r + j16, it.rows - 1)) * D + 8 * q4;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[r][ks] = *reinterpret_cast<const bf16x8*>(src + 32 * ks);
    m[r] = -INFINITY;
    l[r] = 0.f;
    seen[r] = 0;
  }
  out_keep();
  static_for<QB * DB>([&](auto ic) { out_write<decltype(ic)::value>(f32x4{0.f, 0.f, 0.f, 0.f}); });

  // The rare step: a score above the reference by more than LAZY.  top: largest score of this lane, in powers of two.
  auto raise = [&](auto rc, float top) {
    constexpr int r = decltype(rc)::value;
    top = fmaxf(top, lane_xor<16>(top, lane));
    top = fmaxf(top, lane_xor<32>(top, lane));
    const float m_new = fmaxf(m[r], top);
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[r] - m_new);
    l[r] *= alpha;
    m[r] = m_new;
    out_settle_result();
    static_for<DB>([&](auto dc) { out_scale<r * DB + decltype(dc)::value>(alpha); });
  };

  // ---- a tile that some rows do not see whole; there: its blocks of 16 tokens that have a page ----
  auto cut_tile = [&](int t, int there) {
    const int tok0 = t * TOK;
    const unsigned base = lds_base + (unsigned)((t % HP_NSTAGE) * (2 * HP_TILE)), kb = base + k_at, vb = base + v_at;
    f32x4 s[QB][TB];
    {
      constexpr int N = KS * TB, AHEAD = D == 128 ? 8 : 4;
      bf16x8 kf[AHEAD];
      static_for<AHEAD>([&](auto ic) {
        constexpr int x = decltype(ic)::value;
        lds_read_b128<(x % TB) * (16 * RC * 16)>(kf[x], kb ^ ((x / TB) << 6));
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
        if constexpr (x + AHEAD < N) lds_read_b128<((x + AHEAD) % TB) * (16 * RC * 16)>(kf[x % AHEAD], kb ^ (((x + AHEAD) / TB) << 6));
      });
    }
    constexpr int NV = DB * (TB / 2), VA = 4;
    u32x2 lo[VA], hi[VA];
    auto value = [&](auto yc) {
      constexpr int y = decltype(yc)::value;
      lds_read_tr_b64<(y / DB) * (32 * RC * 16)>(lo[y % VA], vb ^ ((y % DB) << 5));
      lds_read_tr_b64<(y / DB) * (32 * RC * 16) + 16 * RC * 16>(hi[y % VA], vb ^ ((y % DB) << 5));
    };
    out_settle_result();
#pragma unroll
    for (int r = 0; r < QB; ++r)
#pragma unroll
      for (int n = 0; n < TB; ++n) settle_scores(s[r][n]);

    bf16x8 p[QB][TB / 2];
    static_for<QB>([&](auto rc) {
      constexpr int r = decltype(rc)::value;
#pragma unroll
      for (int n = 0; n < TB; ++n) {
        const int left = ((there >> n) & 1) ? sees[r] - tok0 - 16 * n - 4 * q4 : 0;
        seen[r] |= left > 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[r][n][i] = i < left ? s[r][n][i] : -INFINITY;
      }
      float top = s[r][0][0];
#pragma unroll
      for (int n = 0; n < TB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][n][i]);
      top *= a.scale_log2;
      if (__any(top > m[r] + LAZY)) raise(rc, top);
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
    const bool odd = __builtin_amdgcn_readfirstlane(lds_read_page(odd_tile + t % HP_NSTAGE)) == t + 1;
    if (!odd) {
      static_for<VA>([&](auto ic) { value(ic); });
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
          lds_read_tr_b64<0>(vlo, (vb ^ (d << 5)) + h * (32 * RC * 16));
          lds_read_tr_b64<16 * RC * 16>(vhi, (vb ^ (d << 5)) + h * (32 * RC * 16));
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

  // ---- a tile that all rows of the workgroup see ----
  static_assert(HP_NSTAGE * 2 * HP_TILE <= 65536, "places within the offset of an LDS read");
  unsigned k_reg[KS], v_reg[DB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_reg[ks] = lds_base + (k_at ^ (ks << 6));
#pragma unroll
  for (int d = 0; d < DB; ++d) v_reg[d] = lds_base + (v_at ^ (d << 5));
  // PLACE: t % HP_NSTAGE, so that the places are offsets of the reads and not addresses to be added.
  auto plain_tile = [&](auto place) {
    constexpr int NS = KS * TB, NV = DB * (TB / 2), VA = 4, AT = decltype(place)::value * 2 * HP_TILE;
    f32x4 s[QB][TB];
    bf16x8 kf[NS], p[QB][TB / 2];
    u32x2 lo[VA], hi[VA];
    static_for<NS>([&](auto ic) {
      constexpr int x = decltype(ic)::value;
      lds_read_b128<AT + (x % TB) * (16 * RC * 16)>(kf[x], k_reg[x / TB]);
    });
    static_for<NS>([&](auto ic) {
      constexpr int x = decltype(ic)::value, ks = x / TB, n = x % TB;
      lds_wait<NS - 1 - x>(kf[x]);
#pragma unroll
      for (int r = 0; r < QB; ++r) {
        if constexpr (ks == 0)
          score_first(s[r][n], kf[x], q[r][ks]);
        else
          score_more(s[r][n], kf[x], q[r][ks]);
      }
    });
    // the first values start now, so that their way from LDS passes under the softmax
    auto value = [&](auto yc) {
      constexpr int y = decltype(yc)::value;
      lds_read_tr_b64<AT + (y / DB) * (32 * RC * 16)>(lo[y % VA], v_reg[y % DB]);
      lds_read_tr_b64<AT + (y / DB) * (32 * RC * 16) + 16 * RC * 16>(hi[y % VA], v_reg[y % DB]);
    };
    static_for<VA>([&](auto ic) { value(ic); });
    out_settle_write();
    out_settle_write();
#pragma unroll
    for (int r = 0; r < QB; ++r)
#pragma unroll
      for (int n = 0; n < TB; ++n) settle_scores(s[r][n]);
    static_for<QB>([&](auto rc) {
      constexpr int r = decltype(rc)::value;
      float top = s[r][0][0];
#pragma unroll
      for (int n = 0; n < TB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[r][n][i]);
      top *= a.scale_log2;
      if (__any(top > m[r] + LAZY)) raise(rc, top);
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
    static_for<NV>([&](auto ic) {
      constexpr int x = decltype(ic)::value, d = x % DB, h = x / DB, ahead = NV - 1 - x < VA - 1 ? NV - 1 - x : VA - 1;
      lds_wait<2 * ahead>(lo[x % VA], hi[x % VA]);
      const u32x4 v = {lo[x % VA][0], lo[x % VA][1], hi[x % VA][0], hi[x % VA][1]};
      static_for<QB>([&](auto rc) { out_product<decltype(rc)::value * DB + d>(v, p[decltype(rc)::value][h]); });
      if constexpr (x + VA < NV) value(std::integral_constant<int, x + VA>{});
    });
  };

  const int t0 = u.k0 / TOK, t1 = (u.k1 + TOK - 1) / TOK;
  const int id_tiles = (int)min(max((long long)(HP_IDS - 1) * pt / TOK, 1ll), 1ll << 26);           // tiles whose pages fit in ids, wherever in a page they begin
  for (int c0 = t0; c0 < t1; c0 += id_tiles) {
    const int c1 = min(t1, c0 + id_tiles);
    if (c0 > t0) __syncthreads();                      // the ids and tiles before are read
    id0 = page_of(c0 * TOK);
    int missing = 0x7fffffff;
    for (int x = tid; x < HP_IDS; x += HP_NW * 64) {
      const int p = id0 + x;
      if (p < a.max_pages && (long long)p * pt < (long long)min(keys, c1 * TOK)) {
        const int id = table[p];
        ids[x] = id;
        if (id < 0) missing = min(missing, p);
      }
    }
    if (__any(missing != 0x7fffffff))
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) missing = min(missing, __shfl_xor(missing, d));
    if (lane == 0) first_hole[wave] = missing;
    __syncthreads();
    // tiles that exist whole and that every row of the workgroup sees
    int hole = first_hole[0];
#pragma unroll
    for (int w = 1; w < HP_NW; ++w) hole = min(hole, first_hole[w]);
    hole = __builtin_amdgcn_readfirstlane(hole);
    const int plain = hole == 0x7fffffff ? least : min(least, hole * pt);
    const int whole = min(c1, max(c0, plain / TOK));
    seek(c0);
    for (int t = c0; t < min(c1, c0 + HP_NSTAGE - 1); ++t) issue(t);
#pragma unroll
    for (int r = 0; r < QB; ++r)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[r][ks]));         // complete before the loop (and on every path to it: a wait within would be for the tiles)
    int t = c0;
    // the page ids of the tile that is requested next, read a tile ahead
    const int last_id = page_of(max(min(keys, c1 * TOK) - 1, 0)) - id0;
    int id[CURS];
#pragma unroll
    for (int j = 0; j < CURS; ++j) id[j] = lds_read_page(ids + min(cur[j].page - id0, last_id));
    for (; t < whole; ++t) {
      out_keep();
      arrived(t, c1);
      __builtin_amdgcn_s_barrier();                    // tile t is there for all waves, tile t - 1 is no longer read
      asm volatile("" ::: "memory");
      const int next = t + HP_NSTAGE - 1;
      if (next < c1) {
        if ((next + 1) * TOK <= keys) {
          issue_whole(next, id);
          advance();
        } else {
          issue(next);
        }
      }
#pragma unroll
      for (int j = 0; j < CURS; ++j) lds_request_page(id[j], ids + min(cur[j].page - id0, last_id));
      static_for<HP_NSTAGE>([&](auto place) {
        if (t % HP_NSTAGE == decltype(place)::value) plain_tile(place);
      });
#pragma unroll
      for (int j = 0; j < CURS; ++j) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(id[j]) : : "memory");      // (long there)
    }
    if (t > c0) seen[0] = seen[1] = 1;
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
      cut_tile(t, there);
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

// grid: (items, HP_MERGE_Y): the rows of an item dealt over workgroups.  The parts of a row in their order, a thread for four columns.
constexpr int HP_MERGE_Y = 4;
template <int D>
__global__ void __launch_bounds__(256) heads_prompts_merge_kernel(HeadsArgs a) {
  constexpr int LPR = D / 4, AT_ONCE = 256 / LPR;
  if (a.plan[0] == 0x7fffffff) return;                 // nothing was split
  PromptUnit u;
  if (!prompt_unit<true, true>(a, blockIdx.x, u) || u.parts == 1) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  const int c = 4 * (threadIdx.x % LPR);
  for (int r = blockIdx.y * AT_ONCE + threadIdx.x / LPR; r < HP_ROWS && u.it.row0 + r < u.it.rows; r += HP_MERGE_Y * AT_ONCE) {
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
    const int row = u.it.row0 + r;
    const size_t out = (size_t)(u.it.first + row / a.G) * a.H + u.it.kvh * a.G + row % a.G;
    const float inv = heads_inverse(sum);
    store4(a.o, out * D + c, a.o_dtype, sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv);
    if (a.lse && c == 0) a.lse[out] = heads_lse(M, sum);
  }
}

static int64_t prompts_items(const tpla_heads_t& sh, int64_t T) { return (T * (sh.H / sh.H_kv) / HP_ROWS + sh.B) * sh.H_kv; }

HeadsPlan heads_prompts_plan(const tpla_heads_t& sh, int64_t T, int32_t max_new, int32_t max_pages) {
  HeadsPlan p;
  p.kernel = HEADS_PROMPTS;
  p.rows = HP_ROWS;
  p.items = prompts_items(sh, T);
  p.tiles = (int)(p.items / sh.H_kv);
  p.n_wg = HP_PER_CU * device_cu_count();                      // workgroups that the chip holds
  // Split where the items do not fill it twice and there are tokens to split; n_splits: rounds of partial results that there is room for.
  const bool split = p.items < 2 * p.n_wg && (int64_t)max_pages * sh.page_tokens > HP_CHUNK_MIN;
  p.n_splits = split ? (int)(p.items / p.n_wg) + 2 : 1;
  p.slots = split ? p.n_splits * (int64_t)p.n_wg : 0;
  p.workspace = p.slots > 0 ? (size_t)p.slots * p.rows * (sh.d_v + 2) * sizeof(float) + 16 : 0;
  return p;
}

size_t heads_prompts_room(const tpla_heads_t& sh, int64_t T, int32_t max_pages) {
  if ((int64_t)max_pages * sh.page_tokens <= HP_CHUNK_MIN) return 0;
  const int64_t n_wg = HP_PER_CU * device_cu_count();
  return (size_t)((std::min(prompts_items(sh, T), 2 * n_wg - 1) / n_wg + 2) * n_wg) * HP_ROWS * (sh.d_v + 2) * sizeof(float) + 16;
}

template <int D>
static auto prompts_kernel_of(bool parts, bool one) -> void (*)(HeadsArgs) {
  return parts ? (one ? heads_prompts_kernel<D, true, true> : heads_prompts_kernel<D, true, false>)
               : (one ? heads_prompts_kernel<D, false, true> : heads_prompts_kernel<D, false, false>);
}

int launch_heads_prompts(const HeadsArgs& a, const HeadsPlan& p, hipStream_t st) {
  const bool parts = p.n_splits > 1, one = a.page_tokens % (HP_TILE / (2 * a.d_k)) == 0;
  void (*fn)(HeadsArgs) = a.d_k == 128 ? prompts_kernel_of<128>(parts, one) : prompts_kernel_of<64>(parts, one);
  int rc = allow_lds(reinterpret_cast<const void*>(fn), HP_LDS, "heads_prompts_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3((unsigned)(parts ? p.slots : p.items)), dim3(HP_NW * 64), HP_LDS, st, a);
  if ((rc = check_launch("heads_prompts_kernel")) || !parts) return rc;
  hipLaunchKernelGGL(a.d_k == 128 ? heads_prompts_merge_kernel<128> : heads_prompts_merge_kernel<64>, dim3((unsigned)p.items, HP_MERGE_Y), dim3(256), 0, st, a);
  return check_launch("heads_prompts_merge_kernel");
}

}  // namespace tpla
