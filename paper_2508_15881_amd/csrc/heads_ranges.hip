// Attention of a few rows per head of keys (single tokens; a few new tokens) over paged keys and values on the bf16 matrix instructions.
//
//   S^T[token, row] = K[token, :] . Q[row, :],   O^T[dim, row] += V^T[dim, token] . P^T[token, row]
//
// Bound by the bytes of the cache: a group of up to 16 query heads shares one block of 16 columns.  Tiles of 8 KB of keys and 8 KB of values
// of all items (sequence, head of keys, tile of rows) are laid end to end and cut into equal ranges, one per workgroup.  Its four waves take
// the tiles of an item in turn, each with a place of its own in LDS that direct loads fill: no barrier within an item, the next keys are
// requested once the scores have read the last ones, the next values after the output product, and eight waves on a compute unit keep some
// 100 KB on their way.  An item that lies in one range is written at once, the parts of the others are merged by a second kernel.
// 48 sequences of 500 to 32000 tokens, 32 heads on 8, 128 columns (1.53 GB): 240 us with the merge = 6.4 TB/s, where a pure reader reaches 7.2; one sequence of
// 9001 tokens 17.5 us: under the profiler the kernel's 14.5 (lengths, page ids, first tiles, each a round trip, four tiles per wave and the join) and 4 of merge.
//
// The weights are rounded to bf16 for the second product, as in the latent decode: its instruction takes both operands in one type, and a second one with what
// the rounding left would double that product.  References, sums and the log-sum-exp are floats of unrounded weights.  Against 64 bits, in norms, outputs in bf16
// are off by 0.0018 to 0.0023, where float weights (the plain form) leave 0.0016, the rounding of the output.
#include "heads_tile.h"

#include <algorithm>

namespace tpla {

constexpr int HN_NW = 4;
constexpr int HN_TILE = 8192;            // bytes of keys, and of values, of a tile
constexpr int HN_LOADS = HN_TILE / 1024; // direct-to-LDS loads each
// Rows per head of keys at most: more fill the tiles of heads_prompts.hip (4000 tokens: 2 sequences, 32 rows 15.4 us here, 29.8 there; 8 sequences of 8 heads of
// keys, 20 rows 38.4 and 39.7, 48 rows 138 and 41).
constexpr int HN_MOST = 32;
constexpr int HN_IDS = 1024;             // page ids held at once
// Cache policy of the loads: not kept behind their use.  The cache is read once per step, and lines kept for it push out what is on its way (48 ragged
// sequences, 1.5 GB: 269 us with the ordinary policy, 240 so).
constexpr int HN_AUX = 2;
constexpr int HN_MIN_UNITS = 4;          // tiles of a range at least: one per wave
// Units of an item ahead of its tiles, for what it costs besides them (page ids, queries, the way of the first tiles, the join): many short items
// are spread over the workgroups, and ranges with several of them end with the others.
constexpr int HN_START = 4;
constexpr int HN_LDS = HN_NW * 2 * HN_TILE + HN_IDS * 4;

__host__ __device__ __forceinline__ int range_start(int n_wg, int units, int w) { return (int)((long long)w * units / n_wg); }
// The last workgroup whose range begins at or before unit u.
__host__ __device__ __forceinline__ int range_owner(int n_wg, int units, int u) { return (int)((((long long)u + 1) * n_wg - 1) / units); }

// The range of tiles of this workgroup, [pos, end), and the item that tile `pos` lies in.  An item has one tile at least, so that somebody
// writes the rows that see nothing.
template <int TOK, int ROWS>
struct HeadsWalk {
  struct Units {
    HeadsItem it;
    int tiles, blocks;         // no new tokens: no blocks
  };
  int units, n_wg, w, pos, range0, end, front_incl;
  Units front;
  // the item
  HeadsItem it;
  int item, tiles, t0, t1, slot, last;
  bool whole;

  static __device__ __forceinline__ Units units_of(const HeadsArgs& a, int b) {
    Units u{};
    if (b >= a.B) return u;
    int first;
    const int n = heads_new(a, b, first);
    u.it.b = b;
    u.it.first = first;
    u.it.rows = n * a.G;
    heads_lens(a, b, n, u.it);
    u.blocks = (u.it.rows + ROWS - 1) / ROWS;
    u.tiles = max((u.it.keys + TOK - 1) / TOK, 1);
    return u;
  }
  __device__ __forceinline__ int count(const HeadsArgs& a, const Units& u) const { return u.blocks * (u.tiles + HN_START) * a.H_kv; }
  // One workgroup per item.
  __device__ __forceinline__ bool take_item(const HeadsArgs& a) {
    item = blockIdx.x;
    const int block = item % a.tiles, v = item / a.tiles;
    it.b = v / a.H_kv;
    it.kvh = v % a.H_kv;
    it.row0 = block * ROWS;
    const int n = heads_new(a, it.b, it.first);
    it.rows = n * a.G;
    if (it.row0 >= it.rows) return false;
    heads_lens(a, it.b, n, it);
    t0 = 0;
    t1 = tiles = max((it.keys + TOK - 1) / TOK, 1);
    whole = true;
    pos = end = 0;
    return true;
  }
  __device__ __forceinline__ bool begin(const HeadsArgs& a) {
    const int lane = threadIdx.x & 63;
    front = units_of(a, lane);
    front_incl = wave_prefix(count(a, front));
    units = __builtin_amdgcn_readlane(front_incl, 63);
    for (int b0 = 64; b0 < a.B; b0 += 64) units += __builtin_amdgcn_readlane(wave_prefix(count(a, units_of(a, b0 + lane))), 63);
    n_wg = max(1, min(a.n_wg, units / HN_MIN_UNITS));
    w = blockIdx.x;
    if (w >= n_wg || units == 0) return false;
    range0 = pos = range_start(n_wg, units, w);
    end = range_start(n_wg, units, w + 1);
    return true;
  }
  // The next item with tiles in the range; false: there is none.  a.tiles: items per (sequence, head of keys) that the plan has room for.
  __device__ __forceinline__ bool find(const HeadsArgs& a) {
    const int lane = threadIdx.x & 63;
    while (pos < end) {
      int b0 = 0, incl = front_incl;
      Units u = front;
      unsigned long long past = __ballot(incl > pos);
      while (past == 0) {                              // ends: pos lies below the sum over all sequences
        b0 += 64;
        const int base = __builtin_amdgcn_readlane(incl, 63);
        u = units_of(a, b0 + lane);
        incl = wave_prefix(count(a, u)) + base;
        past = __ballot(incl > pos);
      }
      const int src = __builtin_ctzll(past), rem = pos - __builtin_amdgcn_readlane(incl - count(a, u), src);
      tiles = __builtin_amdgcn_readlane(u.tiles, src);
      const int span = tiles + HN_START, which = rem / span, at = rem - which * span, stop = min(span, at + (end - pos));
      const bool first = pos == range0;
      last = pos - at + span - 1;
      pos += stop - at;
      t0 = max(at - HN_START, 0);
      t1 = stop - HN_START;
      if (t1 <= t0) continue;                          // the range ends before the item's first tile
      it.b = b0 + src;
      it.first = __builtin_amdgcn_readlane(u.it.first, src);
      it.rows = __builtin_amdgcn_readlane(u.it.rows, src);
      it.L = __builtin_amdgcn_readlane(u.it.L, src);
      it.keys = __builtin_amdgcn_readlane(u.it.keys, src);
      const int blocks = __builtin_amdgcn_readlane(u.blocks, src);
      it.kvh = which / blocks;
      const int block = which - it.kvh * blocks;
      it.row0 = block * ROWS;
      item = (it.b * a.H_kv + it.kvh) * a.tiles + block;
      whole = t0 == 0 && t1 == tiles;
      slot = 2 * w + (first ? 0 : 1);
      return true;
    }
    return false;
  }
  // Where the merge finds the item's parts: whoever has its first tile says so.
  __device__ __forceinline__ void note(const HeadsArgs& a) const {
    if (t0 != 0 || threadIdx.x != 0) return;
    a.plan[3 * item] = w;
    a.plan[3 * item + 1] = range_owner(n_wg, units, last) - w + 1;
    a.plan[3 * item + 2] = slot & 1;
  }
};

// D: width.  RB: blocks of 16 rows.
template <int D, int RB>
__global__ void __launch_bounds__(HN_NW * 64, RB == 1 ? 2 : 1) heads_ranges_kernel(HeadsArgs a) {
  constexpr int RC = D / 8, TOK = HN_TILE / (2 * D), TB = TOK / 16, KS = D / 32, DB = D / 16, ROWS = 16 * RB;
  constexpr int LOAD_TOK = 64 / RC;                    // tokens per direct load
  extern __shared__ u32x4 smem[];
  char* const lds = reinterpret_cast<char*>(smem);
  int* const ids = reinterpret_cast<int*>(lds + HN_NW * 2 * HN_TILE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j16 = lane & 15, q4 = lane >> 4;
  char* const kbuf = lds + wave * 2 * HN_TILE;
  char* const vbuf = kbuf + HN_TILE;

  HeadsWalk<TOK, ROWS> walk;
  const bool items = a.n_wg == 0;                      // short contexts: a workgroup per item
  if (!(items ? walk.take_item(a) : walk.begin(a) && walk.find(a))) return;

  unsigned ld_at[HN_LOADS], k_at[KS], v_at[DB];
#pragma unroll
  for (int k = 0; k < HN_LOADS; ++k) {
    const int tok = k * LOAD_TOK + lane / RC;
    ld_at[k] = (unsigned)(tok * (2 * D) + ((lane % RC) ^ heads_swz<RC>(tok)) * 16);
  }
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_at[ks] = lds_at(kbuf) + (j16 * RC + ((4 * ks + q4) ^ heads_swz<RC>(j16))) * 16;
  const int v_tok = 4 * q4 + (j16 >> 2);
#pragma unroll
  for (int d = 0; d < DB; ++d) v_at[d] = lds_at(vbuf) + (v_tok * RC + ((2 * d + ((j16 & 3) >> 1)) ^ heads_swz<RC>(v_tok))) * 16 + (j16 & 1) * 8;
  const int pt = a.page_tokens, shift = (pt & (pt - 1)) == 0 ? __builtin_ctz(pt) : -1;
  auto page_of = [&](int t) { return shift >= 0 ? t >> shift : t / pt; };
  const bool one_page = pt % TOK == 0;                 // a tile never crosses a page
  const size_t page_bytes = (size_t)a.H_kv * pt * (2 * D);

  do {
    const HeadsItem it = walk.it;
    const int keys = it.keys;
    const int32_t* table = a.table + (size_t)it.b * a.max_pages;
    const char* k_head = static_cast<const char*>(a.k_pool) + (size_t)it.kvh * pt * (2 * D);
    const char* v_head = static_cast<const char*>(a.v_pool) + (size_t)it.kvh * pt * (2 * D);
    int id0 = 0;                                       // first page in ids

    // The keys or values of tile t on their way.  Tokens past the end repeat the last one, those of missing pages are page 0's; they are masked.
    auto issue = [&](const char* head, char* dst, int t) {
      const int tok0 = t * TOK;
      if (one_page && tok0 + TOK <= keys) {
        const int p = page_of(tok0), id = max(__builtin_amdgcn_readfirstlane(lds_read_page(ids + (p - id0))), 0);
        const char* src = head + (size_t)id * page_bytes + (size_t)(tok0 - p * pt) * (2 * D);
#pragma unroll
        for (int k = 0; k < HN_LOADS; ++k)
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + ld_at[k]),
                                           (__attribute__((address_space(3))) void*)(dst + k * 1024), 16, 0, HN_AUX);
      } else {
#pragma unroll
        for (int k = 0; k < HN_LOADS; ++k) {
          const int at = k * LOAD_TOK + lane / RC, tok = min(tok0 + at, keys - 1), p = page_of(tok), id = max(lds_read_page(ids + (p - id0)), 0);
          const char* src = head + (size_t)id * page_bytes + (size_t)(tok - p * pt) * (2 * D) + ((lane % RC) ^ heads_swz<RC>(at)) * 16;
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                           (__attribute__((address_space(3))) void*)(dst + k * 1024), 16, 0, HN_AUX);
        }
      }
    };

    bf16x8 q[RB][KS];
    int sees[RB];
    size_t out_row[RB];
    f32x4 acc[RB][DB];
    float m[RB], l[RB];
    int seen[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const int row = it.row0 + 16 * r + j16, mine = min(row, it.rows - 1);
      sees[r] = row < it.rows ? it.sees(mine, a.G) : 0;
      out_row[r] = (size_t)(it.first + mine / a.G) * a.H + it.kvh * a.G + mine % a.G;
      m[r] = -INFINITY;
      l[r] = 0.f;
      seen[r] = 0;
#pragma unroll
      for (int d = 0; d < DB; ++d) acc[r][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int least = it.sees(it.row0, a.G);           // tokens that every row of the item sees

    const int id_tiles = (int)min(max((long long)(HN_IDS - 1) * pt / TOK, 1ll), 1ll << 26);         // tiles whose pages fit in ids, wherever in a page they begin
    for (int c0 = walk.t0; c0 < walk.t1; c0 += id_tiles) {
      const int c1 = min(walk.t1, c0 + id_tiles);
      __syncthreads();                                 // ids, and the waves' places of the item before, are read
      id0 = page_of(c0 * TOK);
      for (int x = tid; x < HN_IDS; x += HN_NW * 64) {
        const int p = id0 + x;
        if (p < a.max_pages && (long long)p * pt < (long long)keys) ids[x] = table[p];
      }
      __syncthreads();
      int t = c0 + wave;
      if (t < c1 && keys > 0) {
        issue(k_head, kbuf, t);
        issue(v_head, vbuf, t);
      }
      if (c0 == walk.t0) {
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) q[r][ks] = *reinterpret_cast<const bf16x8*>(static_cast<const bf16_t*>(a.q) + out_row[r] * D + 32 * ks + 8 * q4);
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[r][ks]));
      }
      if (keys == 0) break;
      for (; t < c1; t += HN_NW) {
        const int tok0 = t * TOK;
        const bool more = t + HN_NW < c1;
        // which of the tile's blocks of 16 tokens have a page
        int there = 0;
        if (one_page) {
          there = __builtin_amdgcn_readfirstlane(lds_read_page(ids + (page_of(tok0) - id0))) >= 0 ? (1 << TB) - 1 : 0;
        } else {
#pragma unroll
          for (int n = 0; n < TB; ++n)
            if (tok0 + 16 * n < keys && __builtin_amdgcn_readfirstlane(lds_read_page(ids + (page_of(tok0 + 16 * n) - id0))) >= 0) there |= 1 << n;
        }
        const bool ragged = tok0 + TOK > least || there != (1 << TB) - 1;

        // ---- scores ----
        loads_wait<HN_LOADS>();
        f32x4 s[RB][TB];
        {
          constexpr int N = KS * TB, AHEAD = N < 8 ? N : 8;
          bf16x8 kf[AHEAD];
          static_for<AHEAD>([&](auto ic) {
            constexpr int x = decltype(ic)::value;
            lds_read_b128<(x % TB) * (16 * RC * 16)>(kf[x], k_at[x / TB]);
          });
          static_for<N>([&](auto ic) {
            constexpr int x = decltype(ic)::value, ks = x / TB, n = x % TB;
            lds_wait<(N - 1 - x < AHEAD - 1 ? N - 1 - x : AHEAD - 1)>(kf[x % AHEAD]);
#pragma unroll
            for (int r = 0; r < RB; ++r)
              s[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[x % AHEAD], q[r][ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[r][n], 0, 0, 0);
            if constexpr (x + AHEAD < N) lds_read_b128<((x + AHEAD) % TB) * (16 * RC * 16)>(kf[x % AHEAD], k_at[(x + AHEAD) / TB]);
          });
        }
        if (more) issue(k_head, kbuf, t + HN_NW);

        // ---- running maximum and sum ----
        bf16x8 p[RB][TB / 2];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          float top = -INFINITY;
#pragma unroll
          for (int n = 0; n < TB; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (ragged) {
                const bool vis = ((there >> n) & 1) && tok0 + 16 * n + 4 * q4 + i < sees[r];
                seen[r] |= vis;
                s[r][n][i] = vis ? s[r][n][i] * a.scale_log2 : -INFINITY;
              } else {
                s[r][n][i] *= a.scale_log2;
              }
              top = fmaxf(top, s[r][n][i]);
            }
          if (!ragged) seen[r] = 1;
          top = fmaxf(top, lane_xor<16>(top, lane));
          top = fmaxf(top, lane_xor<32>(top, lane));
          const float m_new = fmaxf(m[r], top), ref = m_new == -INFINITY ? 0.f : m_new;
          const float alpha = __builtin_amdgcn_exp2f(m[r] - ref);
          m[r] = m_new;
          l[r] *= alpha;
#pragma unroll
          for (int n = 0; n < TB; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = __builtin_amdgcn_exp2f(s[r][n][i] - ref);
              l[r] += e;
              p[r][n / 2][4 * (n & 1) + i] = (bf16_t)e;
            }
#pragma unroll
          for (int d = 0; d < DB; ++d) acc[r][d] *= alpha;
        }

        // ---- output ----
        if (more)
          loads_wait<HN_LOADS>();
        else
          loads_wait<0>();
        bool odd = false;
        if (ragged) {
          // rows that are no tokens become zeros; values that are not finite among those that some rows see and others do not
          // (read and written here through the compiler: its waits for the loads above only come early)
#pragma unroll 1
          for (int k = 0; k < HN_LOADS; ++k) {
            const int at = k * LOAD_TOK + lane / RC;
            u32x4* piece = reinterpret_cast<u32x4*>(vbuf + k * 1024 + lane * 16);
            if (tok0 + at >= keys || !((there >> (at >> 4)) & 1)) {
              *piece = u32x4{0u, 0u, 0u, 0u};
            } else if (tok0 + at >= least) {
              const u32x4 v = *piece;
#pragma unroll
              for (int e = 0; e < 4; ++e) odd = odd || not_finite_pair(v[e]);
            }
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          odd = __any(odd);
        }
        if (!odd) {
          constexpr int N = DB * (TB / 2), AHEAD = 4;
          u32x2 lo[AHEAD], hi[AHEAD];
          static_for<AHEAD>([&](auto ic) {
            constexpr int x = decltype(ic)::value;
            lds_read_tr_b64<(x / DB) * (32 * RC * 16)>(lo[x], v_at[x % DB]);
            lds_read_tr_b64<(x / DB) * (32 * RC * 16) + 16 * RC * 16>(hi[x], v_at[x % DB]);
          });
          static_for<N>([&](auto ic) {
            constexpr int x = decltype(ic)::value, d = x % DB, h = x / DB, ahead = N - 1 - x < AHEAD - 1 ? N - 1 - x : AHEAD - 1;
            lds_wait<2 * ahead>(lo[x % AHEAD], hi[x % AHEAD]);
            const u32x4 v = {lo[x % AHEAD][0], lo[x % AHEAD][1], hi[x % AHEAD][0], hi[x % AHEAD][1]};
#pragma unroll
            for (int r = 0; r < RB; ++r)
              acc[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), p[r][h], acc[r][d], 0, 0, 0);
            if constexpr (x + AHEAD < N) {
              constexpr int y = x + AHEAD;
              lds_read_tr_b64<(y / DB) * (32 * RC * 16)>(lo[x % AHEAD], v_at[y % DB]);
              lds_read_tr_b64<(y / DB) * (32 * RC * 16) + 16 * RC * 16>(hi[x % AHEAD], v_at[y % DB]);
            }
          });
        } else {
          // A weight of zero does not silence what is not finite: one token at a time, kept by the rows that see it.
#pragma unroll 1
          for (int tok = 0; tok < TOK; ++tok) {
            const unsigned h = tok >> 5;
            const u32x4 keep = keep_token(tok, q4);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
              u32x2 lo, hi;
              lds_read_tr_b64<0>(lo, v_at[d] + h * (32 * RC * 16));
              lds_read_tr_b64<16 * RC * 16>(hi, v_at[d] + h * (32 * RC * 16));
              lds_wait<0>(lo, hi);
              const u32x4 v = u32x4{lo[0], lo[1], hi[0], hi[1]} & keep;
#pragma unroll
              for (int r = 0; r < RB; ++r) {
                u32x4 w = __builtin_bit_cast(u32x4, p[r][0]);
                if constexpr (TB == 4) w = (w & (h - 1u)) | (__builtin_bit_cast(u32x4, p[r][1]) & (0u - h));
                const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w & keep), acc[r][d], 0, 0, 0);
                const bool vis = ((there >> (tok >> 4)) & 1) && tok0 + tok < sees[r];
                acc[r][d] = vis ? x : acc[r][d];
              }
            }
          }
        }
        if (more) issue(v_head, vbuf, t + HN_NW);
      }
    }
    if (!items) walk.note(a);

    // ---- the four waves' references, sums and columns, joined through their places ----
    float2* ml = reinterpret_cast<float2*>(ids);
    float* cols = reinterpret_cast<float*>(lds);       // [wave][row][D + 4]
    static_assert(HN_NW * 16 * (D + 4) * 4 <= HN_NW * 2 * HN_TILE && HN_NW * ROWS * 8 <= HN_IDS * 4, "one block of rows at a time");
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      l[r] += lane_xor<16>(l[r], lane);
      l[r] += lane_xor<32>(l[r], lane);
      int any = seen[r];
      any |= __shfl_xor(any, 16);
      any |= __shfl_xor(any, 32);
      heads_close(m[r], l[r], any);
    }
    __syncthreads();                                   // ids and tiles are read
#pragma unroll
    for (int r = 0; r < RB; ++r)
      if (q4 == 0) ml[(wave * RB + r) * 16 + j16] = make_float2(m[r], l[r]);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      if (r > 0) __syncthreads();                      // the block before is read
      float* x = cols + (wave * 16 + j16) * (D + 4) + 4 * q4;
#pragma unroll
      for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(x + 16 * d) = acc[r][d];
      __syncthreads();
      // a thread joins four columns of a row
      for (int y = tid; y < 16 * (D / 4); y += HN_NW * 64) {
        const int j = y / (D / 4), c = 4 * (y % (D / 4)), row = it.row0 + 16 * r + j;
        if (row >= it.rows) continue;
        float2 part[HN_NW];
        float M = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < HN_NW; ++w) {
          part[w] = ml[(w * RB + r) * 16 + j];
          M = fmaxf(M, part[w].x);
        }
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < HN_NW; ++w) {
          const float by = heads_join(M, part[w], sum);
          if (part[w].x != -INFINITY) o += *reinterpret_cast<const f32x4*>(cols + (w * 16 + j) * (D + 4) + c) * by;
        }
        if (walk.whole) {
          const size_t at = (size_t)(it.first + row / a.G) * a.H + it.kvh * a.G + row % a.G;
          const float inv = heads_inverse(sum);
          store4(a.o, at * D + c, a.o_dtype, sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv);
          if (a.lse && c == 0) a.lse[at] = heads_lse(M, sum);
        } else {
          const size_t at = (size_t)walk.slot * ROWS + 16 * r + j;
          *reinterpret_cast<f32x4*>(a.part_acc + at * D + c) = o;
          if (c == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(M, sum);
        }
      }
    }
  } while (!items && walk.find(a));
}

// grid: (items, rows of an item).  The parts of a row in equal shares over groups of D / 4 threads, then over the groups, in a fixed order.  What a thread
// reads of the first parts is on its way before the largest reference of the row is known.
template <int D, int ROWS>
__global__ void __launch_bounds__(256) heads_ranges_merge_kernel(HeadsArgs a) {
  constexpr int LPR = D / 4, GROUPS = 256 / LPR, BATCH = 64 / GROUPS;
  __shared__ f32x4 cols[GROUPS][LPR];
  __shared__ float sums[GROUPS];
  const int item = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, c = tid % LPR, group = tid / LPR;
  const int block = item % a.tiles, v = item / a.tiles, b = v / a.H_kv, kvh = v % a.H_kv, row = block * ROWS + r;
  const int w0 = a.plan[3 * item], parts = a.plan[3 * item + 1], odd = a.plan[3 * item + 2];        // (not looked at for rows that are none)
  int first;
  const int n = heads_new(a, b, first);
  if (row >= n * a.G || parts == 1) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  auto slot = [&](int s) { return (size_t)(2 * (w0 + s) + (s == 0 ? odd : 0)) * ROWS + r; };
  f32x4 x[BATCH];
  float2 part[BATCH];
  auto request = [&](int s0) {
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const size_t at = slot(min(s0 + k * GROUPS, parts - 1));
      part[k] = ml[at];
      x[k] = *reinterpret_cast<const f32x4*>(a.part_acc + at * D + 4 * c);
    }
  };
  request(group);
  float M = -INFINITY;
  for (int s = tid & 63; s < parts; s += 64) M = fmaxf(M, ml[slot(s)].x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) M = fmaxf(M, __shfl_xor(M, d));
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = group; s < parts; s += BATCH * GROUPS) {
    if (s > group) request(s);
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (s + k * GROUPS < parts) {
        const float by = heads_join(M, part[k], sum);
        if (part[k].x != -INFINITY) o += x[k] * by;
      }
  }
  cols[group][c] = o;
  if (c == 0) sums[group] = sum;
  __syncthreads();
  if (group > 0) return;
  for (int g = 1; g < GROUPS; ++g) {
    o += cols[g][c];
    sum += sums[g];
  }
  const size_t at = (size_t)(first + row / a.G) * a.H + kvh * a.G + row % a.G;
  const float inv = heads_inverse(sum);
  store4(a.o, at * D + 4 * c, a.o_dtype, sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * inv);
  if (a.lse && c == 0) a.lse[at] = heads_lse(M, sum);
}

bool heads_mfma_supported(const tpla_heads_t& sh) {
  return sh.dtype == TPLA_BF16 && sh.d_k == sh.d_v && (sh.d_k == 64 || sh.d_k == 128) && sh.page_tokens % 16 == 0;
}
bool heads_ranges_fit(const tpla_heads_t& sh, int32_t max_new) {
  return (int64_t)(sh.H / sh.H_kv) * (max_new > 0 ? max_new : 1) <= HN_MOST;
}

static int ranges_blocks(const tpla_heads_t& sh, int32_t max_new) {        // of 16 rows
  const int64_t rows = (int64_t)(sh.H / sh.H_kv) * (max_new > 0 ? max_new : 1);
  return rows <= 16 ? 1 : 2;
}

// A workgroup per item, nothing to merge: short contexts, by the width of the block table, and longer ones whose items fill the chip.  32 heads on 8, 128 columns: one
// sequence of 100 tokens 10.2 us in ranges, 7.6 so, of 1000 12.4 and 16.0; 32 of 500 21.9 and 14.8, of 2000 50.8 and 44.5; 8 of 1000 (64 items) 16.2 and 16.6.  (Wider tables may hold one
// long sequence among short ones, which only ranges divide.)
static bool items_alone(int64_t tokens, int64_t items) { return tokens <= 512 || (tokens <= 2048 && items >= device_cu_count()); }

HeadsPlan heads_ranges_plan(const tpla_heads_t& sh, int32_t max_new, int32_t max_pages) {
  HeadsPlan p;
  p.kernel = HEADS_RANGES;
  const int rb = ranges_blocks(sh, max_new);
  const int64_t rows = (int64_t)(sh.H / sh.H_kv) * (max_new > 0 ? max_new : 1);
  p.rows = 16 * rb;
  p.tiles = (int)((rows + p.rows - 1) / p.rows);
  p.items = (int64_t)sh.B * sh.H_kv * p.tiles;
  p.n_splits = 1;
  if (items_alone((int64_t)max_pages * sh.page_tokens, p.items)) {
    p.n_wg = 0;
    p.slots = 0;
    p.workspace = 0;
    return p;
  }
  const int tok = HN_TILE / (2 * sh.d_k);
  const double tiles = (double)p.items * (((double)max_pages * sh.page_tokens + tok - 1) / tok + HN_START);
  const int most = device_cu_count() * (rb == 1 ? 2 : 1);
  p.n_wg = (int)std::max(1.0, std::min((double)most, tiles / HN_MIN_UNITS));
  p.slots = 2 * (int64_t)p.n_wg;
  p.workspace = ((size_t)p.slots * p.rows * (sh.d_v + 2) * sizeof(float) + (size_t)p.items * 3 * sizeof(int32_t) + 15) / 16 * 16;
  return p;
}

size_t heads_ranges_room(const tpla_heads_t& sh, int32_t max_new, int32_t max_pages) {
  size_t most = 0;
  for (int32_t n = 1; n <= max_new && heads_ranges_fit(sh, n); ++n) most = std::max(most, heads_ranges_plan(sh, n, max_pages).workspace);
  return most;
}

int launch_heads_ranges(const HeadsArgs& a, const HeadsPlan& p, hipStream_t st) {
  void (*fn)(HeadsArgs);
  void (*merge)(HeadsArgs);
  if (a.d_k == 128) {
    fn = p.rows == 16 ? heads_ranges_kernel<128, 1> : heads_ranges_kernel<128, 2>;
    merge = p.rows == 16 ? heads_ranges_merge_kernel<128, 16> : heads_ranges_merge_kernel<128, 32>;
  } else {
    fn = p.rows == 16 ? heads_ranges_kernel<64, 1> : heads_ranges_kernel<64, 2>;
    merge = p.rows == 16 ? heads_ranges_merge_kernel<64, 16> : heads_ranges_merge_kernel<64, 32>;
  }
  int rc = allow_lds(reinterpret_cast<const void*>(fn), HN_LDS, "heads_ranges_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3((unsigned)(p.n_wg > 0 ? p.n_wg : p.items)), dim3(HN_NW * 64), HN_LDS, st, a);
  if ((rc = check_launch("heads_ranges_kernel"))) return rc;
  if (p.n_wg <= 1) return TPLA_OK;
  const int rows = a.G * (a.cu ? a.max_new : 1);
  hipLaunchKernelGGL(merge, dim3((unsigned)p.items, (unsigned)(rows < p.rows ? rows : p.rows)), dim3(256), 0, st, a);
  return check_launch("heads_ranges_merge_kernel");
}

}  // namespace tpla
