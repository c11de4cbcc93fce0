// Attention of drafted tokens on the matrix cores: bf16, slices of 64, 128, 256 or 512 columns, 64 of RoPE key.
//
// The T H rows of a (slice, sequence) all read the same cache rows, so the rows are the MFMA N dimension and a tile of 32 tokens
// is shared by everything the workgroup holds:
//   S^T[token, row] = K[token, :] . Q[row, :]           M = tokens (LDS), N = rows (Q in registers for the whole item)
//   O^T[dim, row]  += V^T[dim, token] . P^T[token, row]  V = the first dl columns of the same LDS rows, read transposed
// A workgroup is 4 waves of RB blocks of 16 rows.  Every wave reads the whole tile from LDS, and a fragment it reads feeds RB
// MFMAs: RB decides how far LDS keeps up with the matrix cores.
//
// All 32-token tiles of all items (slice, sequence, row block) are laid end to end and cut into equal ranges, one per workgroup;
// an item that lies in one range is written at once, the others leave partial results for the merge (tree.hip).
#include "lds_tile.h"

#include <float.h>

#include <algorithm>

namespace tpla {

constexpr int TR_TOK = 32;           // tokens per tile
constexpr int TR_NW = 4;
// Page ids in LDS: chunks of 256 in a ring of 4.  A chunk is a whole number of tiles, at least 8, whatever the page size.  The
// first tile of a chunk to be requested requests the ids of the next one: at most NSTAGE - 1 tiles are requested between two
// barriers, so what is overwritten (three chunks back) is read by nobody, and the ids have arrived when 8 tiles later the
// first of them is read (the wait for the tile after the request covers them).
constexpr int TR_IDS = 256, TR_ID_RING = 4 * TR_IDS;

// QL: every second k-step, the first QL of them, of the queries lies in LDS and not in registers.
template <int DL, int RB, int QL>
struct TreeTile {
  static constexpr int RC = (DL + 64) / 8;             // 16-byte pieces per row
  static constexpr int BYTES = TR_TOK * RC * 16;
  static constexpr int CPT = TR_TOK * RC / 64 / TR_NW;  // direct-to-LDS loads per wave and tile
  static constexpr int Q_BYTES = TR_NW * RB * QL * 1024;
  static constexpr int FIT = (158 * 1024 - Q_BYTES - TR_ID_RING * 4) / BYTES;
  static constexpr int NSTAGE = FIT < 8 ? FIT : 8;      // tiles in flight or in use; at most 8 (see TR_IDS)
  static constexpr int IDS = NSTAGE * BYTES, Q = IDS + TR_ID_RING * 4, CLEANED = Q + Q_BYTES, LDS = CLEANED + 16;
  static_assert(TR_TOK * RC % (64 * TR_NW) == 0, "every wave issues the same number of loads");
  static_assert(NSTAGE >= 4, "a tile whose values are read, two whose scores are, and one on its way");
};

// LDS reads of the score product, in program order: K fragments x = 2 ks + tb, KRING of them ahead; the queries of an LDS
// k-step at the first fragment of the k-step before; V fragments (two reads each) in place of the last KRING K fragments.
// How many reads are younger than what fragment x needs when it is waited for (LDS answers in order).
template <int KS, int QL, int RB, int KRING>
struct ScoreReads {
  static constexpr int NQ = 2 * KS;
  static constexpr bool in_lds(int ks) { return ks < KS && (ks & 1) && ks / 2 < QL; }
  static constexpr int in_regs(int ks) { return ks - (ks / 2 < QL ? ks / 2 : QL); }       // index among the k-steps in registers
  static constexpr int q_reads(int x) { return x % 2 == 0 && in_lds(x / 2 + 1) ? RB : 0; }
  static constexpr int tail_reads(int x, bool with_v) { return x + KRING < NQ ? 1 : (with_v ? 2 : 0); }
  static constexpr int younger(int x, bool with_v) {
    int issued = KRING, need = x < KRING ? x : -1;
    for (int y = 0; y <= x; ++y) {
      issued += q_reads(y);
      if (x % 2 == 0 && in_lds(x / 2) && y == x - 2 && issued - 1 > need) need = issued - 1;   // the queries of this k-step
      if (y < x) {
        if (y + KRING == x && issued > need) need = issued;
        issued += tail_reads(y, with_v);
      }
    }
    return issued - need - 1;
  }
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
// Units of sequence b: `unit` tokens of one row block are a tile, and an item is its tiles behind START units that hold none.
// Those stand for what an item costs a workgroup besides its tiles (its queries, the first tiles' way from memory, its result),
// so that ranges with many short items end with the others.
struct TreeUnits {
  TreeLens len;
  int tiles, blocks;           // no drafts: none
};
__device__ __forceinline__ TreeUnits tree_units(const TreeArgs& a, int unit, int b) {
  TreeUnits r;
  if (b >= a.B) {
    r.len = TreeLens{0, 0, 0};
    r.tiles = r.blocks = 0;
    return r;
  }
  r.len = tree_lens(a, b);
  r.tiles = r.len.n > 0 ? max((r.len.keys + unit - 1) / unit, 1) : 0;
  r.blocks = (r.len.n * a.H + a.p.block - 1) / a.p.block;
  return r;
}

// The range of units of this workgroup, [pos, end), and the item that unit `pos` lies in.
template <int UNIT, int START>
struct TreeWalk {
  TreeUnits front;             // the first 64 sequences stay in the lanes: a search among them loads nothing
  int front_incl, per_slice, units, n_wg, w, pos, range0, end;
  // the item
  int i, b, v, item, rb, rows, L, keys, tiles, t0, t1, slot, last;
  bool whole;

  static __device__ __forceinline__ int units_of(const TreeUnits& u) { return u.blocks * (u.tiles + START); }
  __device__ __forceinline__ bool begin(const TreeArgs& a) {
    const int lane = threadIdx.x & 63;
    front = tree_units(a, UNIT, lane);
    front_incl = tree_prefix(units_of(front));
    per_slice = __builtin_amdgcn_readlane(front_incl, 63);
    int tiles_all = __builtin_amdgcn_readlane(tree_prefix(front.blocks * front.tiles), 63);
    for (int b0 = 64; b0 < a.B; b0 += 64) {
      const TreeUnits u = tree_units(a, UNIT, b0 + lane);
      per_slice += __builtin_amdgcn_readlane(tree_prefix(units_of(u)), 63);
      tiles_all += __builtin_amdgcn_readlane(tree_prefix(u.blocks * u.tiles), 63);
    }
    units = per_slice * a.n_shards;
    n_wg = max(1, min(a.p.n_wg, tiles_all * a.n_shards / a.p.split_tokens));             // no shorter ranges than pay
    // ranges that lie side by side (the row blocks of a sequence, which read the same pages) on one XCD: workgroups go to the eight in turn
    w = n_wg % 8 == 0 ? (blockIdx.x & 7) * (n_wg >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    if ((int)blockIdx.x >= n_wg || units == 0) return false;
    range0 = pos = tree_start(n_wg, units, w);
    end = tree_start(n_wg, units, w + 1);
    return true;
  }
  // The next item with tiles in the range; false: there is none.
  __device__ __forceinline__ bool find(const TreeArgs& a) {
    const int lane = threadIdx.x & 63;
    while (pos < end) {
      i = pos / per_slice;
      const int rem = pos - i * per_slice;
      b = 0;
      TreeUnits u = front;
      int incl = front_incl;
      unsigned long long past = __ballot(incl > rem);
      while (past == 0) {                            // ends: rem lies below the sum over all sequences
        b += 64;
        const int base = __builtin_amdgcn_readlane(incl, 63);
        u = tree_units(a, UNIT, b + lane);
        incl = tree_prefix(units_of(u)) + base;
        past = __ballot(incl > rem);
      }
      const int src = __builtin_ctzll(past);
      b += src;
      const int before = __builtin_amdgcn_readlane(incl - units_of(u), src);
      tiles = __builtin_amdgcn_readlane(u.tiles, src);
      const int span = tiles + START;
      rb = (rem - before) / span;
      const int at = rem - before - rb * span, stop = min(span, at + (end - pos));
      t0 = max(at - START, 0);
      t1 = stop - START;
      const int first = pos;
      pos += stop - at;
      last = first - at + span - 1;
      if (t1 <= t0) continue;                        // the range ends before the item's first tile
      L = __builtin_amdgcn_readlane(u.len.L, src);
      keys = __builtin_amdgcn_readlane(u.len.keys, src);
      rows = __builtin_amdgcn_readlane(u.len.n, src) * a.H;
      v = i * a.B + b;
      item = v * a.p.blocks + rb;
      whole = t0 == 0 && t1 == tiles;
      slot = 2 * w + (first == range0 ? 0 : 1);
      return true;
    }
    return false;
  }
  // Where the merge finds the item's results: whoever has its first tile says so, once its first loads are on their way (512 rows, 64-wide
  // slices: 352 us ahead of them, 347 so).
  __device__ __forceinline__ void note(const TreeArgs& a) const {
    if (t0 != 0 || threadIdx.x != 0) return;
    a.plan[3 * item] = w;
    a.plan[3 * item + 1] = tree_owner(n_wg, units, last) - w + 1;
    a.plan[3 * item + 2] = slot & 1;
  }
};

// ---- matrix instructions on registers of our choice ----
// The output accumulators are the accumulation registers a0 .. themselves, quad N of them at a[4 N : 4 N + 3], and everything else
// stays in the other 256.  Left to the compiler the accumulators exist twice (a branch may rescale them, and it copies them over for
// every tile so that this branch finds them in ordinary registers): no room for 64 rows a wave.  So both products and what else touches
// the accumulators are written out, with the wait states that the compiler then does not insert: 2 between an ordinary write and a
// matrix instruction that reads it, 11 (here 18) between a matrix instruction and an ordinary one that reads its result.
// acc_keep() stands at every step of the loop: nothing of the compiler's may live in these registers across it.  That it puts nothing
// there in between either is checked on the assembly (tests/test_isa_tree_waits.py), and so are the wait states on every path
// (tests/test_isa_tree_results.py).
#define TR_ACC_REGS \
  "a0", "a1", "a2", "a3", "a4", "a5", "a6", "a7", "a8", "a9", "a10", "a11", "a12", "a13", "a14", "a15", "a16", "a17", "a18", "a19", "a20", "a21", "a22", \
  "a23", "a24", "a25", "a26", "a27", "a28", "a29", "a30", "a31", "a32", "a33", "a34", "a35", "a36", "a37", "a38", "a39", "a40", "a41", "a42", "a43", \
  "a44", "a45", "a46", "a47", "a48", "a49", "a50", "a51", "a52", "a53", "a54", "a55", "a56", "a57", "a58", "a59", "a60", "a61", "a62", "a63", "a64", \
  "a65", "a66", "a67", "a68", "a69", "a70", "a71", "a72", "a73", "a74", "a75", "a76", "a77", "a78", "a79", "a80", "a81", "a82", "a83", "a84", "a85", \
  "a86", "a87", "a88", "a89", "a90", "a91", "a92", "a93", "a94", "a95", "a96", "a97", "a98", "a99", "a100", "a101", "a102", "a103", "a104", "a105", \
  "a106", "a107", "a108", "a109", "a110", "a111", "a112", "a113", "a114", "a115", "a116", "a117", "a118", "a119", "a120", "a121", "a122", "a123", \
  "a124", "a125", "a126", "a127", "a128", "a129", "a130", "a131", "a132", "a133", "a134", "a135", "a136", "a137", "a138", "a139", "a140", "a141", \
  "a142", "a143", "a144", "a145", "a146", "a147", "a148", "a149", "a150", "a151", "a152", "a153", "a154", "a155", "a156", "a157", "a158", "a159", \
  "a160", "a161", "a162", "a163", "a164", "a165", "a166", "a167", "a168", "a169", "a170", "a171", "a172", "a173", "a174", "a175", "a176", "a177", \
  "a178", "a179", "a180", "a181", "a182", "a183", "a184", "a185", "a186", "a187", "a188", "a189", "a190", "a191", "a192", "a193", "a194", "a195", \
  "a196", "a197", "a198", "a199", "a200", "a201", "a202", "a203", "a204", "a205", "a206", "a207", "a208", "a209", "a210", "a211", "a212", "a213", \
  "a214", "a215", "a216", "a217", "a218", "a219", "a220", "a221", "a222", "a223", "a224", "a225", "a226", "a227", "a228", "a229", "a230", "a231", \
  "a232", "a233", "a234", "a235", "a236", "a237", "a238", "a239", "a240", "a241", "a242", "a243", "a244", "a245", "a246", "a247", "a248", "a249", \
  "a250", "a251", "a252", "a253", "a254", "a255"
__device__ __forceinline__ void acc_keep() {
#ifdef __HIP_DEVICE_COMPILE__                         // (the host's compiler does not know the names)
  asm volatile("" : : : TR_ACC_REGS);
#endif
}
__device__ __forceinline__ void mm_first(f32x4& s, const bf16x8& k, const bf16x8& q) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
}
__device__ __forceinline__ void mm_score(f32x4& s, const bf16x8& k, const bf16x8& q) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
template <int N>
__device__ __forceinline__ void mm_out(const u32x4& v, const bf16x8& p) {
  asm volatile("v_mfma_f32_16x16x32_bf16 a[%2:%3], %0, %1, a[%2:%3]" : : "v"(v), "v"(p), "n"(4 * N), "n"(4 * N + 3));
}
__device__ __forceinline__ void mm_settle_write() { asm volatile("s_nop 1" ::: "memory"); }
__device__ __forceinline__ void mm_settle_result() { asm volatile("s_nop 15\n\ts_nop 1" ::: "memory"); }
template <int N>
__device__ __forceinline__ void acc_zero() {
  asm volatile("v_accvgpr_write_b32 a[%0], 0\n\tv_accvgpr_write_b32 a[%1], 0\n\tv_accvgpr_write_b32 a[%2], 0\n\tv_accvgpr_write_b32 a[%3], 0"
               : : "n"(4 * N), "n"(4 * N + 1), "n"(4 * N + 2), "n"(4 * N + 3));
}
template <int A>
__device__ __forceinline__ float acc_read_one() {
  float x;
  asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(x) : "n"(A));
  return x;
}
template <int N>
__device__ __forceinline__ f32x4 acc_read() {
  const float x = acc_read_one<4 * N>(), y = acc_read_one<4 * N + 1>(), z = acc_read_one<4 * N + 2>(), w = acc_read_one<4 * N + 3>();
  return f32x4{x, y, z, w};
}
template <int A>
__device__ __forceinline__ void acc_scale_one(float by) {
  float t;
  asm volatile("v_accvgpr_read_b32 %0, a[%2]\n\tv_mul_f32 %0, %0, %1\n\tv_accvgpr_write_b32 a[%2], %0" : "=&v"(t) : "v"(by), "n"(A));
}
template <int N>
__device__ __forceinline__ void acc_scale(float by) {
  acc_scale_one<4 * N>(by);
  acc_scale_one<4 * N + 1>(by);
  acc_scale_one<4 * N + 2>(by);
  acc_scale_one<4 * N + 3>(by);
}

__device__ __forceinline__ unsigned lds_read_id(unsigned addr) {
  unsigned id;
  asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(id) : "v"(addr) : "memory");
  return id;
}

// The value, made known here: what is computed from it on a rare path is not computed ahead of the loop and kept.
template <typename T>
__device__ __forceinline__ T here(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Zero for what is not finite among two bfloat16.
__device__ __forceinline__ unsigned finite_pair(unsigned u) {
  if ((u & 0x7F80u) == 0x7F80u) u &= 0xFFFF0000u;
  if ((u & 0x7F800000u) == 0x7F800000u) u &= 0xFFFFu;
  return u;
}

template <int DL, int RB, int QL>
__global__ void __launch_bounds__(TR_NW * 64, 1) tree_mfma_kernel(TreeArgs a) {
  using Tile = TreeTile<DL, RB, QL>;
  constexpr int RC = Tile::RC, CPT = Tile::CPT, NSTAGE = Tile::NSTAGE;
  constexpr int KS = (DL + 64) / 32, DB = DL / 16, NQ = 2 * KS;
  constexpr int RING = 4;                              // K and V fragments on their way
  constexpr int PAIRS = RB * 4;                        // pairs of weights per lane and tile
  using Reads = ScoreReads<KS, QL, RB, RING>;
  extern __shared__ u32x4 smem[];
  char* const lds = reinterpret_cast<char*>(smem);
  volatile int* const cleaned = reinterpret_cast<volatile int*>(lds + Tile::CLEANED);      // some value of this item's tiles was
  const unsigned lds_base = lds_at(lds);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j16 = lane & 15, q4 = lane >> 4;

  // A small item costs 7 us besides 0.95 a tile (R = 64, 4 sequences of 300 to 600 tokens: 32.3 us without start units, 29.3 with
  // six; one user of 1237 tokens 40.1 and 36.2).  The wide blocks' items are long: start units cost them 2 % (8192 tokens, 512 rows,
  // 64-wide slices: 352 and 360; 192 rows, 256-wide ones: 184 and 188).
  TreeWalk<TR_TOK, RB == 1 ? 6 : 0> walk;
  if (!walk.begin(a)) return;

  // ---- per-lane LDS offsets: rows begin at whole 128 bytes, so that the pieces of a row differ in address bits 4 to 6 alone ----
  static_assert(RC % 8 == 0, "rows of whole 128 bytes");
  const unsigned k_off = (unsigned)((j16 * RC + (q4 ^ swz(j16))) * 16);
  const int v_tok = 4 * q4 + (j16 >> 2);
  const unsigned v_off = (unsigned)((v_tok * RC + (((j16 & 3) >> 1) ^ swz(v_tok))) * 16 + (j16 & 1) * 8);
  const unsigned lds_q = lds_base + Tile::Q + wave * (RB * QL * 1024) + lane * 16;
  unsigned ld_at[CPT];                                 // byte of this lane's piece within a page that holds the tile's 32 rows
#pragma unroll
  for (int j = 0; j < CPT; ++j) {
    const int x = (wave + j * TR_NW) * 64 + lane, tok = x / RC;
    ld_at[j] = (unsigned)(tok * (RC * 16) + ((x % RC) ^ swz(tok)) * 16);
  }
  const int pt = a.page_tokens, shift = (pt & (pt - 1)) == 0 ? __builtin_ctz(pt) : -1;
  auto page_of = [&](int t) { return shift >= 0 ? t >> shift : t / pt; };
  const bool one_page = pt % TR_TOK == 0;              // a tile never crosses a page

  while (walk.find(a)) {
    const int i = walk.i, b = walk.b, v = walk.v, rb = walk.rb, L = walk.L, keys = walk.keys, rows = walk.rows, t0 = walk.t0, t1 = walk.t1;
    const int row0 = rb * a.p.block + wave * (16 * RB);          // this wave's first row
    const bool alive = row0 < rows;
    const int all_rows = a.T * a.H;
    const char* pool = static_cast<const char*>(tree_pool(a, i));
    const int32_t* table = a.block_table + (size_t)b * a.max_pages;

    // ---- page ids and tiles on their way ----
    int chunk = page_of(t0 * TR_TOK) / TR_IDS;
    auto request_ids = [&](int c) {
      const int p = min(c * TR_IDS + wave * 64 + lane, a.max_pages - 1);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(table + p),
                                       (__attribute__((address_space(3))) void*)(lds + Tile::IDS + ((c & 3) * TR_IDS + wave * 64) * 4), 4, 0, 0);
    };
    auto id_at = [&](int p) { return lds_base + Tile::IDS + (unsigned)(p & (TR_ID_RING - 1)) * 4; };
    auto id_of = [&](int t) { return id_at(page_of(t * TR_TOK)); };
    auto issue = [&](int t, unsigned id) {           // id: page of the tile, where tiles do not cross pages
      const int k0 = t * TR_TOK, p0 = __builtin_amdgcn_readfirstlane(page_of(k0));
      char* dst = lds + (t % NSTAGE) * Tile::BYTES + wave * 1024;
      if (one_page && k0 + TR_TOK <= keys) {
        const int page = max(__builtin_amdgcn_readfirstlane(id), 0);
        const char* src = pool + ((size_t)page * pt + (k0 - p0 * pt)) * (RC * 16);
#pragma unroll
        for (int j = 0; j < CPT; ++j)
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + ld_at[j]),
                                           (__attribute__((address_space(3))) void*)(dst + j * TR_NW * 1024), 16, 0, 0);
      } else {
        // rows of several pages, or past the end: those repeat the last token (and are masked)
#pragma unroll 1
        for (int j = 0; j < CPT; ++j) {
          const int x = (wave + j * TR_NW) * 64 + here(lane), tok = x / RC, k = min(k0 + tok, keys - 1), p = page_of(k);
          const int row_id = max((int)lds_read_id(id_at(p)), 0);
          const char* src = pool + ((size_t)row_id * pt + (k - p * pt)) * (RC * 16) + ((x % RC) ^ swz(tok)) * 16;
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                           (__attribute__((address_space(3))) void*)(dst + j * TR_NW * 1024), 16, 0, 0);
        }
      }
      const int c = p0 / TR_IDS;
      if (c != chunk) {
        chunk = c;
        request_ids(c + 1);
      }
    };
    lds_barrier();                                   // the item before this one no longer reads LDS
    if (tid == 0) *cleaned = 0;
    request_ids(chunk);
    request_ids(chunk + 1);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __builtin_amdgcn_s_barrier();
    for (int t = t0; t < t1 && t < t0 + NSTAGE - 1; ++t) issue(t, lds_read_id(id_of(t)));
    walk.note(a);

    // In the middle of the values of tile t: tile t + 2 is there for all waves, tile t - 1 is no longer read by any and another takes its place.
    auto arrived = [&](int t) {
      if (t + NSTAGE - 2 < t1)
        __builtin_amdgcn_s_waitcnt(vmcnt_imm((NSTAGE - 4) * CPT));
      else
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __builtin_amdgcn_s_barrier();
    };
    auto refill = [&](int t, unsigned id) {
      if (t + NSTAGE - 1 < t1) issue(t + NSTAGE - 1, id);
    };
    // Values of drafts are masked per row, and a weight of zero does not silence an infinity or a NaN: what is not finite in tile t becomes
    // zero here, behind its scores and ahead of the product with its weights.  The merge makes it good for the rows that see such a draft; it is told
    // by the sign of the partial sums, or by -1 workgroups of an item that one has whole.
    auto clean = [&](int t) {
      lds_barrier();
#pragma unroll 1
      for (int x = here(tid); x < TR_TOK * RC; x += TR_NW * 64) {
        const int tok = x / RC, c = (x % RC) ^ swz(tok);
        if (c >= DL / 8 || t * TR_TOK + tok < L) continue;
        u32x4* at = smem + (t % NSTAGE) * (TR_TOK * RC) + x;
        const u32x4 was = *at, u = {finite_pair(was[0]), finite_pair(was[1]), finite_pair(was[2]), finite_pair(was[3])};
        if (((u[0] ^ was[0]) | (u[1] ^ was[1]) | (u[2] ^ was[2]) | (u[3] ^ was[3])) == 0) continue;
        *at = u;
        *cleaned = 1;
      }
      lds_barrier();
    };
    auto first_tiles = [&]() {                       // tiles t0 and t0 + 1 are there
      if (t0 + NSTAGE - 2 < t1)
        __builtin_amdgcn_s_waitcnt(vmcnt_imm((NSTAGE - 3) * CPT));
      else
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __builtin_amdgcn_s_barrier();
    };

    if (!alive) {                                    // no rows: this wave only loads
      first_tiles();
      for (int t = t0; t < t1; ++t) {
        if ((t + 1) * TR_TOK > L) clean(t);
        if (t == t1 - 1) break;
        arrived(t);
        refill(t, lds_read_id(id_of(t + NSTAGE - 1)));
      }
      continue;
    }

    int entry = draft_entry(a, b, page_of(L + lane));
    // ---- queries as B operands: block r, lane holds row row0 + 16 r + j16 ----
    bf16x8 q[RB][KS - QL];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const int row = min(row0 + 16 * r + j16, rows - 1);
      const bf16_t* ql = static_cast<const bf16_t*>(a.q_lat) + ((size_t)v * all_rows + row) * DL + q4 * 8;
      const bf16_t* qp = static_cast<const bf16_t*>(a.q_pe) + ((size_t)b * all_rows + row) * 64 + q4 * 8;
      __builtin_amdgcn_sched_barrier(0);             // one block's addresses at a time
      static_for<KS>([&](auto ic) {
        constexpr int ks = decltype(ic)::value;
        const bf16x8 x = *reinterpret_cast<const bf16x8*>(ks * 32 < DL ? ql + ks * 32 : qp + (ks * 32 - DL));
        if constexpr (Reads::in_lds(ks))
          *reinterpret_cast<bf16x8*>(lds + Tile::Q + ((wave * RB + r) * QL + ks / 2) * 1024 + lane * 16) = x;
        else
          q[r][Reads::in_regs(ks)] = x;
      });
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));        // complete before the loop: nothing there waits for them
    asm volatile("" : "+v"(entry));
    first_tiles();

    f32x4 s[RB][2], next[RB][2];
    // The reference starts at the lowest finite number: every finite score moves it, -inf keeps weight 0 against it.
    float m_run[RB], l_run[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      m_run[r] = -FLT_MAX;
      l_run[r] = 0.f;
      next[r][0] = next[r][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    static_for<RB * DB>([](auto n) { acc_zero<decltype(n)::value>(); });
    acc_keep();
    u32x2 vlo[RING], vhi[RING];
    auto read_v = [&](auto ic, unsigned va) {
      constexpr int d = decltype(ic)::value;
      lds_read_tr_b64<(d >> 2) * 128>(vlo[d % RING], va ^ ((d & 3) << 5));
      lds_read_tr_b64<(d >> 2) * 128 + 16 * RC * 16>(vhi[d % RING], va ^ ((d & 3) << 5));
    };
    bf16x8 kf[RING];
    auto read_k = [&](auto ic, unsigned ka) {
      constexpr int x = decltype(ic)::value, ks = x / 2, tb = x % 2;
      lds_read_b128<(ks >> 1) * 128 + tb * (16 * RC * 16)>(kf[x % RING], ka ^ ((ks & 1) << 6));
    };
    // Scores of a tile (at ka), whose first RING fragments are on their way; slice(x) runs behind fragment x.  with_v: the first V fragments
    // (at va) follow the last K fragments.
    auto scores = [&](unsigned ka, f32x4 (&s)[RB][2], auto with_v, unsigned va, auto&& slice) {
      constexpr bool WV = decltype(with_v)::value;
      bf16x8 qf[RB];
      static_for<NQ>([&](auto ic) {
        constexpr int x = decltype(ic)::value, ks = x / 2, tb = x % 2;
        if constexpr (Reads::q_reads(x) > 0)
          static_for<RB>([&](auto rc) {
            constexpr int r = decltype(rc)::value;
            lds_read_b128<(r * QL + (ks + 1) / 2) * 1024>(qf[r], lds_q);
          });
        lds_wait<Reads::younger(x, WV)>(kf[x % RING]);
        if constexpr (Reads::in_lds(ks) && tb == 0)
#pragma unroll
          for (int r = 0; r < RB; ++r) lds_wait<Reads::younger(x, WV)>(qf[r]);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          if constexpr (ks == 0)
            mm_first(s[r][tb], kf[x % RING], q[r][0]);
          else if constexpr (Reads::in_lds(ks))
            mm_score(s[r][tb], kf[x % RING], qf[r]);
          else
            mm_score(s[r][tb], kf[x % RING], q[r][Reads::in_regs(ks)]);
        }
        if constexpr (x + RING < NQ)
          read_k(std::integral_constant<int, x + RING>{}, ka);
        else if constexpr (WV)
          read_v(std::integral_constant<int, x + RING - NQ>{}, va);
        slice(ic);
        acc_keep();
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto top_of = [&](const f32x4 (&s)[RB][2], int r) {
      float m = fmaxf(s[r][0][0], s[r][0][1]);
#pragma unroll
      for (int e = 2; e < 8; ++e) m = fmaxf(m, s[r][e >> 2][e & 3]);
      return m * a.scale_log2;
    };
    unsigned long long over = 0;                     // lanes with a score of the next tile far above their reference
    auto look = [&](const f32x4 (&s)[RB][2], int r) { over |= __ballot(top_of(s, r) > m_run[r] + LAZY); };
    auto tile_at = [&](int t) { return lds_base + (unsigned)((t % NSTAGE) * Tile::BYTES); };

    // One tile: its scores are in s; the scores of the next one go into next under the exponentials of this one.
    auto step = [&](int t, auto last_tile) {
      constexpr bool LAST = decltype(last_tile)::value;
      if ((t + 1) * TR_TOK > L) {                    // drafts, or past the end: masked here, and looked at again
        over = 0;
        const unsigned long long there = drafts_there(here(entry));
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const int row = min(row0 + 16 * r + here(j16), rows - 1);
          const unsigned long long bits = a.mask[(size_t)b * a.T + row / a.H] & there;
#pragma unroll
          for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int k = t * TR_TOK + 16 * tb + 4 * here(q4) + e, j = k - L;
              if (j >= 0 && (k >= keys || !((bits >> (j & 63)) & 1))) s[r][tb][e] = -INFINITY;
            }
          look(s, r);
        }
        clean(t);
      }
      if (over) {
        mm_settle_result();
        static_for<RB>([&](auto rc) {
          constexpr int r = decltype(rc)::value;
          float m = top_of(s, r);
          m = fmaxf(m, __shfl_xor(m, 16));
          m = fmaxf(m, __shfl_xor(m, 32));
          m = fmaxf(m, m_run[r]);
          const float alpha = __builtin_amdgcn_exp2f(m_run[r] - m);
          l_run[r] *= alpha;
          m_run[r] = m;
          static_for<DB>([&](auto d) { acc_scale<r * DB + decltype(d)::value>(alpha); });
          acc_keep();
        });
        mm_settle_write();
        over = 0;
      }
      // weights: lane = one row per block, tokens 32 t + 16 tb + 4 q4 + e.  They go into the second product in bf16, at most 2^-8
      // off each; their sum is that of the unrounded ones, so that lse has float accuracy
      bf16x8 pb[RB];
      auto weights = [&](auto pc) {
        constexpr int p = decltype(pc)::value, r = p / 4, tb = (p % 4) / 2, e = 2 * (p % 2);
        const float x = __builtin_amdgcn_exp2f(fmaf(s[r][tb][e], a.scale_log2, -m_run[r]));
        const float y = __builtin_amdgcn_exp2f(fmaf(s[r][tb][e + 1], a.scale_log2, -m_run[r]));
        l_run[r] += x + y;
        pb[r][4 * tb + e] = (bf16_t)x;
        pb[r][4 * tb + e + 1] = (bf16_t)y;
        acc_keep();
      };
      const unsigned va = tile_at(t) + v_off;
      if constexpr (!LAST) {
        scores(tile_at(t + 1) + k_off, next, std::true_type{}, va, [&](auto ic) {
          constexpr int x = decltype(ic)::value, p0 = x * PAIRS / NQ, p1 = (x + 1) * PAIRS / NQ;
          static_for<p1 - p0>([&](auto k) { weights(std::integral_constant<int, p0 + decltype(k)::value>{}); });
        });
      } else {
        static_for<RING>([&](auto ic) { lds_wait<0>(kf[decltype(ic)::value]); });     // (of no tile)
        static_for<RING>([&](auto ic) { read_v(ic, va); });
        static_for<PAIRS>(weights);
      }

      // O^T += V^T P^T; under it the next tile's maxima, the tile after that arrives, and its first K fragments (of whatever lies there behind the
      // last tile) follow the last V fragments
      const unsigned ka = tile_at(t + 2) + k_off;
      unsigned id;
      constexpr int middle = DB / 2 < DB - RING ? DB / 2 : DB - RING;
      static_for<DB>([&](auto ic) {
        constexpr int d = decltype(ic)::value, left = DB - 1 - d;
        if constexpr (!LAST && d == middle) {
          arrived(t);
          asm volatile("ds_read_b32 %0, %1" : "=v"(id) : "v"(id_of(t + NSTAGE - 1)) : "memory");
        }
        lds_wait<2 * (left < RING - 1 ? left : RING - 1) + (!LAST && RING - 1 - left > 0 ? RING - 1 - left : 0)>(vlo[d % RING], vhi[d % RING]);
        const u32x4 v4 = {vlo[d % RING][0], vlo[d % RING][1], vhi[d % RING][0], vhi[d % RING][1]};
        if constexpr (d == 0) {
#pragma unroll
          for (int r = 0; r < RB; ++r) asm volatile("" : "+v"(pb[r]));      // written before the wait states
          mm_settle_write();
        }
        static_for<RB>([&](auto r) { mm_out<decltype(r)::value * DB + d>(v4, pb[decltype(r)::value]); });
        acc_keep();
        if constexpr (d + RING < DB)
          read_v(std::integral_constant<int, d + RING>{}, va);
        else if constexpr (!LAST)
          read_k(std::integral_constant<int, d + RING - DB>{}, ka);
        if constexpr (!LAST && d == DB - 1) {                 // (the wait for the last V fragment covered the page id)
          asm volatile("" : "+v"(id));
          refill(t, id);
        }
        // the scores of the next tile are complete: 64 clocks of matrix instructions and more lie behind their last one
        constexpr int from = DB - RB > 4 ? DB - RB : DB;
        if constexpr (!LAST && d >= from) look(next, d - from);
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (LAST) return;
      if constexpr (DB - RB <= 4) {
        mm_settle_result();
#pragma unroll
        for (int r = 0; r < RB; ++r) look(next, r);
      }
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) s[r][tb] = next[r][tb];
    };

    {
      static_for<RING>([&](auto ic) { read_k(ic, tile_at(t0) + k_off); });
      scores(tile_at(t0) + k_off, s, std::false_type{}, 0u, [](auto) {});
      static_for<RING>([&](auto ic) { read_k(ic, tile_at(t0 + 1) + k_off); });
      mm_settle_result();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < RB; ++r) look(s, r);
    }
#pragma unroll 1
    for (int t = t0; t < t1 - 1; ++t) step(t, std::false_type{});
    step(t1 - 1, std::true_type{});

    // ---- the item's result, or a partial one ----
    mm_settle_result();
    const int was_cleaned = *cleaned;
    if (was_cleaned && walk.whole && tid == 0) a.plan[3 * walk.item + 1] = -1;
    static_for<RB>([&](auto rc) {
      constexpr int r = decltype(rc)::value;
      const int local = wave * (16 * RB) + 16 * r + here(j16), row = rb * a.p.block + local;
      float l = l_run[r];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      const bool there = row < rows;
      if (walk.whole && __any(l == 0.f)) {
        const unsigned long long drafts = drafts_there(here(entry));
        if (there && l == 0.f && (L > 0 || drafts_seen(a, b, row / a.H, L, keys, drafts) != 0)) l = __builtin_nanf("");
      }
      const float inv = walk.whole ? (l != 0.f ? 1.0f / l : 0.f) : 1.f;
      float* out = walk.whole ? a.o_lat + ((size_t)v * all_rows + row) * DL : a.part_acc + ((size_t)walk.slot * a.p.block + local) * DL;
      static_for<DB>([&](auto dc) {
        constexpr int d = decltype(dc)::value;
        const f32x4 x = acc_read<r * DB + d>() * inv;
        if (there) *reinterpret_cast<f32x4*>(out + 16 * d + 4 * q4) = x;
      });
      acc_keep();
      if (there && q4 == 0) {
        if (!walk.whole)
          *reinterpret_cast<float2*>(a.part_ml + 2 * ((size_t)walk.slot * a.p.block + local)) = make_float2(m_run[r], was_cleaned ? -l : l);
        else if (a.lse)
          a.lse[(size_t)v * all_rows + row] = l != 0.f ? (m_run[r] + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
    });
  }
}

// ---------------------------------------------------------------------------
// Few rows: up to 64 (TEAMS = 2) or 128 (TEAMS = 1) per item.  What bounds these is how fast one compute unit gets through its cache rows, and a
// single wave per SIMD leaves most of its time to waits.  Here 8 waves share rounds of 64 tokens, two waves per SIMD: one's matrix products run
// under the other's exponentials and reads.  A wave has 16 rows.  Where an item has fewer blocks of 16 than there are waves, the waves left over
// take the second 32 tokens of every round for the first blocks, and what both have is joined through LDS at the end of the item (with TEAMS = 2
// that is every block).  Waves 0 .. 3 lie on different SIMDs, so few blocks have one each: 64 x 8192 tokens, 16 rows: 121 us with the second wave on
// another SIMD, 142 with it on the same; 80 rows: 212 with five waves, 198 with eight.
constexpr int TP_NW = 8, TP_TOK = 64;

template <int DL>
struct PairTile {
  static constexpr int RC = (DL + 64) / 8;
  static constexpr int BYTES = TP_TOK * RC * 16;       // a round
  static constexpr int CPT = TP_TOK * RC / 64 / TP_NW;
  static constexpr int NSTAGE = 3;
  static constexpr int IDS = NSTAGE * BYTES, CLEANED = IDS + TR_ID_RING * 4, LDS = CLEANED + 16;
  static_assert(TP_TOK * RC % (64 * TP_NW) == 0, "every wave issues the same number of loads");
  static_assert(4 * (DL / 16 + 1) * 1024 <= NSTAGE * BYTES, "the join of two teams fits the ring");
};

template <int DL, int TEAMS>
__global__ void __launch_bounds__(TP_NW * 64, 2) tree_pair_kernel(TreeArgs a) {
  using Tile = PairTile<DL>;
  constexpr int RC = Tile::RC, CPT = Tile::CPT, NSTAGE = Tile::NSTAGE;
  constexpr int KS = (DL + 64) / 32, DB = DL / 16;
  constexpr int KRING = 6, VRING = 4;
  // streaming, not kept in L2 (32 x 32768 tokens, 64 rows: 284 -> 271 us with merge and combine; 64 x 8192, 80 rows: 204 -> 198; eight blocks of
  // 128 rows, which find the rows of each other in the last-level cache, lose nothing)
  constexpr int STREAM = 2;
  extern __shared__ u32x4 smem[];
  char* const lds = reinterpret_cast<char*>(smem);
  volatile int* const cleaned = reinterpret_cast<volatile int*>(lds + Tile::CLEANED);      // some value of this item's tiles was
  const unsigned lds_base = lds_at(lds);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j16 = lane & 15, q4 = lane >> 4;
  TreeWalk<TP_TOK, 0> walk;                            // (rounds are long: four start units gain nothing for 16 heads and lose 2 % for 64 rows of 32768 tokens)
  if (!walk.begin(a)) return;

  const unsigned k_off = (unsigned)((j16 * RC + (q4 ^ swz(j16))) * 16);
  const int v_tok = 4 * q4 + (j16 >> 2);
  const unsigned v_off = (unsigned)((v_tok * RC + (((j16 & 3) >> 1) ^ swz(v_tok))) * 16 + (j16 & 1) * 8);
  unsigned ld_at[CPT];                                 // byte of this lane's piece within a page that holds the round's 64 rows
#pragma unroll
  for (int j = 0; j < CPT; ++j) {
    const int x = (wave + j * TP_NW) * 64 + lane, tok = x / RC;
    ld_at[j] = (unsigned)(tok * (RC * 16) + ((x % RC) ^ swz(tok)) * 16);
  }
  const int pt = a.page_tokens, shift = (pt & (pt - 1)) == 0 ? __builtin_ctz(pt) : -1;
  auto page_of = [&](int t) { return shift >= 0 ? t >> shift : t / pt; };
  const bool one_page = pt % TP_TOK == 0;

  while (walk.find(a)) {
    const int b = walk.b, v = walk.v, L = walk.L, keys = walk.keys, rows = walk.rows, t0 = walk.t0, t1 = walk.t1;
    // Blocks of 16 rows; where there are fewer than waves, the first `joined` have a second wave, which takes the other half of every round.
    const int n_blocks = min((rows - walk.rb * a.p.block + 15) / 16, TP_NW), joined = min(n_blocks, TP_NW - n_blocks);
    const int team = wave < n_blocks ? 0 : 1, member = team ? wave - n_blocks : wave;
    const bool alive = wave < n_blocks + joined, both = member >= joined;
    const int row0 = walk.rb * a.p.block + member * 16, all_rows = a.T * a.H;
    const char* pool = static_cast<const char*>(tree_pool(a, walk.i));
    const int32_t* table = a.block_table + (size_t)b * a.max_pages;

    // ---- page ids and rounds on their way (as in the kernel above; a chunk of ids is at least 4 rounds, 2 are requested ahead) ----
    int chunk = page_of(t0 * TP_TOK) / TR_IDS;
    auto request_ids = [&](int c) {
      if (wave >= TR_IDS / 64) return;
      const int p = min(c * TR_IDS + wave * 64 + lane, a.max_pages - 1);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(table + p),
                                       (__attribute__((address_space(3))) void*)(lds + Tile::IDS + ((c & 3) * TR_IDS + wave * 64) * 4), 4, 0, 0);
    };
    auto id_at = [&](int p) { return lds_base + Tile::IDS + (unsigned)(p & (TR_ID_RING - 1)) * 4; };
    auto issue = [&](int t) {
      const int k0 = t * TP_TOK, p0 = __builtin_amdgcn_readfirstlane(page_of(k0));
      char* dst = lds + (t % NSTAGE) * Tile::BYTES + wave * 1024;
      if (one_page && k0 + TP_TOK <= keys) {
        const int page = max(__builtin_amdgcn_readfirstlane(lds_read_id(id_at(p0))), 0);
        const char* src = pool + ((size_t)page * pt + (k0 - p0 * pt)) * (RC * 16);
#pragma unroll
        for (int j = 0; j < CPT; ++j)
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + ld_at[j]),
                                           (__attribute__((address_space(3))) void*)(dst + j * TP_NW * 1024), 16, 0, STREAM);
      } else {
        // rows of several pages, or past the end: those repeat the last token (and are masked)
#pragma unroll 1
        for (int j = 0; j < CPT; ++j) {
          const int x = (wave + j * TP_NW) * 64 + here(lane), tok = x / RC, k = min(k0 + tok, keys - 1), p = page_of(k);
          const int row_id = max((int)lds_read_id(id_at(p)), 0);
          const char* src = pool + ((size_t)row_id * pt + (k - p * pt)) * (RC * 16) + ((x % RC) ^ swz(tok)) * 16;
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                           (__attribute__((address_space(3))) void*)(dst + j * TP_NW * 1024), 16, 0, STREAM);
        }
      }
      const int c = p0 / TR_IDS;
      if (c != chunk) {
        chunk = c;
        request_ids(c + 1);
      }
    };
    lds_barrier();                                   // the item before this one no longer reads LDS
    if (tid == 0) *cleaned = 0;
    request_ids(chunk);
    request_ids(chunk + 1);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __builtin_amdgcn_s_barrier();
    for (int t = t0; t < t1 && t < t0 + NSTAGE - 1; ++t) issue(t);
    walk.note(a);

    const int entry = draft_entry(a, b, page_of(L + lane));
    bf16x8 q[KS];
    {
      const int row = min(row0 + j16, rows - 1);
      const bf16_t* ql = static_cast<const bf16_t*>(a.q_lat) + ((size_t)v * all_rows + row) * DL + q4 * 8;
      const bf16_t* qp = static_cast<const bf16_t*>(a.q_pe) + ((size_t)b * all_rows + row) * 64 + q4 * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8*>(ks * 32 < DL ? ql + ks * 32 : qp + (ks * 32 - DL));
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[ks]));   // complete before the loop
    }
    const unsigned long long there = drafts_there(entry);
    f32x4 acc[DB];
    float m_run = -FLT_MAX, l_run = 0.f;             // see the kernel above
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto clean = [&](int t) {                        // round t; see the kernel above
      lds_barrier();
#pragma unroll 1
      for (int x = here(tid); x < TP_TOK * RC; x += TP_NW * 64) {
        const int tok = x / RC, c = (x % RC) ^ swz(tok);
        if (c >= DL / 8 || t * TP_TOK + tok < L) continue;
        u32x4* at = smem + (t % NSTAGE) * (TP_TOK * RC) + x;
        const u32x4 was = *at, u = {finite_pair(was[0]), finite_pair(was[1]), finite_pair(was[2]), finite_pair(was[3])};
        if (((u[0] ^ was[0]) | (u[1] ^ was[1]) | (u[2] ^ was[2]) | (u[3] ^ was[3])) == 0) continue;
        *at = u;
        *cleaned = 1;
      }
      lds_barrier();
    };

    // 32 SUBS tokens of round t, from its token 32 sub on.  (Both halves at once, not one after the other: one wait for the first fragments, one
    // step of the softmax, four independent sums.)
    auto tile_of = [&](auto subs, int t, int sub) {
      constexpr int SUBS = decltype(subs)::value, TB = 2 * SUBS, N = KS * TB, NV = DB * SUBS;
      const unsigned tile = lds_base + (unsigned)((t % NSTAGE) * Tile::BYTES + sub * (32 * RC * 16));
      const bool tail = (t + 1) * TP_TOK > L;
      f32x4 s[TB];
#pragma unroll
      for (int tb = 0; tb < TB; ++tb) s[tb] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (alive) {
        bf16x8 kf[KRING];
        const unsigned ka = tile + k_off;
        auto read_k = [&](auto ic) {
          constexpr int x = decltype(ic)::value, ks = x / TB, tb = x % TB;
          lds_read_b128<(ks >> 1) * 128 + tb * (16 * RC * 16)>(kf[x % KRING], ka ^ ((ks & 1) << 6));
        };
        static_for<KRING>(read_k);
        static_for<N>([&](auto ic) {
          constexpr int x = decltype(ic)::value, left = N - 1 - x;
          lds_wait<(left < KRING - 1 ? left : KRING - 1)>(kf[x % KRING]);
          s[x % TB] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[x % KRING], q[x / TB], s[x % TB], 0, 0, 0);
          if constexpr (x + KRING < N) read_k(std::integral_constant<int, x + KRING>{});
        });
      }
      if (tail) clean(t);
      if (!alive) return;
      u32x2 vlo[VRING], vhi[VRING];
      const unsigned va = tile + v_off;
      auto read_v = [&](auto ic) {                   // block d of the columns, 32 tokens of it
        constexpr int x = decltype(ic)::value, d = x / SUBS, at = (x % SUBS) * (32 * RC * 16) + (d >> 2) * 128;
        lds_read_tr_b64<at>(vlo[x % VRING], va ^ ((d & 3) << 5));
        lds_read_tr_b64<at + 16 * RC * 16>(vhi[x % VRING], va ^ ((d & 3) << 5));
      };
      if (tail) {
        const int row = min(row0 + here(j16), rows - 1);
        const unsigned long long bits = a.mask[(size_t)b * a.T + row / a.H] & there;
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = t * TP_TOK + 32 * sub + 16 * tb + 4 * here(q4) + e, j = k - L;
            if (j >= 0 && (k >= keys || !((bits >> (j & 63)) & 1))) s[tb][e] = -INFINITY;
          }
      }
      static_for<VRING>(read_v);
      float mx = fmaxf(s[0][0], s[0][1]);
#pragma unroll
      for (int e = 2; e < 4 * TB; ++e) mx = fmaxf(mx, s[e >> 2][e & 3]);
      mx *= a.scale_log2;
      if (__any(mx > m_run + LAZY)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        mx = fmaxf(mx, m_run);
        const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
        l_run *= alpha;
        m_run = mx;
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] *= alpha;
      }
      bf16x8 pb[SUBS];                               // weights in bf16, their sum from the unrounded ones
#pragma unroll
      for (int e = 0; e < 4 * TB; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3], a.scale_log2, -m_run));
        l_run += p;
        pb[e >> 3][e & 7] = (bf16_t)p;
      }
      static_for<NV>([&](auto ic) {
        constexpr int x = decltype(ic)::value, d = x / SUBS, left = NV - 1 - x;
        lds_wait<2 * (left < VRING - 1 ? left : VRING - 1)>(vlo[x % VRING], vhi[x % VRING]);
        const u32x4 v4 = {vlo[x % VRING][0], vlo[x % VRING][1], vhi[x % VRING][0], vhi[x % VRING][1]};
        acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v4), pb[x % SUBS], acc[d], 0, 0, 0);
        if constexpr (x + VRING < NV) read_v(std::integral_constant<int, x + VRING>{});
      });
    };

    for (int t = t0; t < t1; ++t) {
      if (t + 1 < t1)
        __builtin_amdgcn_s_waitcnt(vmcnt_imm((NSTAGE - 2) * CPT));
      else
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __builtin_amdgcn_s_barrier();                  // round t is there for all waves, round t - 1 is no longer read
      if (t + NSTAGE - 1 < t1) issue(t + NSTAGE - 1);
      if constexpr (TEAMS == 1) {
        if (both) {
          tile_of(std::integral_constant<int, 2>{}, t, 0);
          continue;
        }
      }
      tile_of(std::integral_constant<int, 1>{}, t, team);
    }

    // ---- the halves of a block's tokens, then the result ----
    if (joined > 0) {
      lds_barrier();                                 // the last round is no longer read
      char* const at = lds + member * ((DB + 1) * 1024) + lane * 16;
      if (alive && team == 1) {
#pragma unroll
        for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(at + d * 1024) = acc[d];
        *reinterpret_cast<float2*>(at + DB * 1024) = make_float2(m_run, l_run);
      }
      lds_barrier();
      if (team == 1) continue;
      if (!both) {
        const float2 ml = *reinterpret_cast<const float2*>(at + DB * 1024);
        const float m = fmaxf(m_run, ml.x), mine = __builtin_amdgcn_exp2f(m_run - m), theirs = __builtin_amdgcn_exp2f(ml.x - m);
        m_run = m;
        l_run = l_run * mine + ml.y * theirs;
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = acc[d] * mine + *reinterpret_cast<const f32x4*>(at + d * 1024) * theirs;
      }
    }
    const int was_cleaned = *cleaned;
    if (was_cleaned && walk.whole && tid == 0) a.plan[3 * walk.item + 1] = -1;
    float l = l_run;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const int local = member * 16 + j16, row = row0 + j16;
    if (!alive || row >= rows) continue;
    if (walk.whole && l == 0.f && (L > 0 || drafts_seen(a, b, row / a.H, L, keys, there) != 0)) l = __builtin_nanf("");
    const float inv = walk.whole ? (l != 0.f ? 1.0f / l : 0.f) : 1.f;
    float* out = walk.whole ? a.o_lat + ((size_t)v * all_rows + row) * DL : a.part_acc + ((size_t)walk.slot * a.p.block + local) * DL;
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(out + 16 * d + 4 * q4) = acc[d] * inv;
    if (q4 == 0) {
      if (!walk.whole)
        *reinterpret_cast<float2*>(a.part_ml + 2 * ((size_t)walk.slot * a.p.block + local)) = make_float2(m_run, was_cleaned ? -l : l);
      else if (a.lse)
        a.lse[(size_t)v * all_rows + row] = l != 0.f ? (m_run + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
  }
}

bool tree_mfma_supported(const tpla_shape_t& sh) {
  const int dl = sh.d_c / sh.g;
  return sh.dtype == TPLA_BF16 && sh.d_r == 64 && (dl == 64 || dl == 128 || dl == 256 || dl == 512);
}

// The kernel and the rows of an item, from the rows R of a sequence and the 32-token tiles of 64 rows per compute unit (by the block table's width:
// the host does not know the lengths).  Best of three runs of 8 calls with their merge, us, over batches of 1 to 64 sequences of 300 to 32768 tokens
// (lengths from two thirds of that on):
//   little work: 64 rows on 4 waves (A).  More workgroups, shorter prologues, smaller partial results.  256-wide, 16 x 1237 tokens: R = 128 A 31,
//     128 rows on 8 waves (B) 43, 192 rows (C) 47; 16 x 4096, R = 80 to 192 A 45 to 62, B 50 to 67.  64-wide slices pass sooner: one sequence of 8192,
//     R = 80 A 26.5, B 23.4
//   up to 64 rows: two teams of 4 waves (D).  64 x 8192 tokens, R = 48: 256-wide A 130.5, D 126.9, B 140; 128-wide 168.6 / 167.4 / 175; 64-wide 282 / 260 / 274
//   more: B, or C (256 rows of narrower slices) where its blocks are filled and long enough.  256-wide: R = 80, 64 x 8192: B 161, C 211; R = 192 315 / 247; 64 x
//     2048: R = 384 171 / 170, 512 206 / 219.  128-wide, R = 1024: 64 x 2048 489 / 473, 16 x 1237 113 / 125; R = 192, 64 x 2048 135 / 143; 64-wide 741 / 730, 164 / 173.
// Per tile C takes 1.45 (256-wide) and 1.95 (narrower) times what B takes for a full block, and B's last block half of that and what its rows add.
// (128 rows on 4 waves were up to 13 % slower than B and not kept.)  512-wide slices have A alone: the accumulators of more rows do not fit.
void tree_mfma_plan(const tpla_shape_t& sh, int n_shards, int T, int max_pages, TreePlan* p) {
  const int dl = sh.d_c / sh.g, rows = T * sh.H, large = dl == 256 ? 192 : 256, cus = device_cu_count();
  const double tiles = std::max(((double)max_pages * sh.page_tokens + TR_TOK - 1) / TR_TOK, 1.0), per_row_block = (double)n_shards * sh.B * tiles / cus;
  const auto blocks = [&](int of) { return (rows + of - 1) / of; };
  p->mfma = 1;
  p->teams = 0;
  p->block = 64;
  if (dl < 512 && per_row_block * blocks(64) >= (dl == 64 ? 14 : 40)) {
    p->teams = rows <= 64 ? 2 : 1;
    p->block = 128 / p->teams;
    const double pair = rows / 128 + (rows % 128 ? 0.5 + rows % 128 / 256.0 : 0.0), wide = blocks(large) * (dl == 256 ? 1.45 : 1.95);
    if (rows > 128 && per_row_block * blocks(large) >= (dl == 256 ? 24 : 100) && wide < pair) {
      p->teams = 0;
      p->block = large;
    }
  }
  p->blocks = blocks(p->block);
  p->n_wg = (int)std::min((double)cus, (double)n_shards * sh.B * p->blocks * tiles);
  p->n_splits = 1;
  p->split_tokens = 4;         // fewest units of a range: a partial result costs as much as some (one user of 1237 tokens, R = 64: 4 tiles 21 us, 8 25)
}

template <int DL, int RB, int QL = 0>
static int launch_tree(const TreeArgs& a, hipStream_t st) {
  const auto fn = tree_mfma_kernel<DL, RB, QL>;
  constexpr int lds = TreeTile<DL, RB, QL>::LDS;
  const int rc = allow_lds(reinterpret_cast<const void*>(fn), lds, "tree_mfma_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3(a.p.n_wg), dim3(TR_NW * 64), lds, st, a);
  return check_launch("tree_mfma_kernel");
}

template <int DL, int TEAMS>
static int launch_pair(const TreeArgs& a, hipStream_t st) {
  const auto fn = tree_pair_kernel<DL, TEAMS>;
  constexpr int lds = PairTile<DL>::LDS;
  const int rc = allow_lds(reinterpret_cast<const void*>(fn), lds, "tree_pair_kernel");
  if (rc) return rc;
  hipLaunchKernelGGL(fn, dim3(a.p.n_wg), dim3(TP_NW * 64), lds, st, a);
  return check_launch("tree_pair_kernel");
}

int launch_tree_mfma(const TreeArgs& a, hipStream_t st) {
  if (a.p.teams) {
    switch (a.dl * 8 + a.p.teams) {
      case 64 * 8 + 1: return launch_pair<64, 1>(a, st);
      case 64 * 8 + 2: return launch_pair<64, 2>(a, st);
      case 128 * 8 + 1: return launch_pair<128, 1>(a, st);
      case 128 * 8 + 2: return launch_pair<128, 2>(a, st);
      case 256 * 8 + 1: return launch_pair<256, 1>(a, st);
      case 256 * 8 + 2: return launch_pair<256, 2>(a, st);
    }
    return fail(TPLA_ERR_UNSUPPORTED, "no kernel of %d teams for slices of %d columns", a.p.teams, a.dl);
  }
  switch (a.dl * 8 + a.p.block / 64) {
    case 64 * 8 + 1: return launch_tree<64, 1>(a, st);
    case 64 * 8 + 4: return launch_tree<64, 4, 1>(a, st);
    case 128 * 8 + 1: return launch_tree<128, 1>(a, st);
    case 128 * 8 + 4: return launch_tree<128, 4, 3>(a, st);
    case 256 * 8 + 1: return launch_tree<256, 1>(a, st);
    case 256 * 8 + 3: return launch_tree<256, 3, 2>(a, st);
    case 512 * 8 + 1: return launch_tree<512, 1>(a, st);
  }
  return fail(TPLA_ERR_UNSUPPORTED, "no kernel for slices of %d columns in blocks of %d rows", a.dl, a.p.block);
}

}  // namespace tpla
