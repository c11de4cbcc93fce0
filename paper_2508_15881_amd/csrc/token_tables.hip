// Bookkeeping of a paged batch on the GPU: pages, slots and positions of new tokens from the request lengths, and the move
// of accepted drafts behind the committed tokens.  Nothing here rounds; both are bound by latency until there are
// hundreds of thousands of tokens.
#include "tpla_internal.h"

#include <algorithm>

namespace tpla {

constexpr int EX_THREADS = 1024;   // most threads of a workgroup, and sequences per step of the prefix sums
constexpr int EX_BATCH = 4;        // table entries per thread on their way together

// Inclusive sum over the workgroup; `carry` is what came before and moves on.  part: one entry of LDS per wave.
__device__ __forceinline__ long long block_sum(long long v, long long& carry, long long* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  long long before = carry, all = carry;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    if (w < wave) before += part[w];
    all += part[w];
  }
  __syncthreads();
  carry = all;
  return before + v;
}

__device__ __forceinline__ int clip_int(long long v, long long hi) { return (int)(v < 0 ? 0 : (v > hi ? hi : v)); }
__device__ __forceinline__ int new_tokens(const ExtendArgs& a, int b) {
  return clip_int(a.add_lens[b], a.row_tokens ? a.row_tokens : 2147483647LL);
}
__device__ __forceinline__ int held_tokens(const ExtendArgs& a, int b) { return clip_int(a.seq_lens[b], (long long)a.max_pages * a.page_tokens); }

// The last of n ascending values that is not above x; the first is not.
template <typename T>
__device__ __forceinline__ int last_not_above(const T* v, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Slots and positions of EX_BATCH tokens, first, first + step, ..., below a.n_tokens: each is a search among the sequences, their lengths, and a
// table entry.  cu: [B + 1], in LDS or memory.
__device__ __forceinline__ void place_tokens(const ExtendArgs& a, const int32_t* cu, long long first, int step) {
  if (first < a.n_tokens) {
    int slot[EX_BATCH], position[EX_BATCH];
#pragma unroll
    for (int k = 0; k < EX_BATCH; ++k) {
      const int at = (int)min(first + k * step, (long long)a.n_tokens - 1);
      int b, i;
      bool there;
      if (a.row_tokens) {
        b = at / a.row_tokens;
        i = at - b * a.row_tokens;
        there = i < new_tokens(a, b);
      } else {
        b = last_not_above(cu, a.B, at);
        i = at - cu[b];
        there = at < cu[b + 1];
      }
      const int L = held_tokens(a, b);
      const long long t = (long long)L + i, page = t / a.page_tokens;
      const int entry = a.block_table[(size_t)b * a.max_pages + min(page, (long long)a.max_pages - 1)];
      slot[k] = there && page < a.held_out[b] && entry >= 0 ? entry * a.page_tokens + (int)(t - page * a.page_tokens) : -1;
      position[k] = there ? clip_int(a.depths ? (long long)L + a.depths[at] : t, 2147483647LL) : 0;
    }
#pragma unroll
    for (int k = 0; k < EX_BATCH; ++k)
      if (first + k * step < a.n_tokens) {
        a.slots[first + k * step] = slot[k];
        a.positions[first + k * step] = position[k];
      }
  }
}

// One workgroup: prefix sums over the sequences and the new pages of each.
__global__ void __launch_bounds__(EX_THREADS) extend_sequences_kernel(ExtendArgs a) {
  __shared__ long long part[EX_THREADS / 64];
  __shared__ long long first_of[EX_THREADS];         // pages wanted before a sequence of this step, and of those given
  __shared__ int held_of[EX_THREADS];
  const int tid = threadIdx.x, n_thr = blockDim.x;
  long long tokens = 0, pages = 0;
  for (int b0 = 0; b0 < a.B; b0 += n_thr) {
    const int b = b0 + tid, here = min(n_thr, a.B - b0);
    long long n = 0, need = 0;
    int held = 0;
    if (b < a.B) {
      n = new_tokens(a, b);
      held = clip_int(a.held[b], a.max_pages);
      const int L = held_tokens(a, b);
      const long long want = min(((long long)L + n + a.page_tokens - 1) / a.page_tokens, (long long)a.max_pages);
      need = max(want - held, 0LL);
    }
    const long long pages_before = min(pages, (long long)a.n_free);
    const long long end = block_sum(n, tokens, part), first = block_sum(need, pages, part) - need;
    const long long from = min(first, (long long)a.n_free), given = min(first + need, (long long)a.n_free) - from;
    if (b < a.B) {
      if (b == 0) a.cu[0] = 0;
      a.cu[b + 1] = clip_int(end, a.n_tokens);
      a.held_out[b] = held + (int)given;
      for (long long k = given; k < need; ++k) a.block_table[(size_t)b * a.max_pages + held + k] = -1;      // no page: see extend_together_kernel
    }
    first_of[tid] = from;
    held_of[tid] = held;
    __syncthreads();
    // all pages of this step, whoever they go to
    const long long pages_end = min(pages, (long long)a.n_free);
    for (long long x0 = pages_before + tid; x0 < pages_end; x0 += EX_BATCH * n_thr) {
      int page[EX_BATCH];
#pragma unroll
      for (int k = 0; k < EX_BATCH; ++k) page[k] = a.free_pages[min(x0 + k * n_thr, pages_end - 1)];
#pragma unroll
      for (int k = 0; k < EX_BATCH; ++k) {
        const long long x = x0 + k * n_thr;
        if (x < pages_end) {
          const int s = last_not_above(first_of, here, x);      // (of sequences that begin at the same page the last is the one that gets it)
          a.block_table[(size_t)(b0 + s) * a.max_pages + held_of[s] + (x - first_of[s])] = page[k];
        }
      }
    }
    __syncthreads();
  }
  if (tid == 0) {
    const long long taken = min(pages, (long long)a.n_free);
    a.counts[0] = (int)taken;
    a.counts[1] = clip_int(pages - taken, 2147483647LL);
  }
}

__global__ void __launch_bounds__(256) place_tokens_kernel(ExtendArgs a) {
  __shared__ int cu_of[EX_THREADS + 1];
  const bool local = a.row_tokens == 0 && a.B <= EX_THREADS;
  if (local) {
    for (int b = threadIdx.x; b <= a.B; b += 256) cu_of[b] = a.cu[b];
    __syncthreads();
  }
  // the tokens of a workgroup lie side by side: few sequences, whole lines of slots
  place_tokens(a, local ? cu_of : a.cu, (long long)blockIdx.x * (256 * EX_BATCH) + threadIdx.x, 256);
}

// The usual case, at most EX_ROOM sequences, in one launch: every workgroup takes the prefix sums over all sequences for itself (their lengths
// are one round trip to memory, another kernel is two and a launch), then its share of the tokens and of the pages.  A token in a new page
// finds it in the list of free ones, so nothing waits for the table.  pages_held is read by all of them: where it is also the output there
// has to be one workgroup only.
constexpr int EX_ROOM = 1024, EX_ONE = 256, EX_TOKENS = 1024;
__global__ void __launch_bounds__(EX_ONE) extend_together_kernel(ExtendArgs a) {
  __shared__ long long part[EX_ONE / 64];
  __shared__ int cu_of[EX_ROOM + 1], from_of[EX_ROOM], held_of[EX_ROOM], length_of[EX_ROOM], given_of[EX_ROOM], need_of[EX_ROOM];
  const int tid = threadIdx.x;
  const unsigned cap = (unsigned)a.max_pages * (unsigned)a.page_tokens, pt = a.page_tokens;       // below 2^31
  long long tokens = 0, pages = 0;
  if (tid == 0) cu_of[0] = 0;
  for (int b0 = 0; b0 < a.B; b0 += EX_ONE) {
    const int b = b0 + tid;
    int n = 0, need = 0, held = 0, L = 0;
    if (b < a.B) {
      n = new_tokens(a, b);
      held = clip_int(a.held[b], a.max_pages);
      L = held_tokens(a, b);
      const unsigned last = (unsigned)min((long long)L + n, (long long)cap);
      need = max((int)((last + pt - 1) / pt) - held, 0);
    }
    const long long end = block_sum(n, tokens, part), first = block_sum(need, pages, part) - need;
    if (b < a.B) {
      cu_of[b + 1] = clip_int(end, a.n_tokens);
      from_of[b] = (int)min(first, (long long)a.n_free);
      given_of[b] = (int)min((long long)need, max(a.n_free - first, 0LL));
      need_of[b] = need;
      held_of[b] = held;
      length_of[b] = L;
    }
  }
  __syncthreads();                                   // (and every length and count is read)
  if (blockIdx.x == 0) {
    for (int b = tid; b <= a.B; b += EX_ONE) {
      a.cu[b] = cu_of[b];
      if (b < a.B) {
        a.held_out[b] = held_of[b] + given_of[b];
        // A page that was not there is -1 and not whatever the row held: what reads the row knows that these tokens have no place.
        for (int k = given_of[b]; k < need_of[b]; ++k) a.block_table[(size_t)b * a.max_pages + held_of[b] + k] = -1;
      }
    }
    const long long taken = min(pages, (long long)a.n_free);
    if (tid == 0) a.counts[0] = (int)taken;
    if (tid == 1) a.counts[1] = clip_int(pages - taken, 2147483647LL);
  }
  const int n_taken = (int)min(pages, (long long)a.n_free), step = gridDim.x * EX_ONE;
  for (int x0 = blockIdx.x * EX_ONE + tid; x0 < n_taken; x0 += EX_BATCH * step) {
    int page[EX_BATCH];
#pragma unroll
    for (int k = 0; k < EX_BATCH; ++k) page[k] = a.free_pages[min((long long)x0 + (long long)k * step, (long long)n_taken - 1)];
#pragma unroll
    for (int k = 0; k < EX_BATCH; ++k) {
      const long long x = (long long)x0 + (long long)k * step;
      if (x >= n_taken) break;
      const int b = last_not_above(from_of, a.B, (int)x);       // (of sequences that begin at the same page the last is the one that gets it)
      a.block_table[(size_t)b * a.max_pages + held_of[b] + ((int)x - from_of[b])] = page[k];
    }
    if ((long long)x0 + (long long)EX_BATCH * step >= n_taken) break;
  }
  const int begin = blockIdx.x * EX_TOKENS, stop = (int)min((long long)a.n_tokens, (long long)begin + EX_TOKENS);
  int entry[EX_TOKENS / EX_ONE], offset[EX_TOKENS / EX_ONE], position[EX_TOKENS / EX_ONE];
#pragma unroll
  for (int k = 0; k < EX_TOKENS / EX_ONE; ++k) {
    const int at = begin + k * EX_ONE + tid;
    entry[k] = -1;
    offset[k] = position[k] = 0;
    if (at >= stop) continue;
    int b, i;
    bool there;
    if (a.row_tokens) {
      b = (unsigned)at / (unsigned)a.row_tokens;
      i = at - b * a.row_tokens;
      there = i < new_tokens(a, b);
    } else {
      b = last_not_above(cu_of, a.B, at);
      i = at - cu_of[b];
      there = at < cu_of[b + 1];
    }
    const long long t = (long long)length_of[b] + i;
    if (!there) continue;
    position[k] = clip_int(a.depths ? (long long)length_of[b] + a.depths[at] : t, 2147483647LL);
    if (t >= (long long)cap) continue;
    const int page = (int)((unsigned)t / pt), fresh = page - held_of[b];
    if (fresh >= given_of[b]) continue;
    offset[k] = (int)((unsigned)t - (unsigned)page * pt);
    entry[k] = fresh < 0 ? a.block_table[(size_t)b * a.max_pages + page] : a.free_pages[(long long)from_of[b] + fresh];
  }
#pragma unroll
  for (int k = 0; k < EX_TOKENS / EX_ONE; ++k) {
    const int at = begin + k * EX_ONE + tid;
    if (at >= stop) continue;
    a.slots[at] = entry[k] < 0 ? -1 : entry[k] * a.page_tokens + offset[k];
    a.positions[at] = position[k];
  }
}

int launch_extend_sequences(const ExtendArgs& a, hipStream_t st) {
  const int blocks = std::max((int)(((long long)a.n_tokens + EX_TOKENS - 1) / EX_TOKENS), 1);
  if (a.B <= EX_ROOM && (blocks == 1 || a.held != a.held_out)) {
    hipLaunchKernelGGL(extend_together_kernel, dim3(blocks), dim3(EX_ONE), 0, st, a);
    return check_launch("extend_together_kernel");
  }
  hipLaunchKernelGGL(extend_sequences_kernel, dim3(1), dim3(EX_THREADS), 0, st, a);
  const int rc = check_launch("extend_sequences_kernel");
  if (rc || a.n_tokens == 0) return rc;
  hipLaunchKernelGGL(place_tokens_kernel, dim3(blocks), dim3(256), 0, st, a);
  return check_launch("place_tokens_kernel");
}

// One workgroup per sequence.  Row k goes behind the committed ones from draft accepted[k] >= k, so a row that is written was
// read before, in this step or an earlier one: a step reads its rows of all slices (CM_BATCH pieces of 16 bytes per thread, on their way
// together), waits for all of the workgroup, and writes them.  Where every row lies is found once, by a thread each.
// (kernel alone, 240 sequences with up to 60 rows of four slices: 256 threads of 16 pieces 12.7 us, 512 of 8 8.5, 1024 of 8 7.1; with the
// check of the pages 7.3)
constexpr int CM_THREADS = 1024, CM_BATCH = 8;
__global__ void __launch_bounds__(CM_THREADS) commit_drafts_kernel(CommitArgs a) {
  __shared__ long long src_of[TPLA_MAX_DRAFTS], dst_of[TPLA_MAX_DRAFTS];      // byte offsets in a pool; -1: stays where it is
  __shared__ int n_of;
  const int b = blockIdx.x, tid = threadIdx.x;
  const unsigned cap = (unsigned)a.max_pages * (unsigned)a.page_tokens, pt = a.page_tokens;       // below 2^31
  const int picked = tid < a.T ? a.accepted[(size_t)b * a.T + tid] : 0;
  const int L = clip_int(a.seq_lens[b], cap);
  if (tid < 64) {                                    // (one wave: a draft each)
    int n = min(clip_int(a.n_accepted[b], a.T), (int)min(cap - L, (unsigned)a.T));
    bool placed = true;
    if (tid < n) {
      const int j = min(max(picked, 0), a.T - 1);
      const unsigned from = (unsigned)L + j, to = (unsigned)L + tid;
      const int32_t* table = a.block_table + (size_t)b * a.max_pages;
      const bool there = from < cap, moves = j != tid && there;
      const int to_page = table[to / pt], from_page = table[min(from, cap - 1) / pt];
      placed = to_page >= 0 && (from_page >= 0 || !there);
      src_of[tid] = moves ? ((long long)from_page * pt + from % pt) * a.row_bytes : -1;
      dst_of[tid] = ((long long)to_page * pt + to % pt) * a.row_bytes;
    }
    // a draft without a page was never written: the path ends before it
    const unsigned long long absent = __ballot(!placed);
    if (absent) n = __builtin_ctzll(absent);
    if (tid == 0) n_of = n;
  }
  __syncthreads();
  const int n = n_of;
  if (tid == 0) a.new_lens[b] = L + n;               // (every wave has read the length that it may replace)
  const unsigned pieces = a.row_bytes / 16, per_row = pieces * a.n_shards;
  // whole rows per step, so that no row is written while another thread has yet to read it; a row wider than a step goes in parts, whose
  // pieces are their own
  const int step_rows = max(1u, CM_THREADS * CM_BATCH / per_row);
  for (int k0 = 0; k0 < n; k0 += step_rows) {
    const int all = min(step_rows, n - k0) * per_row;
    for (int x0 = 0; x0 < all; x0 += CM_THREADS * CM_BATCH) {
      u32x4 v[CM_BATCH];
      char* dst[CM_BATCH];
#pragma unroll
      for (int e = 0; e < CM_BATCH; ++e) {
        const unsigned x = x0 + e * CM_THREADS + tid, k = k0 + x / per_row, c = x % per_row;
        dst[e] = nullptr;
        if ((int)x < all && src_of[k] >= 0) {
          const unsigned i = c / pieces;
          char* pool = static_cast<char*>(i == 0 ? a.pools.p[0] : i == 1 ? a.pools.p[1] : i == 2 ? a.pools.p[2] : i == 3 ? a.pools.p[3] :
                                          i == 4 ? a.pools.p[4] : i == 5 ? a.pools.p[5] : i == 6 ? a.pools.p[6] : a.pools.p[7]) + (c - i * pieces) * 16;
          v[e] = *reinterpret_cast<const u32x4*>(pool + src_of[k]);
          dst[e] = pool + dst_of[k];
        }
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < CM_BATCH; ++e)
        if (dst[e]) *reinterpret_cast<u32x4*>(dst[e]) = v[e];
    }
    __syncthreads();
  }
}

int launch_commit_drafts(const CommitArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(commit_drafts_kernel, dim3(a.B), dim3(CM_THREADS), 0, st, a);
  return check_launch("commit_drafts_kernel");
}

}  // namespace tpla
