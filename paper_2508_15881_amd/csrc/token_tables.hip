// Bookkeeping of a paged batch on the GPU: pages, slots and positions of new tokens from the request lengths, and the move
// of accepted drafts behind the committed tokens.  Nothing here rounds; both are bound by latency until there are
// hundreds of thousands of tokens.
#include "tpla_internal.h"

namespace tpla {

constexpr int EX_THREADS = 1024;

// Inclusive sum over the workgroup; `carry` is what came before and moves on.  part: EX_THREADS / 64 entries of LDS.
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
  for (int w = 0; w < EX_THREADS / 64; ++w) {
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

// Slot and position of token `at`: sequence b, token i of its n new ones.
__device__ __forceinline__ void place_token(const ExtendArgs& a, int at, int b, int i, int n) {
  const long long t = (long long)clip_int(a.seq_lens[b], (long long)a.max_pages * a.page_tokens) + i;
  int slot = -1, position = 0;
  if (i < n) {
    const long long page = t / a.page_tokens;
    if (page < a.held_out[b])
      slot = a.block_table[(size_t)b * a.max_pages + page] * a.page_tokens + (int)(t - page * a.page_tokens);
    position = clip_int(a.depths ? t - i + a.depths[at] : t, 2147483647LL);
  }
  a.slots[at] = slot;
  a.positions[at] = position;
}

__device__ __forceinline__ void place_tokens(const ExtendArgs& a, int first, int step) {
  for (int at = first; at < a.n_tokens; at += step) {
    if (a.row_tokens) {
      const int b = at / a.row_tokens, i = at - b * a.row_tokens;
      place_token(a, at, b, i, new_tokens(a, b));
      continue;
    }
    int lo = 0, hi = a.B;                            // the last sequence that begins at or before this token
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] <= at) lo = mid; else hi = mid;
    }
    const int end = a.cu[lo + 1];
    place_token(a, at, lo, at - a.cu[lo], at < end ? 2147483647 : 0);
  }
}

// One workgroup: prefix sums over the sequences, the new pages of each, and (few tokens) their slots.
__global__ void __launch_bounds__(EX_THREADS) extend_sequences_kernel(ExtendArgs a, int with_tokens) {
  __shared__ long long part[EX_THREADS / 64];
  __shared__ int need_of[EX_THREADS], held_of[EX_THREADS];
  __shared__ long long first_of[EX_THREADS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long cap = (long long)a.max_pages * a.page_tokens;
  long long tokens = 0, pages = 0;
  for (int b0 = 0; b0 < a.B; b0 += EX_THREADS) {
    const int b = b0 + tid;
    long long n = 0, need = 0;
    int held = 0;
    if (b < a.B) {
      n = new_tokens(a, b);
      held = clip_int(a.held[b], a.max_pages);
      const int L = clip_int(a.seq_lens[b], cap);
      const long long want = min(((long long)L + n + a.page_tokens - 1) / a.page_tokens, (long long)a.max_pages);
      need = max(want - held, 0LL);
    }
    const long long end = block_sum(n, tokens, part), first = block_sum(need, pages, part) - need;
    const int given = clip_int(min(need, a.n_free - first), a.max_pages);
    if (b < a.B) {
      if (b == 0) a.cu[0] = 0;
      a.cu[b + 1] = clip_int(end, a.n_tokens);
      a.held_out[b] = held + given;
    }
    need_of[tid] = given;
    held_of[tid] = held;
    first_of[tid] = first;
    __syncthreads();
    for (int s = wave; s < EX_THREADS && b0 + s < a.B; s += EX_THREADS / 64)
      for (int k = lane; k < need_of[s]; k += 64)
        a.block_table[(size_t)(b0 + s) * a.max_pages + held_of[s] + k] = a.free_pages[first_of[s] + k];
    __syncthreads();
  }
  if (tid == 0) {
    const long long taken = min(pages, (long long)a.n_free);
    a.counts[0] = (int)taken;
    a.counts[1] = clip_int(pages - taken, 2147483647LL);
  }
  if (with_tokens) place_tokens(a, tid, EX_THREADS);
}

__global__ void __launch_bounds__(256) place_tokens_kernel(ExtendArgs a) {
  place_tokens(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

int launch_extend_sequences(const ExtendArgs& a, hipStream_t st) {
  const bool small = a.n_tokens <= 16 * EX_THREADS;
  hipLaunchKernelGGL(extend_sequences_kernel, dim3(1), dim3(EX_THREADS), 0, st, a, small ? 1 : 0);
  int rc = check_launch("extend_sequences_kernel");
  if (rc || small) return rc;
  const int blocks = (int)(((long long)a.n_tokens + 255) / 256);
  hipLaunchKernelGGL(place_tokens_kernel, dim3(blocks), dim3(256), 0, st, a);
  return check_launch("place_tokens_kernel");
}

// One workgroup per sequence.  Row k goes behind the committed ones from draft accepted[k] >= k, so a row that is written was
// read before, in this step or an earlier one: a step reads its rows of all slices, waits, and writes them.
constexpr int CM_THREADS = 512;
__global__ void __launch_bounds__(CM_THREADS) commit_drafts_kernel(CommitArgs a) {
  const int b = blockIdx.x, tid = threadIdx.x;
  const long long cap = (long long)a.max_pages * a.page_tokens;
  const int L = clip_int(a.seq_lens[b], cap);
  const int n = min(clip_int(a.n_accepted[b], a.T), (int)min(cap - L, (long long)a.T));
  const int pieces = a.row_bytes / 16, per_row = pieces * a.n_shards;
  auto row_of = [&](long long t) {
    return (size_t)a.block_table[(size_t)b * a.max_pages + t / a.page_tokens] * a.page_tokens + (size_t)(t % a.page_tokens);
  };
  // whole rows per step, so that no row is written while another thread has yet to read it
  const int step_rows = max(1, CM_THREADS / per_row);
  for (int k0 = 0; k0 < n; k0 += step_rows) {
    const int rows = min(step_rows, n - k0);
    for (int x0 = 0; x0 < rows * per_row; x0 += CM_THREADS) {
      const int x = x0 + tid, k = k0 + x / per_row, c = x % per_row;
      u32x4 v = {0, 0, 0, 0};
      char* dst = nullptr;
      if (x < rows * per_row) {
        const int j = min(max(a.accepted[(size_t)b * a.T + k], 0), a.T - 1);
        if (j != k && L + (long long)j < cap) {
          char* pool = static_cast<char*>(a.pools.p[c / pieces]) + (c % pieces) * 16;
          v = *reinterpret_cast<const u32x4*>(pool + row_of(L + (long long)j) * a.row_bytes);
          dst = pool + row_of(L + (long long)k) * a.row_bytes;
        }
      }
      __syncthreads();
      if (dst) *reinterpret_cast<u32x4*>(dst) = v;
    }
    __syncthreads();
  }
  if (tid == 0) a.new_lens[b] = L + n;
}

int launch_commit_drafts(const CommitArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(commit_drafts_kernel, dim3(a.B), dim3(CM_THREADS), 0, st, a);
  return check_launch("commit_drafts_kernel");
}

}  // namespace tpla
