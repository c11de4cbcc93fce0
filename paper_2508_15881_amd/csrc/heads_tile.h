// What the matrix-core kernels of grouped heads share: tiles of keys and of values of 32 or 64 tokens in LDS, rows of 128 or 256 bytes.
#pragma once
#include "lds_tile.h"
#include "heads.h"

namespace tpla {

// Place of the 16-byte pieces of row `tok` within the row: piece c lies at c ^ heads_swz(tok).  Rows of 256 bytes begin at the same bank, so
// that the four rows of a transposing read must differ by two pieces at least, and the eight of a row-wise one by one; rows of 128 bytes
// alternate between the halves of the banks.
template <int RC>
__device__ __forceinline__ int heads_swz(int tok) {
  if constexpr (RC == 16) return ((tok & 3) << 1) | ((tok >> 2) & 1) | (tok & 8);
  return tok & 7;
}

// Read and waited for here: left to the compiler, a read of LDS waits for the direct loads on their way.
__device__ __forceinline__ int lds_read_page(const int* at) {
  int id;
  asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(id) : "v"(lds_at(reinterpret_cast<const char*>(at))) : "memory");
  return id;
}
template <int N>
__device__ __forceinline__ void loads_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// Whether two bfloat16 hold an infinity or a NaN.
__device__ __forceinline__ bool not_finite_pair(unsigned u) { return (u & 0x7F80u) == 0x7F80u || (u & 0x7F800000u) == 0x7F800000u; }

// Token 32 h + 16 g + 4 c + i of a tile is element 4 g + i of k-step h in the lanes with lane >> 4 = c: what keeps that one element.
__device__ __forceinline__ u32x4 keep_token(int tok, int q4) {
  const int e = 4 * ((tok >> 4) & 1) + (tok & 3);
  u32x4 keep;
#pragma unroll
  for (int x = 0; x < 4; ++x) keep[x] = q4 == ((tok >> 2) & 3) && x == (e >> 1) ? ((e & 1) ? 0xFFFF0000u : 0xFFFFu) : 0u;
  return keep;
}

}  // namespace tpla
