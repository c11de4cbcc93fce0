// What the matrix-core kernels of grouped heads share: tiles of keys and of values of 32 or 64 tokens in LDS, rows of 128 or 256 bytes.
#pragma once
#include "lds_tile.h"
#include "heads.h"

namespace tpla {

// Place of the 16-byte pieces of row `tok` within the row: piece c lies at c ^ heads_swz(tok).  Row-wise reads (ds_read_b128: 16 tokens at one piece) run in groups
// of 16 lanes that take tokens 0-3 and 12-15 at one piece and 4-11 at the next one; transposing reads (ds_read_b64_tr_b16) in groups of 8 tokens
// at a pair of pieces.  Rows of 128 bytes alternate between the halves of the banks, tok & 7 is right for both.  Rows of 256 bytes all begin at the
// same bank: bits 1 to 3 of the swizzle have to tell 8 tokens apart, and all four, with the shift of the group above, 16.
template <int RC>
__device__ __forceinline__ int heads_swz(int tok) {
  if constexpr (RC == 16) return ((tok & 3) << 1) | ((tok >> 2) & 1) | ((((tok >> 2) ^ (tok >> 3)) & 1) << 3);
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

// A page id on its way: all LDS reads are waited for (lgkmcnt 0), with the id as an operand, before it is used.
__device__ __forceinline__ void lds_request_page(int& id, const int* at) {
  asm volatile("ds_read_b32 %0, %1" : "=v"(id) : "v"(lds_at(reinterpret_cast<const char*>(at))) : "memory");
}

// ---- output accumulators in registers of our choice ----
// Quad N is v[192 + 4 N : 195 + 4 N], N < 16: the top of the 256 that two waves per SIMD leave each.  Left to the compiler the accumulators exist twice: a
// branch may rescale them, and it copies them for every tile so that the branch finds them in other registers (16384 tokens, 64 of them: 2870 us).
// So the products and what else touches them are written out, with the wait states that the compiler then does not insert: 2 between an ordinary
// write and a matrix instruction that reads it, 11 (here 18) between a matrix instruction and an ordinary one that touches its result.  (Not
// accumulation registers: a kernel that names those gets half of its registers of that kind, and spills.)  out_keep() stands at every step of a loop:
// nothing of the compiler's may live in these registers across it.
constexpr int OUT0 = 192;
__device__ __forceinline__ void out_keep() {
#ifdef __HIP_DEVICE_COMPILE__                         // (the host's compiler does not know the names)
  asm volatile("" : : : "v192", "v193", "v194", "v195", "v196", "v197", "v198", "v199", "v200", "v201", "v202", "v203", "v204", "v205", "v206", "v207", "v208", "v209",
               "v210", "v211", "v212", "v213", "v214", "v215", "v216", "v217", "v218", "v219", "v220", "v221", "v222", "v223", "v224", "v225", "v226", "v227",
               "v228", "v229", "v230", "v231", "v232", "v233", "v234", "v235", "v236", "v237", "v238", "v239", "v240", "v241", "v242", "v243", "v244", "v245",
               "v246", "v247", "v248", "v249", "v250", "v251", "v252", "v253", "v254", "v255");
#endif
}
__device__ __forceinline__ void score_first(f32x4& s, const bf16x8& k, const bf16x8& q) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(s) : "v"(k), "v"(q));
}
__device__ __forceinline__ void score_more(f32x4& s, const bf16x8& k, const bf16x8& q) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(s) : "v"(k), "v"(q));
}
template <int N>
__device__ __forceinline__ void out_product(const u32x4& v, const bf16x8& p) {
  asm volatile("v_mfma_f32_16x16x32_bf16 v[%2:%3], %0, %1, v[%2:%3]" : : "v"(v), "v"(p), "n"(OUT0 + 4 * N), "n"(OUT0 + 4 * N + 3));
}
// The weights are in place: what follows multiplies with them.
__device__ __forceinline__ void settle_weights(bf16x8& p) { asm volatile("s_nop 1" : "+v"(p) : : "memory"); }
__device__ __forceinline__ void settle_scores(f32x4& s) { asm volatile("" : "+v"(s)); }
__device__ __forceinline__ void out_settle_write() { asm volatile("s_nop 1" ::: "memory"); }
__device__ __forceinline__ void out_settle_result() { asm volatile("s_nop 15\n\ts_nop 1" ::: "memory"); }
template <int A>
__device__ __forceinline__ float out_read_one() {
  float x;
  asm volatile("v_mov_b32 %0, v[%1]" : "=v"(x) : "n"(OUT0 + A));
  return x;
}
template <int N>
__device__ __forceinline__ f32x4 out_read() {
  const float x = out_read_one<4 * N>(), y = out_read_one<4 * N + 1>(), z = out_read_one<4 * N + 2>(), w = out_read_one<4 * N + 3>();
  return f32x4{x, y, z, w};
}
template <int N>
__device__ __forceinline__ void out_write(f32x4 x) {
  constexpr int A = OUT0 + 4 * N;
  asm volatile("v_mov_b32 v[%4], %0\n\tv_mov_b32 v[%5], %1\n\tv_mov_b32 v[%6], %2\n\tv_mov_b32 v[%7], %3"
               : : "v"(x[0]), "v"(x[1]), "v"(x[2]), "v"(x[3]), "n"(A), "n"(A + 1), "n"(A + 2), "n"(A + 3));
}
template <int N>
__device__ __forceinline__ void out_scale(float by) {
  constexpr int A = OUT0 + 4 * N;
  asm volatile("v_mul_f32 v[%1], v[%1], %0\n\tv_mul_f32 v[%2], v[%2], %0\n\tv_mul_f32 v[%3], v[%3], %0\n\tv_mul_f32 v[%4], v[%4], %0"
               : : "v"(by), "n"(A), "n"(A + 1), "n"(A + 2), "n"(A + 3));
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
