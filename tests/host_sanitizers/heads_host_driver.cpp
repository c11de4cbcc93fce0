// The grouped-head entry points under AddressSanitizer and UndefinedBehaviorSanitizer on the host code, as abi_host_driver.cpp has the others: argument
// checks with values at the ends of their types, workspaces against the plans that use them, and what the launchers ask for over a sweep of shapes
// (launches are recorded by recorded_launches.h, nothing runs).  Exit status 0 = every expectation held and no sanitizer report was raised.
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>

#include "tpla.h"
#include "heads.h"
#include "recorded_launches.h"

static int g_failures = 0;
#define EXPECT(cond)                                                                                             \
  do {                                                                                                           \
    if (!(cond)) {                                                                                               \
      fprintf(stderr, "%s:%d: expectation failed: %s (last error: %s)\n", __FILE__, __LINE__, #cond, tpla_last_error()); \
      ++g_failures;                                                                                              \
    }                                                                                                            \
  } while (0)

static void* const A = (void*)(uintptr_t)4096;        // aligned, never dereferenced
static void* const B = (void*)((uintptr_t)1 << 40);
static const int32_t* const Ai = (const int32_t*)A;
static const double* const Ad = (const double*)A;
static float* const Af = (float*)A;
constexpr size_t BIG = (size_t)1 << 60;

static tpla_heads_t shape(int B, int H, int H_kv, int d_k, int d_v, int page, int dtype) { return tpla_heads_t{B, H, H_kv, d_k, d_v, page, dtype, 0.1f}; }

static int norm(const tpla_heads_t& s, int64_t T, int64_t q_ts, int64_t q_hs, int64_t o_ts, int64_t o_hs, int rot = 0) {
  return tpla_norm_rotary_heads(&s, TPLA_ROTARY_HALF, rot, Ad, 1.f, NULL, NULL, 1e-6f, Ai, T, A, q_ts, q_hs, B, o_ts, o_hs, NULL, 0, 0, NULL, 0, 0, NULL);
}
static int append(const tpla_heads_t& s, int64_t T, int64_t ts, int64_t hs) {
  return tpla_append_heads(&s, TPLA_ROTARY_INTERLEAVED, 8, Ad, 1.f, NULL, NULL, 1e-6f, Ai, T, NULL, 0, 0, NULL, 0, 0, A, ts, hs, A, ts, hs, Ai, B, B, NULL);
}
static int decode(const tpla_heads_t& s, int pages, size_t n) { return tpla_decode_heads(&s, A, A, A, Ai, pages, Ai, A, n, B, TPLA_F32, Af, NULL); }
static int prefill(const tpla_heads_t& s, int pages, int64_t T, int most, size_t n) {
  return tpla_prefill_heads(&s, A, A, A, Ai, pages, Ai, Ai, T, most, A, n, B, TPLA_BF16, Af, NULL);
}

// Values at the ends of their types: refused or taken, never an overflow on the way.
static void extreme_arguments() {
  const tpla_heads_t s = shape(2, 8, 2, 64, 64, 64, TPLA_BF16);
  for (int64_t big : {(int64_t)1 << 40, (int64_t)1 << 59, (int64_t)1 << 60, (int64_t)1 << 61, (int64_t)1 << 62, INT64_MAX, INT64_MAX - 7, (int64_t)INT64_MIN, (int64_t)INT64_MIN + 8}) {
    for (int dtype : {TPLA_BF16, TPLA_F32}) {
      const int esz = dtype == TPLA_F32 ? 4 : 2;
      const bool sound = big > 0 && big % (16 / esz) == 0 && (__int128)big * esz < (__int128)1 << 62;      // of strides: whole 16 bytes, offsets below 2^62
      tpla_heads_t x = s;
      x.dtype = dtype;
      g_launches.clear();
      const int in = norm(x, 2, big, 64, 512, 64), out = norm(x, 2, 512, 64, big, 64), heads = norm(x, 2, 512, big, 64, 128), cache = append(x, 2, big, 64);
      EXPECT((in == TPLA_OK) == sound && (out == TPLA_OK) == sound && (cache == TPLA_OK) == sound);
      EXPECT(heads == TPLA_OK || heads == TPLA_ERR_SHAPE || heads == TPLA_ERR_ALIGN);
      EXPECT(norm(x, 3, 512, 64, big, big) != TPLA_OK);                                       // (two rows at one place)
    }
    EXPECT(norm(s, big, 512, 64, 512, 64) == TPLA_ERR_SHAPE && append(s, big, 128, 64) == TPLA_ERR_SHAPE);
    EXPECT(prefill(s, 64, big, INT_MAX, BIG) != TPLA_OK && tpla_workspace_bytes_prefill_heads(&s, big, INT_MAX, 64) == 0);
  }
  for (int big : {INT_MAX, INT_MAX - 7, 1 << 30, INT_MIN, -1}) {
    EXPECT(decode(s, big, BIG) != TPLA_OK && prefill(s, big, 9, 9, BIG) != TPLA_OK && tpla_workspace_bytes_heads(&s, big) == 0);
    EXPECT((prefill(s, 64, 9, big, BIG) == TPLA_OK) == (big > 0));
    for (int field = 0; field < 6; ++field) {
      tpla_heads_t x = s;
      int32_t* const f[] = {&x.B, &x.H, &x.H_kv, &x.d_k, &x.d_v, &x.page_tokens};
      *f[field] = big;
      g_launches.clear();
      const int one = decode(x, 4, BIG), many = prefill(x, 4, 100, 50, BIG);
      EXPECT(one != TPLA_OK && many != TPLA_OK && g_launches.empty());
      EXPECT(tpla_workspace_bytes_heads(&x, 4) == 0 && tpla_workspace_bytes_prefill_heads(&x, 100, 50, 4) == 0);
      if (field > 0) (void)norm(x, 2, 1 << 20, 64, 1 << 20, 64), (void)append(x, 2, 1 << 20, 64);
    }
  }
}

static void launch_limits(const char* what, const tpla_heads_t& s, int64_t T) {
  EXPECT(!g_launches.empty());
  for (const RecordedLaunch& l : g_launches) {
    const bool fits = l.grid.x > 0 && l.grid.y > 0 && (uint64_t)l.grid.x * l.block.x < (uint64_t)1 << 32 && l.grid.y <= 65535 && l.grid.z == 1 && l.lds <= 160 * 1024 &&
                      (int)l.lds <= l.lds_allowed;
    EXPECT(fits);
    if (!fits) fprintf(stderr, "%s B=%d H=%d H_kv=%d d=%d/%d T=%lld: grid %u x %u, %zu bytes of LDS\n", what, s.B, s.H, s.H_kv, s.d_k, s.d_v, (long long)T, l.grid.x, l.grid.y, l.lds);
  }
}

// Rows: a token's waves take all of its groups of rows, long calls in parts that together are all tokens.
static void rows_launches() {
  g_record_ints = {1, 2};                              // waves of a token, groups of each
  for (int dtype : {TPLA_BF16, TPLA_F32})
    for (int d : {8, 24, 64, 96, 128, 200, 256})
      for (int H : {1, 7, 64, 4099, 65535})
        for (int64_t T : {(int64_t)1, (int64_t)2047, (int64_t)2048, ((int64_t)1 << 20) + 1, ((int64_t)1 << 22) - 1})
          for (int rot : {0, 2, d}) {
            const tpla_heads_t s = shape(1, H, 1, d, d, 64, dtype);
            g_launches.clear();
            EXPECT(norm(s, T, (int64_t)H * d, d, (int64_t)H * d, d, rot) == TPLA_OK);
            launch_limits("rows", s, T);
            const int lanes = d <= 32 ? 4 : d <= 64 ? 8 : d <= 128 ? 16 : 32, groups = (H + 64 / lanes - 1) / (64 / lanes);
            EXPECT((int64_t)g_launches.size() == (T + ((1 << 20) - 1)) / (1 << 20));
            int64_t left = T;
            for (const RecordedLaunch& l : g_launches) {
              const int64_t here = std::min<int64_t>(left, 1 << 20);
              EXPECT((int64_t)l.ints[0] * l.ints[1] >= groups && (int64_t)(l.ints[0] - 1) * l.ints[1] < groups);
              EXPECT((int64_t)l.grid.x * 4 >= here * l.ints[0] && ((int64_t)l.grid.x - 1) * 4 < here * l.ints[0]);
              left -= here;
            }
          }
  g_record_ints.clear();
}

// Attention: the reported workspace is taken and one byte less is not, it holds what the plan says, and that of a longer call serves shorter ones.
static void attention_launches() {
  const int widths[][4] = {{128, 128, 64, TPLA_BF16}, {64, 64, 16, TPLA_BF16}, {96, 96, 16, TPLA_BF16}, {128, 64, 64, TPLA_BF16}, {256, 200, 64, TPLA_F32}, {8, 8, 5, TPLA_F32}};
  int split = 0, whole = 0;
  for (const auto& w : widths)
    for (int H_kv : {1, 8})
      for (int G : {1, 5, 16, 33, 130})
        for (int Bn : {1, 3, 70, 5000})
          for (int tokens : {1, 500, 3000, 40000, 1 << 24}) {
            const tpla_heads_t s = shape(Bn, G * H_kv, H_kv, w[0], w[1], w[2], w[3]);
            const int pages = (tokens + w[2] - 1) / w[2];
            const size_t one = tpla_workspace_bytes_heads(&s, pages);
            g_launches.clear();
            const int rc = decode(s, pages, one);
            if (one == 0) {
              EXPECT(rc == TPLA_ERR_UNSUPPORTED && g_launches.empty());
              continue;
            }
            EXPECT(rc == TPLA_OK);
            launch_limits("decode", s, Bn);
            if (one > 16) EXPECT(decode(s, pages, one - 1) == TPLA_ERR_WORKSPACE);
            size_t before = 0;
            for (int64_t T : {1, 2, 9, 100, 700, 3001, 20000, 200000}) {
              for (int most : {1, 3, 40, 3000, INT_MAX}) {
                const size_t n = tpla_workspace_bytes_prefill_heads(&s, T, most, pages);
                g_launches.clear();
                const int ok = prefill(s, pages, T, most, n);
                if (ok == TPLA_ERR_UNSUPPORTED) {
                  EXPECT(n == 0 && g_launches.empty());
                  continue;
                }
                EXPECT(ok == TPLA_OK);
                launch_limits("prefill", s, T);
                (g_launches.size() > 1 ? split : whole) += 1;
                if (most == INT_MAX) {
                  EXPECT(n >= before);
                  before = n;
                }
                for (int64_t fewer : {(int64_t)1, T / 3, T - 1})
                  for (int less : {1, std::max(1, (int)std::min<int64_t>(most, T) / 2)})
                    if (fewer > 0 && less <= most) EXPECT(prefill(s, pages, fewer, less, n) == TPLA_OK);
              }
            }
          }
  EXPECT(split > 500 && whole > 500);
}

// The plans: partial results and the merge's notes lie in the workspace.
static void plans() {
  for (int d : {64, 128})
    for (int H_kv : {1, 3, 8})
      for (int G : {1, 4, 16, 32})
        for (int Bn : {1, 40, 3000})
          for (int tokens : {64, 512, 2048, 100000}) {
            const tpla_heads_t s = shape(Bn, G * H_kv, H_kv, d, d, 64, TPLA_BF16);
            for (int most : {0, 1, 2, 8}) {
              if (!tpla::heads_ranges_fit(s, most)) continue;
              const tpla::HeadsPlan p = tpla::heads_ranges_plan(s, most, tokens / 64);
              EXPECT(p.tiles == 1 && p.items == (int64_t)Bn * H_kv && p.rows >= G * std::max(most, 1));       // the merge has a workgroup per row and no second block
              EXPECT(p.workspace >= (size_t)p.slots * p.rows * (d + 2) * 4 + (p.n_wg > 0 ? (size_t)p.items * 12 : 0) && p.slots == 2 * p.n_wg);
            }
            for (int64_t T : {1, 200, 5000, 100000}) {
              const tpla::HeadsPlan p = tpla::heads_prompts_plan(s, T, (int)T, tokens / 64);
              EXPECT(p.items >= H_kv * ((T * G + p.rows - 1) / p.rows) && p.tiles == p.items / H_kv);
              EXPECT(p.slots == 0 || p.slots >= p.items);                                                    // (unsplit, every item has a place)
              EXPECT(p.workspace >= (size_t)p.slots * p.rows * (d + 2) * 4 + (p.slots > 0 ? 4 : 0) && (p.slots > 0) == (p.n_splits > 1));
            }
          }
}

int main() {
  extreme_arguments();
  rows_launches();
  attention_launches();
  plans();
  if (g_failures) {
    fprintf(stderr, "%d expectation(s) failed\n", g_failures);
    return 1;
  }
  printf("heads_host_driver: all expectations held\n");
  return 0;
}
