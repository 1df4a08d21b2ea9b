// Host-side exercise of the operators around a block's attention for a build with AddressSanitizer and UndefinedBehaviorSanitizer on the host code: sizes, refusals and the plan
// of each attention return before any GPU call.  Exit status 0 = all checks held.
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <limits>

#include "svdcache.h"

static int failures = 0;
#define EXPECT(cond)                                                              \
  do {                                                                            \
    if (!(cond)) {                                                                \
      std::fprintf(stderr, "line %d: expectation failed: %s\n", __LINE__, #cond); \
      ++failures;                                                                 \
    }                                                                             \
  } while (0)

int main() {
  void* const p = reinterpret_cast<void*>(uintptr_t(4096));      // aligned, never dereferenced
  void* const o = reinterpret_cast<void*>(uintptr_t(8192));
  void* const odd = reinterpret_cast<void*>(uintptr_t(4097));
  const int64_t far = std::numeric_limits<int64_t>::max();
  const int32_t big = std::numeric_limits<int32_t>::max();
  const int64_t rows[] = {0, 1, 127, 128, 129, 4608, 119056, int64_t(1) << 30, (int64_t(1) << 30) + 1, big, (int64_t)big + 1, far, -1, -far - 1};
  const int32_t counts[] = {1, 7, 24, 1 << 16, (1 << 16) + 1, big, 0, -1, -big - 1};
  const int32_t widths[] = {1, 64, 72, 128, 256, 257, big, 0, -1, -big - 1};
  const svdc_heads s{1 << 20, 128, 64};
  for (int64_t batch : {int64_t(0), int64_t(1), int64_t(5), int64_t(65535), int64_t(65536), far, int64_t(-1), -far - 1})
    for (int64_t q : rows)
      for (int64_t k : rows)
        for (int32_t heads : counts)
          for (int32_t d : widths)
            for (int32_t dtype : {0, 1, 2, -1}) {
              svdc_attention a{batch, q, k, q, k, heads, 1, d, dtype, 0.1f, 0, s, s, s, s};
              const size_t ws = svdcache_attention_workspace_bytes(&a);
              const bool sizes = batch >= 0 && batch <= 65535 && q >= 0 && q <= 1 << 30 && k >= 0 && k <= 1 << 30 && heads >= 1 && heads <= 1 << 16 && d >= 1 && d <= 256 && dtype >= 0 && dtype <= 1;
              EXPECT(sizes || ws == 0);
              EXPECT(ws < size_t(1) << 32);
              // a misaligned result is refused whatever the sizes are, unless there are no rows
              EXPECT(svdcache_attention(&a, p, p, p, nullptr, nullptr, nullptr, odd, o, ws, nullptr) < 0 || batch == 0 || q == 0);
              EXPECT(svdcache_attention(&a, p, p, p, static_cast<int32_t*>(odd), nullptr, nullptr, o, o, ws, nullptr) < 0 || batch == 0 || q == 0);
              if (ws) EXPECT(svdcache_attention(&a, p, p, p, nullptr, nullptr, nullptr, o, o, ws - 1, nullptr) == SVDC_E_WORKSPACE);
              svdc_norm_rotate n{batch, q, heads, 1, d, dtype, dtype, 1, d / 2, 0, 1e-6f, 0, 0, s, s, s, s, s, s};
              EXPECT(svdcache_norm_rotate(&n, p, nullptr, nullptr, nullptr, nullptr, static_cast<float*>(p), odd, nullptr, nullptr, nullptr) < 0 || batch == 0 || q == 0);
            }
  for (int64_t x : {int64_t(0), int64_t(1), int64_t(1) << 22, (int64_t(1) << 22) + 1, int64_t(1) << 40, (int64_t(1) << 40) + 1, far, int64_t(-1), -far - 1})
    for (int which = 0; which < 3; ++which) {
      svdc_heads t = s;
      (which == 0 ? t.seq : which == 1 ? t.row : t.head) = x;
      svdc_attention a{2, 100, 100, 0, 0, 4, 2, 64, 1, 0.1f, 0, s, t, s, s};
      const bool ok = x >= 0 && x <= (which == 1 ? int64_t(1) << 22 : int64_t(1) << 40);
      EXPECT(svdcache_attention(&a, p, p, p, nullptr, nullptr, nullptr, odd, o, 1 << 30, nullptr) == (ok ? SVDC_E_ALIGN : SVDC_E_SHAPE));
      svdc_norm_rotate n{2, 100, 4, 2, 64, 1, 1, 1, 32, 0, 1e-6f, 0, x, s, s, s, t, s, s};
      EXPECT(svdcache_norm_rotate(&n, p, nullptr, nullptr, nullptr, nullptr, static_cast<float*>(p), odd, nullptr, nullptr, nullptr) ==
             (ok && x >= 0 && x <= int64_t(1) << 40 ? SVDC_E_ALIGN : SVDC_E_SHAPE));
    }
  for (int64_t n : rows)
    for (int32_t axes : {0, 1, 3, 4, 5, big, -1})
      for (int32_t d : {2, 56, 64, 256, 258, 3, 0, -2, big, -big - 1})
        for (int64_t ld : {int64_t(0), int64_t(axes), int64_t(1) << 24, (int64_t(1) << 24) + 1, far, -far - 1}) {
          svdc_rotary r{n, ld, axes, 1, {d, d, d, d}, {1e4, 1e4, 1e4, 1e4}};
          EXPECT(svdcache_rotary_table(&r, p, static_cast<float*>(odd), nullptr) < 0 || n == 0);
        }
  EXPECT(svdcache_attention(nullptr, p, p, p, nullptr, nullptr, nullptr, o, o, 0, nullptr) == SVDC_E_NULL);
  EXPECT(svdcache_attention_workspace_bytes(nullptr) == 0);
  EXPECT(svdcache_norm_rotate(nullptr, p, p, p, nullptr, nullptr, nullptr, o, o, o, nullptr) == SVDC_E_NULL);
  EXPECT(svdcache_rotary_table(nullptr, p, static_cast<float*>(o), nullptr) == SVDC_E_NULL);
  if (failures) return 1;
  std::puts("host checks of the operators around the attention passed");
  return 0;
}
