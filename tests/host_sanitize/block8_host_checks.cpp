// Host-side exercise of the operators in 8 bits for a build with AddressSanitizer and UndefinedBehaviorSanitizer on the host code: sizes, refusals and the
// choice of a way for each product return before any GPU call.  Exit status 0 = all checks held.
#include <cstdint>
#include <cstdio>
#include <cstring>
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
  void* const odd = reinterpret_cast<void*>(uintptr_t(4097));
  float* const f = static_cast<float*>(p);
  const int64_t far = std::numeric_limits<int64_t>::max();
  const int32_t big = std::numeric_limits<int32_t>::max();
  const int64_t rows[] = {0, 1, 15, 127, 128, 129, 4608, 119056, (int64_t)big, (int64_t)big + 1, far, -1, -far - 1};
  const int32_t widths[] = {1, 7, 127, 128, 129, 512, 3072, 12288, 1 << 20, (1 << 20) + 1, 1 << 24, (1 << 24) + 1, big, 0, -1, -big - 1};
  for (int64_t M : rows)
    for (int32_t D : widths) {
      const size_t q = svdcache_q8_bytes(M, D);
      const bool ok = M >= 0 && M <= big && D >= 1 && D <= 1 << 20;
      EXPECT(ok ? q >= (size_t)M * D && q % 128 == 0 : q == 0);
      for (int32_t br : {1, 128, 0, 2, -1, big}) {
        const size_t s = svdcache_q8_scale_bytes(M, D, br);
        EXPECT(ok && (br == 1 || br == 128) ? s % 4 == 0 && (s > 0) == (M > 0) : s == 0);
      }
      for (int64_t ld : {(int64_t)D, (int64_t)D + 3, (int64_t)1 << 47, far, (int64_t)-1, -far - 1})
        for (int32_t dtype : {0, 1, 2, 7, -1}) {
          svdc_norm8 n{M, D, dtype, dtype, 1e-6f, ld, ld, ld, ld};
          svdc_quant8 z{M, D, dtype, ld, 1, 0};
          // a misaligned result is refused whatever the sizes are, unless there are no rows
          const int32_t a = svdcache_rms_norm8(&n, p, nullptr, nullptr, nullptr, nullptr, odd, p, nullptr);
          const int32_t b = svdcache_quantize8(&z, p, odd, p, nullptr);
          EXPECT(a < 0 || M == 0);
          EXPECT(b < 0 || M == 0);
        }
      for (int32_t K : widths)
        for (int32_t dtype : {0, 1, 2, 3})
          for (int32_t act : {0, 1, 2, 3, -1}) {
            svdc_matmul8 m{M, D, K, dtype, act, D > 0 ? D : 1};
            const size_t ws = svdcache_matmul8_workspace_bytes(&m);
            const bool valid = M >= 0 && M <= big && D >= 1 && D <= (dtype == 2 ? 1 << 20 : 1 << 24) && K >= 1 && K <= 1 << 20 && dtype <= 2 && act >= 0 && act <= 2;
            EXPECT(valid || ws == 0);
            EXPECT(ws % sizeof(float) == 0);
            EXPECT(svdcache_matmul8(&m, odd, p, p, p, f, p, p, p, ws, nullptr) < 0 || M == 0);
            if (ws) EXPECT(svdcache_matmul8(&m, p, p, p, p, f, p, p, p, ws - 1, nullptr) == SVDC_E_WORKSPACE);
          }
    }
  EXPECT(svdcache_rms_norm8(nullptr, p, p, f, p, p, p, p, nullptr) == SVDC_E_NULL);
  EXPECT(svdcache_quantize8(nullptr, p, p, p, nullptr) == SVDC_E_NULL);
  EXPECT(svdcache_matmul8(nullptr, p, p, p, p, f, p, p, p, 0, nullptr) == SVDC_E_NULL);
  EXPECT(svdcache_matmul8_workspace_bytes(nullptr) == 0);
  if (failures) return 1;
  std::puts("host checks of the operators in 8 bits passed");
  return 0;
}
