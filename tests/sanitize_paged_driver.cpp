// Host validation of rotary positions and of the paged cache under AddressSanitizer / UndefinedBehaviorSanitizer: every call is refused
// before a launch (no GPU needed; pointers are never followed).  Built and run by tests/test_paged_sanitizers.py.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "thrift.h"

#define EXPECT(call, want) do { int got_ = (int)(call); if (got_ != (want)) { printf("line %d: got %d want %d\n", __LINE__, got_, (want)); bad++; } } while (0)

int main() {
  int bad = 0;
  void* p = (void*)0x1000;
  int32_t *i = (int32_t*)p, *j = (int32_t*)0x2000;
  const double* f = (const double*)p;
  double freqs[512];
  float gain = 0.f;
  const int64_t far[3] = {INT64_MAX, INT64_MIN, -1};
  const int sizes[] = {INT_MIN, -1, 0, 1, 2, 3, 16, 128, 1 << 15, 1 << 23, 1 << 30, INT_MAX};
  long refused = 0;
  for (int a : sizes)
    for (int b : sizes) {
      // each of these has one argument that no size repairs
      EXPECT(thrift_rope(p, far, p, far, a, p, far, p, far, b, THRIFT_F32, i, INT64_MAX, f, 128, 0, 1.f, a, b, 128, nullptr), THRIFT_ERR_DTYPE);
      EXPECT(thrift_rope(p, nullptr, p, nullptr, a, p, nullptr, p, nullptr, b, THRIFT_F16, i, a, f, 127, 0, 1.f, a, b, 128, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_rope_backward(p, nullptr, p, nullptr, 4, nullptr, nullptr, nullptr, nullptr, 0, THRIFT_F16, i, a, f, 128, 7, 1.f, a, b, 128, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_page_map(i, i, a, 17, b, i, a, i, b, i, a, i, i, i, j, j, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_page_map(i, i, a, 16, b, i, a, i, b, i, a, i, i, i, i, j, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_page_release(i, i, a, 0, b, i, b, i, a, i, j, j, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_append(p, far, p, a, p, far, p, far, b, THRIFT_F16, a, i, i, f, 128, 0, 1.f, p, p, b, 24, 128, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_decode(p, THRIFT_F16, p, p, a, i, b, i, a, b, a, 96, 16, 0.f, p, THRIFT_F16, nullptr, p, 0, nullptr), THRIFT_ERR_SHAPE);
      for (int c : sizes) {
        // sizes that are taken need a workspace (one byte less is refused) or none; then 17 is no page size
        const size_t need = thrift_paged_decode_workspace(a, b, c, a, 16, 128);
        const int s = (int)thrift_paged_decode(p, THRIFT_BF16, p, p, 8, i, a, i, a, b, c, 128, need ? 16 : 17, 0.f, p, THRIFT_F32, nullptr, p, need ? need - 1 : 0, nullptr);
        EXPECT(s, need ? THRIFT_ERR_WORKSPACE : THRIFT_ERR_SHAPE);
        refused += need == 0;
      }
      for (int scaling = -1; scaling <= 4; ++scaling) refused += thrift_rope_frequencies(a, (double)b, scaling, (double)b, (double)a, 1.0, 32.0, freqs, &gain) != THRIFT_OK;
    }
  EXPECT(thrift_rope_frequencies(1024, 1e4, THRIFT_ROPE_BY_PARTS, 4.0, 4096.0, 1.0, 32.0, freqs, nullptr), THRIFT_OK);
  EXPECT(thrift_rope_frequencies(1024, 1e4, THRIFT_ROPE_NTK, 1e300, 0.0, 1.0, 32.0, freqs, nullptr), THRIFT_OK);          // base 10^304.6
  EXPECT(thrift_rope_frequencies(1024, 1e4, THRIFT_ROPE_NTK, 1e305, 0.0, 1.0, 32.0, freqs, nullptr), THRIFT_ERR_SHAPE);   // 10^309.6
  printf("paged abi sanitizer pass: %s (%d mismatches, %ld refusals, gain %g)\n", bad ? "FAILED" : "ok", bad, refused, gain);
  return bad != 0;
}
