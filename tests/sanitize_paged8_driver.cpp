// Host validation of the 8-bit paged cache, of reading pages back and of attention over common starts under AddressSanitizer /
// UndefinedBehaviorSanitizer: every call is refused before a launch (no GPU needed; pointers are never followed).  Built and run by
// tests/test_paged8_sanitizers.py.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "thrift.h"

#define EXPECT(call, want) do { int got_ = (int)(call); if (got_ != (want)) { printf("line %d: got %d want %d\n", __LINE__, got_, (want)); bad++; } } while (0)

int main() {
  int bad = 0;
  long refused = 0;
  void* p = (void*)0x1000;
  uint8_t* u = (uint8_t*)p;
  int32_t* i = (int32_t*)p;
  const double* f = (const double*)p;
  const int64_t far[3] = {INT64_MAX, INT64_MIN, -1};
  const int64_t sizes[] = {INT64_MIN, INT_MIN, -1, 0, 1, 2, 3, 16, 128, 4096, 1 << 15, 1 << 23, 1 << 30, INT_MAX, INT64_MAX};
  for (int64_t a : sizes)
    for (int64_t b : sizes) {
      const int x = (int)a, y = (int)b;
      // each of these has one argument that no size repairs
      EXPECT(thrift_paged_append8(p, far, p, x, p, far, p, far, y, THRIFT_F16, a, i, i, f, 128, 0, 1.f, u, u, u, u, y, 24, 128, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_append8(p, far, p, x, p, far, p, far, y, THRIFT_F32, a, i, i, f, 128, 0, 1.f, u, u, u, u, y, 16, 128, nullptr), THRIFT_ERR_DTYPE);
      EXPECT(thrift_paged_decode8(p, THRIFT_F16, u, u, u, u, x, i, y, i, x, y, x, 96, 16, 0.f, p, THRIFT_F16, nullptr, p, 0, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_read(p, p, x, i, y, nullptr, i, x, y, x, 127, 20, p, p, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_read8(u, u, u, u, x, i, y, i, i, y, x, y, 128, 17, p, p, THRIFT_BF16, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_read8(u, u, u, u, x, i, y, i, i, y, x, y, 128, 16, p, p, THRIFT_F32, nullptr), THRIFT_ERR_DTYPE);
      EXPECT(thrift_paged_decode_prefix(p, THRIFT_F16, p, p, x, i, y, i, i, i, 4097, x, y, x, 128, 16, 0.f, p, THRIFT_F16, nullptr, p, SIZE_MAX, nullptr), THRIFT_ERR_SHAPE);
      EXPECT(thrift_paged_decode_prefix8(p, THRIFT_F16, u, u, u, u, x, i, y, i, i, i, 0, x, y, x, 128, 16, 0.f, p, THRIFT_F16, nullptr, p, SIZE_MAX, nullptr), THRIFT_ERR_SHAPE);
      for (int64_t c : sizes) {
        // sizes that are taken need a workspace (one byte less is refused) or none; then 17 is no page size
        const int w = (int)c;
        const size_t need = thrift_paged_decode8_workspace(x, y, w, x, 16, 128);
        EXPECT(thrift_paged_decode8(p, THRIFT_BF16, u, u, u, u, 8, i, x, i, x, y, w, 128, need ? 16 : 17, 0.f, p, THRIFT_F32, nullptr, p, need ? need - 1 : 0, nullptr),
               need ? THRIFT_ERR_WORKSPACE : THRIFT_ERR_SHAPE);
        refused += need == 0;
        for (int bits = 8; bits <= 16; bits += 8) {
          const size_t more = thrift_paged_decode_prefix_workspace(bits, x, y, w, 3, x, 16, 64);
          const int page = more ? 16 : 17;
          const size_t size = more ? more - 1 : 0;
          EXPECT(bits == 16 ? thrift_paged_decode_prefix(p, THRIFT_BF16, p, p, 8, i, x, i, i, i, 3, x, y, w, 64, page, 0.f, p, THRIFT_F32, nullptr, p, size, nullptr)
                            : thrift_paged_decode_prefix8(p, THRIFT_BF16, u, u, u, u, 8, i, x, i, i, i, 3, x, y, w, 64, page, 0.f, p, THRIFT_F32, nullptr, p, size, nullptr),
                 more ? THRIFT_ERR_WORKSPACE : THRIFT_ERR_SHAPE);
          refused += more == 0;
        }
      }
    }
  printf("paged 8-bit abi sanitizer pass: %s (%d mismatches, %ld refusals)\n", bad ? "FAILED" : "ok", bad, refused);
  return bad != 0;
}
