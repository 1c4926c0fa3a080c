// Tokens of a paged cache as dense rows.
#include "thrift_e4m3.h"
#include "thrift_paged.h"

namespace thrift {

namespace {

constexpr int kReadThreads = 256;

// One element of K and of V per thread.
template <typename T, bool CODES>
__global__ void __launch_bounds__(kReadThreads) paged_read_kernel(PagedReadArgs a) {
  const size_t i = (size_t)blockIdx.x * kReadThreads + threadIdx.x;
  const int c = (int)(i % a.D);
  const size_t row = i / a.D;
  if (row >= (size_t)a.B * a.Hkv * a.N) return;
  const int n = (int)(row % a.N), h = (int)(row / a.N % a.Hkv), b = (int)(row / a.N / a.Hkv);
  const int len = min(a.max_pages * a.page_size, a.seqlens[b]);
  const long p = (long)n + (a.first ? max(0, a.first[b]) : 0);
  uint16_t k = 0, v = 0;
  if (p < len) {
    const int page = a.table[(size_t)b * a.max_pages + p / a.page_size];
    if (page >= 0 && page < a.n_pages) {
      const size_t at = ((size_t)page * a.Hkv + h) * a.page_size + p % a.page_size;
      if (CODES) {
        const float most = T::to_float(T::kLargest);
        const float x = e4m3_values<false>(((const uint8_t*)a.k_pages)[at * a.D + c], scale_of(a.k_scales[at])).x;
        const float y = e4m3_values<false>(((const uint8_t*)a.v_pages)[at * a.D + c], scale_of(a.v_scales[at])).x;
        k = T::from_float(x > most ? most : x < -most ? -most : x);
        v = T::from_float(y > most ? most : y < -most ? -most : y);
      } else {
        k = ((const uint16_t*)a.k_pages)[at * a.D + c], v = ((const uint16_t*)a.v_pages)[at * a.D + c];
      }
    }
  }
  a.k_out[i] = k, a.v_out[i] = v;
}

}  // namespace

void launch_paged_read(const PagedReadArgs& a, thrift_dtype dt, hipStream_t st) {
  const long all = (long)a.B * a.Hkv * a.N * a.D;
  const dim3 grid((unsigned)((all + kReadThreads - 1) / kReadThreads)), block(kReadThreads);
  if (a.k_scales == nullptr) paged_read_kernel<F16, false><<<grid, block, 0, st>>>(a);
  else if (dt == THRIFT_F16) paged_read_kernel<F16, true><<<grid, block, 0, st>>>(a);
  else paged_read_kernel<BF16, true><<<grid, block, 0, st>>>(a);
}

}  // namespace thrift
