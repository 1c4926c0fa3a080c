// Attention of one new token per sequence over a paged cache of 16 or 8 bits: the choice of the form (kernels: thrift_paged_walk.h).
#include "thrift_paged_walk.h"

namespace thrift {

namespace {

// A CU takes about 40 GB/s from memory, so that a row of its own costs it 6.4 us for 256 KiB of keys and values; where the block table has room for no
// more, that is less than the search for a share and the second launch.  Shares / rows, us, 32/8 heads of 128 channels: 10.3 / 6.3 for 1 x 256,
// 10.7 / 5.7 for 16 x 50-100, 12.8 / 10.7 for 16 x 250-500, 54.3 / 54.6 for 256 x 125-500; beyond: 10.3 / 12.5 for 1 x 1000, 15.2 / 17.8 for
// 16 x 500-1000.  64 channels: 14.0 / 11.5 for 64 x 125-500; 256 channels: 12.5 / 16.2 for 4 x 250-500, 16/16 heads.
// From codes the same rule, though their rows are half the bytes, since a row's time is then the conversion's: 9.2 / 6.8 for 1 x 256, 9.8 / 5.7 for 16 x 50-100,
// 12.2 / 11.2 for 16 x 250-500, 20.9 / 18.7 for 64 x 125-250 of 16/16 heads; beyond: 9.6 / 13.4 for 1 x 1000, 15.1 / 17.4 for 16 x 500-1000.
// With more than four rows per CU the shares are as fast (33.8 / 33.7 for 256 x 63-250) or faster (160 / 226 for 4096 x 15-60).
constexpr long kRowBytes = 256 << 10, kRowMost = 4 * kCus;
bool by_rows(int B, int Hq, int Hkv, int max_pages, int page_size, int D) {
  return Hq / Hkv <= 16 && (long)max_pages * page_size * D * 4 <= kRowBytes && (long)B * Hkv <= kRowMost;
}

template <typename T, int D, bool C8>
void launch(const PagedDecodeArgs& a, hipStream_t st) {
  const Launch z = launch_of(a, C8, a.workspace);
  if (by_rows(a.B, a.Hq, a.Hkv, a.max_pages, a.page_size, a.D)) {
    paged_decode_rows_kernel<T, D, C8><<<dim3((unsigned)((long)a.B * a.Hkv)), dim3(64 * kRowWaves), 0, st>>>(a, z);
    return;
  }
  const dim3 grid(shares_of(C8)), block(64 * waves_of(D));
  if (z.G <= 16) paged_decode_kernel<T, D, 1, C8, false><<<grid, block, 0, st>>>(a, z);
  else paged_decode_kernel<T, D, 2, C8, false><<<grid, block, 0, st>>>(a, z);
  paged_merge_kernel<D, shares_of(C8)><<<dim3(shares_of(C8) * z.G), dim3(kThreads), 0, st>>>(a, z);
}
template <typename T, bool C8>
void launch(const PagedDecodeArgs& a, hipStream_t st) {
  if (a.D == 64) launch<T, 64, C8>(a, st);
  else if (a.D == 128) launch<T, 128, C8>(a, st);
  else launch<T, 256, C8>(a, st);
}

}  // namespace

size_t paged_decode_workspace(int B, int Hq, int Hkv, int max_pages, int page_size, int D) {
  return by_rows(B, Hq, Hkv, max_pages, page_size, D) ? 0 : space_bytes(false, Hq / Hkv, D);
}
size_t paged_decode8_workspace(int B, int Hq, int Hkv, int max_pages, int page_size, int D) {
  return by_rows(B, Hq, Hkv, max_pages, page_size, D) ? 0 : space_bytes(true, Hq / Hkv, D);
}

void launch_paged_decode(const PagedDecodeArgs& a, hipStream_t st) {
  if (a.dt == THRIFT_F16) launch<F16, false>(a, st);
  else launch<BF16, false>(a, st);
}
void launch_paged_decode8(const PagedDecodeArgs& a, hipStream_t st) {
  if (a.dt == THRIFT_F16) launch<F16, true>(a, st);
  else launch<BF16, true>(a, st);
}

}  // namespace thrift
