// Attention of one new token per sequence over a paged cache, sequences one by one.
#include "thrift_e4m3.h"
#include "thrift_paged.h"

namespace thrift {

namespace {

constexpr int kWaves = 4;

// One workgroup per sequence and query head, a wavefront per key: lanes hold D / 64 channels.
template <typename T, bool CODES, int PER>
__global__ void __launch_bounds__(64 * kWaves) paged_plain_kernel(PagedDecodeArgs a) {
  __shared__ float part[kWaves][PER + 2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, kv = h / (a.Hq / a.Hkv);
  const int len = min(a.max_pages * a.page_size, max(0, a.seqlens[b]));
  float q[PER], o[PER] = {}, m = -__builtin_inff(), l = 0.f;
#pragma unroll
  for (int e = 0; e < PER; ++e) q[e] = T::to_float(a.q[(size_t)blockIdx.x * a.D + lane * PER + e]);
  for (int j = wave; j < len; j += kWaves) {
    const int page = min(a.n_pages - 1, max(0, a.table[(size_t)b * a.max_pages + j / a.page_size]));
    const size_t row = ((size_t)page * a.Hkv + kv) * a.page_size + j % a.page_size;
    auto element = [&](const void* pages, int e) {
      const size_t at = row * a.D + lane * PER + e;
      if (CODES) return e4m3_values<false>(((const uint8_t*)pages)[at], 1.f).x;
      return T::to_float(((const uint16_t*)pages)[at]);
    };
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) s = fmaf(q[e], element(a.k_pages, e), s);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    s *= a.scale;
    if (CODES) s *= scale_of(a.k_scales[row]);
    const float top = fmaxf(m, s), keep = m == top ? 1.f : expf(m - top), p = s == top ? 1.f : expf(s - top);
    m = top, l = l * keep + p;
    const float w = CODES ? p * scale_of(a.v_scales[row]) : p;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = fmaf(w, element(a.v_pages, e), o[e] * keep);
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) part[wave][e][lane] = o[e];
  part[wave][PER][lane] = m, part[wave][PER + 1][lane] = l;
  __syncthreads();
  if (wave != 0) return;
  for (int w = 1; w < kWaves; ++w) {
    const float other = part[w][PER][lane], top = fmaxf(m, other);
    const float k1 = m == top ? 1.f : expf(m - top), k2 = other == top ? 1.f : expf(other - top);
    m = top, l = l * k1 + part[w][PER + 1][lane] * k2;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = o[e] * k1 + part[w][e][lane] * k2;
  }
  const float inv = len > 0 ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const size_t to = (size_t)blockIdx.x * a.D + lane * PER + e;
    if (a.out_dt == THRIFT_F32) ((float*)a.out)[to] = o[e] * inv;
    else if (a.out_dt == THRIFT_F16) ((uint16_t*)a.out)[to] = F16::from_float(o[e] * inv);
    else ((uint16_t*)a.out)[to] = BF16::from_float(o[e] * inv);
  }
  if (a.lse != nullptr && lane == 0) a.lse[blockIdx.x] = len > 0 ? m + logf(l) : -__builtin_inff();
}

template <typename T, bool CODES>
void launch(const PagedDecodeArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long)a.B * a.Hq)), block(64 * kWaves);
  if (a.D == 64) paged_plain_kernel<T, CODES, 1><<<grid, block, 0, st>>>(a);
  else if (a.D == 128) paged_plain_kernel<T, CODES, 2><<<grid, block, 0, st>>>(a);
  else paged_plain_kernel<T, CODES, 4><<<grid, block, 0, st>>>(a);
}

}  // namespace

size_t paged_prefix_workspace(int bits, int B, int Hq, int Hkv, int n_groups, int max_pages, int page_size, int D) { return 256; }

void launch_paged_prefix(const PagedPrefixArgs& a, int bits, hipStream_t st) {
  if (bits == 8 && a.d.dt == THRIFT_F16) launch<F16, true>(a.d, st);
  else if (bits == 8) launch<BF16, true>(a.d, st);
  else if (a.d.dt == THRIFT_F16) launch<F16, false>(a.d, st);
  else launch<BF16, false>(a.d, st);
}

}  // namespace thrift
