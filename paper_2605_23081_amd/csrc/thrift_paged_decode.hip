// Attention of one new token per sequence over a paged 16-bit cache.
#include "thrift_device.h"
#include "thrift_paged.h"

namespace thrift {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// One workgroup per (sequence, query head).  A wavefront takes every fourth key, a lane D/64 of its channels, with one running
// maximum and sum; the four states are joined at the end.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) paged_decode_kernel(PagedDecodeArgs a) {
  constexpr int C = D / 64;
  __shared__ float part[kWaves][D + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, hk = h / (a.Hq / a.Hkv);
  const int len = (int)min((long)a.max_pages * a.page_size, (long)max(0, a.seqlens[b]));
  const size_t row = (size_t)b * a.Hq + h;
  float q[C], o[C], m = -__builtin_inff(), l = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) q[c] = T::to_float(a.q[row * D + lane + 64 * c]) * a.scale, o[c] = 0.f;
  for (int j = wave; j < len; j += kWaves) {
    const int page = min(a.n_pages - 1, max(0, a.table[(size_t)b * a.max_pages + j / a.page_size]));
    const size_t at = (((size_t)page * a.Hkv + hk) * a.page_size + j % a.page_size) * D + lane;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) s += q[c] * T::to_float(a.k_pages[at + 64 * c]);
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    const float top = fmaxf(m, s), keep = expf(m - top), p = expf(s - top);
    m = top;
    l = l * keep + p;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = o[c] * keep + p * T::to_float(a.v_pages[at + 64 * c]);
  }
#pragma unroll
  for (int c = 0; c < C; ++c) part[wave][lane + 64 * c] = o[c];
  if (lane == 0) part[wave][D] = m, part[wave][D + 1] = l;
  __syncthreads();
  float top = -__builtin_inff(), sum = 0.f;
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, part[w][D]);
  float weight[kWaves];
  for (int w = 0; w < kWaves; ++w) {
    weight[w] = part[w][D] == -__builtin_inff() ? 0.f : expf(part[w][D] - top);
    sum += weight[w] * part[w][D + 1];
  }
  for (int c = tid; c < D; c += kThreads) {
    float x = 0.f;
    for (int w = 0; w < kWaves; ++w) x += weight[w] * part[w][c];
    x = len ? x / sum : 0.f;
    if (a.out_dt == THRIFT_F32) ((float*)a.out)[row * D + c] = x;
    else if (a.out_dt == THRIFT_F16) ((uint16_t*)a.out)[row * D + c] = F16::from_float(x);
    else ((uint16_t*)a.out)[row * D + c] = BF16::from_float(x);
  }
  if (a.lse != nullptr && tid == 0) a.lse[row] = len ? top + logf(sum) : -__builtin_inff();
}

template <typename T>
void launch(const PagedDecodeArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long)a.B * a.Hq));
  if (a.D == 64) paged_decode_kernel<T, 64><<<grid, dim3(kThreads), 0, st>>>(a);
  else if (a.D == 128) paged_decode_kernel<T, 128><<<grid, dim3(kThreads), 0, st>>>(a);
  else paged_decode_kernel<T, 256><<<grid, dim3(kThreads), 0, st>>>(a);
}

}  // namespace

size_t paged_decode_workspace(int, int, int, int, int, int) { return 0; }

void launch_paged_decode(const PagedDecodeArgs& a, hipStream_t st) {
  if (a.dt == THRIFT_F16) launch<F16>(a, st);
  else launch<BF16>(a, st);
}

}  // namespace thrift
