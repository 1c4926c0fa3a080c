// Rotary positions of the query and key heads of a batch, forward and transposed (the gradient).
#include "thrift_paged.h"
#include "thrift_rotary.h"

namespace thrift {

namespace {

constexpr int kRopeThreads = 128;

// One workgroup per token, a thread per pair or copied channel; cos and sin are formed once for all heads.
template <typename T>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(RopeArgs a) {
  const long token = blockIdx.x;
  const int b = (int)(token / a.N), n = (int)(token % a.N);
  const int position = a.positions ? a.positions[b * a.positions_stride + n] : n;
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < half + (a.D - a.rot); i += kRopeThreads) {
    float c = 1.f, s = 0.f;
    if (i < half) turn(position, a.freqs[i], a.gain, c, s);
    s *= a.sign;
    for (int side = 0; side < 2; ++side) {
      const RopeSide& r = a.side[side];
      for (int h = 0; h < r.heads; ++h) {
        const uint16_t* x = r.x + b * r.xb + h * r.xh + n * r.xn;
        uint16_t* y = r.y + b * r.yb + h * r.yh + n * r.yn;
        if (i >= half) {
          y[half + i] = x[half + i];
          continue;
        }
        const int i0 = a.layout == THRIFT_ROPE_HALF ? i : 2 * i, i1 = a.layout == THRIFT_ROPE_HALF ? i + half : 2 * i + 1;
        const float x0 = T::to_float(x[i0]), x1 = T::to_float(x[i1]);
        y[i0] = T::from_float(x0 * c - x1 * s);
        y[i1] = T::from_float(x1 * c + x0 * s);
      }
    }
  }
}

}  // namespace

void launch_rope(const RopeArgs& a, thrift_dtype dt, hipStream_t st) {
  const unsigned grid = (unsigned)((long)a.B * a.N);
  if (dt == THRIFT_F16) rope_kernel<F16><<<dim3(grid), dim3(kRopeThreads), 0, st>>>(a);
  else rope_kernel<BF16><<<dim3(grid), dim3(kRopeThreads), 0, st>>>(a);
}

}  // namespace thrift
