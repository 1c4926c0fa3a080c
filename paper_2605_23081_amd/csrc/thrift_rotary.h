// Angles of rotary positions, shared by the kernels that turn heads.
#pragma once

#include "thrift_device.h"

namespace thrift {

// cos and sin (times gain) of position * freq.  Far positions times the fastest pair's radian per token are 2^17 and more: in fp32 such an
// angle is off by 2^-7, so it is formed in turns in fp64, where whole turns and then whole quarter turns drop out exactly.
// What is left, at most an eighth of a turn, is fp32 from there: Taylor's polynomials, whose first term left out is below
// 3e-8 at pi/4.
__device__ __forceinline__ void turn(int position, double freq, float gain, float& c, float& s) {
  double t = (double)position * (freq * 0.15915494309189535);     // 1 / (2 pi)
  t -= __builtin_rint(t);
  const double quarters = __builtin_rint(4.0 * t);
  const float x = (float)(4.0 * t - quarters) * 1.5707963267948966f;
  const float x2 = x * x;
  const float sn = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
  const float cs = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320))));
  const int n = (int)quarters;                                     // -2 .. 2
  const float a = (n & 1) ? sn : cs, b = (n & 1) ? cs : sn;        // cos and sin of x + n pi/2 but for the sign
  c = ((n + 1) & 2) ? -a * gain : a * gain;
  s = (n & 2) ? -b * gain : b * gain;
}

}  // namespace thrift
