// Angles of rotary positions, shared by the kernels that turn heads.
#pragma once

#include "thrift_device.h"
#include "thrift_paged.h"

namespace thrift {

// cos and sin (times gain) of position * freq.  Far positions times the fastest pair's radian per token are 2^17 and more: in fp32 such an
// angle is off by 2^-7, so it is formed in turns in fp64, where whole turns and then whole quarter turns drop out exactly.
// What is left, at most an eighth of a turn, is fp32 from there: Taylor's polynomials, whose first term left out is below
// 3e-8 at pi/4; with the roundings, cos and sin are within 9e-8.  Every fused product is written out, here and in rotate: all kernels give a head the same bits.
__device__ __forceinline__ void turn(int position, double freq, float gain, float& c, float& s) {
  const double f = freq * 0.15915494309189535;                     // 1 / (2 pi)
  const double t = 4.0 * __builtin_fma((double)position, f, -__builtin_rint((double)position * f));
  const double quarters = __builtin_rint(t);
  const float x = (float)(t - quarters) * 1.5707963267948966f;
  const float x2 = x * x;
  const float sn = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int n = (int)quarters;                                     // -2 .. 2
  const float a = (n & 1) ? sn : cs, b = (n & 1) ? cs : sn;        // cos and sin of x + n pi/2 but for the sign
  c = ((n + 1) & 2) ? -a * gain : a * gain;
  s = (n & 2) ? -b * gain : b * gain;
}

// One pair turned: each channel is rounded once, from fp32.
__device__ __forceinline__ void rotate(float x0, float x1, float c, float s, float& y0, float& y1) {
  y0 = fmaf(x0, c, -(x1 * s));
  y1 = fmaf(x1, c, x0 * s);
}

// ---- heads in 16-byte chunks: an item is two chunks of a head, so that a lane turns eight pairs ----
//
// Half layout: chunk i and its partner half a rotated part away, and behind the rotated part neighbours.  Interleaved: chunks i and
// i + D/16, so that neighbouring lanes read neighbouring chunks.  A workgroup takes `tokens` tokens; `lanes` groups of threads share their heads out,
// and `splits` workgroups the heads of the same tokens.  cos and sin are formed once per token, pair and workgroup, and pass
// through LDS: 30 fp64 and fp32 instructions each, as much as turning four heads.
constexpr int kHeadThreads = 256;
constexpr int kAngles = 2048;              // (cos, sin) pairs of a workgroup's tokens

struct HeadShape {
  int items, tokens, lanes, splits;
};

// `total` heads of `n` tokens
inline HeadShape head_shape(long n, int total, int D, int rot) {
  HeadShape s;
  s.items = D / 16;
  // eight tokens of 128 channels fill a wavefront and are 2 KiB of memory where tokens follow each other; with fewer than 512
  // workgroups of that size the tokens are spread first, down to one each, and then the heads
  int most = s.items <= 64 ? 64 / s.items : 1;
  while (most > 1 && most * (rot / 2) > kAngles) most /= 2;
  s.tokens = 1;
  while (2 * s.tokens <= most && (n + 2 * s.tokens - 1) / (2 * s.tokens) >= 512) s.tokens *= 2;
  s.lanes = kHeadThreads / (s.items * s.tokens);
  if (s.lanes > total) s.lanes = total;
  const long groups = (n + s.tokens - 1) / s.tokens, most_splits = (total + s.lanes - 1) / s.lanes;
  const long wanted = (2048 + groups - 1) / groups;
  s.splits = (int)(wanted < most_splits ? wanted : most_splits);
  return s;
}

template <int LAYOUT>
struct Item {
  int at[2];                               // first channels of the two chunks
  bool turned[2];

  __device__ __forceinline__ Item(int item, int D, int rot) {
    if (LAYOUT == THRIFT_ROPE_HALF) {
      const int own = rot / 16;            // items of the rotated part
      const bool t = item < own;
      at[0] = t ? 8 * item : rot + 16 * (item - own);
      at[1] = t ? at[0] + rot / 2 : at[0] + 8;
      turned[0] = turned[1] = t;
    } else {
      at[0] = 8 * item, at[1] = 8 * (item + D / 16);
      turned[0] = at[0] < rot, turned[1] = at[1] < rot;
    }
  }
  // the eight pairs' cos and sin from one token's row of LDS
  __device__ __forceinline__ void angles(const float2* row, float2 (&cs)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool t = LAYOUT == THRIFT_ROPE_HALF ? turned[0] : turned[e >> 2];
      const int pair = LAYOUT == THRIFT_ROPE_HALF ? at[0] + e : at[e >> 2] / 2 + (e & 3);
      cs[e] = t ? row[pair] : make_float2(1.f, 0.f);
    }
  }
};

// Whether a store instruction fills lines of 128 bytes: neighbouring lanes write neighbouring chunks in the interleaved layout and where the whole
// head is turned by halves; with a part turned by halves, the copied channels are written every other chunk at a time, and the
// turned ones in runs of `rot` bytes.
inline bool fills_lines(int D, int rot, int layout) { return D >= 128 && (layout == THRIFT_ROPE_INTERLEAVED || rot == D); }

// 16 bytes, past the caches where STREAM
template <bool STREAM>
__device__ __forceinline__ v4i chunk_from(const uint16_t* p) {
  return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const v4i*>(p)) : *reinterpret_cast<const v4i*>(p);
}
template <bool STREAM>
__device__ __forceinline__ void chunk_to(uint16_t* p, v4i x) {
  if (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<v4i*>(p));
  else *reinterpret_cast<v4i*>(p) = x;
}

template <typename T>
__device__ __forceinline__ void turn_pair(uint32_t x0, uint32_t x1, float2 cs, uint32_t& y0, uint32_t& y1) {
  float a, b;
  rotate(T::to_float((uint16_t)x0), T::to_float((uint16_t)x1), cs.x, cs.y, a, b);
  y0 = T::from_float(a), y1 = T::from_float(b);
}

// The chunks of one head, turned; chunks behind the rotated part keep their bits.
template <typename T, int LAYOUT>
__device__ __forceinline__ void turn_item(const Item<LAYOUT>& it, v4i (&x)[2], const float2 (&cs)[8]) {
  v4i y[2];
  if (LAYOUT == THRIFT_ROPE_HALF) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t a0, a1, b0, b1;
      turn_pair<T>((uint32_t)x[0][d] & 0xffffu, (uint32_t)x[1][d] & 0xffffu, cs[2 * d], a0, b0);
      turn_pair<T>((uint32_t)x[0][d] >> 16, (uint32_t)x[1][d] >> 16, cs[2 * d + 1], a1, b1);
      y[0][d] = (int)(a0 | (a1 << 16)), y[1][d] = (int)(b0 | (b1 << 16));
    }
  } else {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint32_t a, b;
        turn_pair<T>((uint32_t)x[c][d] & 0xffffu, (uint32_t)x[c][d] >> 16, cs[4 * c + d], a, b);
        y[c][d] = (int)(a | (b << 16));
      }
  }
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (it.turned[c]) x[c] = y[c];
}

}  // namespace thrift
