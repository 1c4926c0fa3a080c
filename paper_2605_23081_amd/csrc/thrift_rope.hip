// Rotary positions of the query and key heads of a batch, forward and transposed (the gradient).
//
// Bound by memory: every element is read and written once (counters: 1.34 GB each way for 131072 tokens of 32/8 heads, which is what they hold), at
// 5.4 TB/s there (493-504 us); a copy in 16-byte chunks past the caches runs at 6.5 from 1 GB on, the runtime's own of 2 GiB at 4.9.  3001 tokens, 61 MB,
// stay in the cache in front of the memory where few other bytes come between: 12.1 us then, 5.1 TB/s.  Up to some hundred tokens the
// call is its launch (3.5-3.7 us of kernel, 4 of host time, 5.8-6.3 in all).
#include "thrift_paged.h"
#include "thrift_rotary.h"

namespace thrift {

namespace {

constexpr int kRopeThreads = 128;

// One workgroup per token, a thread per pair or copied channel; cos and sin are formed once for all heads.  For what cannot be read in
// 16-byte chunks; where it can, the kernel below takes half the time (131072 tokens, 32/8 heads: 1006 us here, 538 there with cached
// stores as well; 32768 tokens with 20 of 128 channels turned, which go here: 398 us, 147 there with 64 turned).
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
        float y0, y1;
        rotate(T::to_float(x[i0]), T::to_float(x[i1]), c, s, y0, y1);
        y[i0] = T::from_float(y0);
        y[i1] = T::from_float(y1);
      }
    }
  }
}

template <typename T, int LAYOUT, bool STREAM>
__global__ void __launch_bounds__(kHeadThreads) rope_items_kernel(RopeArgs a, HeadShape z) {
  __shared__ float2 table[kAngles];
  const int tid = threadIdx.x, half = a.rot / 2, all = a.B * a.N;
  const int first = (int)(blockIdx.x / z.splits) * z.tokens, split = blockIdx.x % z.splits;
  const int item = tid % z.items, rest = tid / z.items, local = rest % z.tokens, group = rest / z.tokens;
  const int token = first + local, heads = a.side[0].heads + a.side[1].heads;
  const bool busy = group < z.lanes && token < all;
  const int b = token / a.N, n = token - b * a.N;
  const Item<LAYOUT> it(item, a.D, a.rot);
  const uint16_t* x[2];
  uint16_t* y[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    x[s] = a.side[s].x + b * a.side[s].xb + n * a.side[s].xn;
    y[s] = a.side[s].y + b * a.side[s].yb + n * a.side[s].yn;
  }
  const int step = z.lanes * z.splits;
  int h = busy ? split * z.lanes + group : heads;
  auto load = [&](int head, v4i (&c)[2]) {
    const int s = head >= a.side[0].heads, i = head - (s ? a.side[0].heads : 0);
    const uint16_t* p = x[s] + i * a.side[s].xh;
    c[0] = chunk_from<STREAM>(p + it.at[0]), c[1] = chunk_from<STREAM>(p + it.at[1]);
  };
  v4i c[2];
  if (h < heads) load(h, c);                 // on its way while the angles are formed
  for (int i = tid; i < z.tokens * half; i += kHeadThreads) {
    const int t = first + i / half, pair = i % half;
    if (t >= all) break;
    const int tb = t / a.N, tn = t - tb * a.N;
    float cs, sn;
    turn(a.positions ? a.positions[tb * a.positions_stride + tn] : tn, a.freqs[pair], a.gain, cs, sn);
    table[i] = make_float2(cs, a.sign * sn);
  }
  __syncthreads();
  float2 cs[8];
  if (busy) it.angles(table + local * half, cs);
  while (h < heads) {
    const int s = h >= a.side[0].heads, i = h - (s ? a.side[0].heads : 0);
    uint16_t* p = y[s] + i * a.side[s].yh;
    h += step;
    v4i next[2];
    if (h < heads) load(h, next);
    turn_item<T, LAYOUT>(it, c, cs);
    chunk_to<STREAM>(p + it.at[0], c[0]), chunk_to<STREAM>(p + it.at[1], c[1]);
    c[0] = next[0], c[1] = next[1];
  }
}

bool in_chunks(const RopeSide& s) {
  return s.heads == 0 || (((uintptr_t)s.x | (uintptr_t)s.y) % 16 == 0 && (s.xb | s.xh | s.xn | s.yb | s.yh | s.yn) % 8 == 0);
}

template <typename T>
void launch(const RopeArgs& a, hipStream_t st) {
  const long tokens = (long)a.B * a.N;
  if (a.D % 16 != 0 || a.rot % 16 != 0 || !in_chunks(a.side[0]) || !in_chunks(a.side[1])) {
    rope_kernel<T><<<dim3((unsigned)tokens), dim3(kRopeThreads), 0, st>>>(a);
    return;
  }
  const HeadShape z = head_shape(tokens, a.side[0].heads + a.side[1].heads, a.D, a.rot);
  const dim3 grid((unsigned)((tokens + z.tokens - 1) / z.tokens * z.splits)), block(kHeadThreads);
  // Past the caches where these cannot hold inputs and results of a pass (cached / streamed: 18.8 / 21.0 us for 84 MB, 36.8 / 35.2 for 168,
  // 50.6 / 48.4 for 268, 72.4 / 67.5 for 336, 142 / 131 for 671, 538 / 499 for 2.7 GB) and where a store fills lines (heads of 64 channels: 88 / 98
  // us for 409 MB; 128 channels with 64 turned by halves: 50 / 65 for 268 MB, 147 / 187 for 671; 256 with 128: 285 / 326 for 1.3 GB).
  const bool stream = 4L * tokens * (a.side[0].heads + a.side[1].heads) * a.D > (128L << 20) && fills_lines(a.D, a.rot, a.layout);
#define THRIFT_ROPE(L_)                                                              \
  if (stream) rope_items_kernel<T, L_, true><<<grid, block, 0, st>>>(a, z);          \
  else rope_items_kernel<T, L_, false><<<grid, block, 0, st>>>(a, z)
  if (a.layout == THRIFT_ROPE_HALF) { THRIFT_ROPE(THRIFT_ROPE_HALF); }
  else { THRIFT_ROPE(THRIFT_ROPE_INTERLEAVED); }
#undef THRIFT_ROPE
}

}  // namespace

void launch_rope(const RopeArgs& a, thrift_dtype dt, hipStream_t st) {
  if (dt == THRIFT_F16) launch<F16>(a, st);
  else launch<BF16>(a, st);
}

}  // namespace thrift
