// New tokens into the 8-bit paged cache: rotation as in thrift_pages.hip, then the scale of every head and its codes.
#include "thrift_e4m3.h"
#include "thrift_paged.h"
#include "thrift_rotary.h"

namespace thrift {

namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kPairs = kRopeMaxDim / 2 / 64;           // of a lane at most

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// One workgroup per row, a wavefront per head, a lane per pair of channels; cos and sin are formed once for all heads.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) paged_append8_kernel(PagedAppend8Args args) {
  __shared__ float2 angles[kRopeMaxDim / 2];
  const PagedAppendArgs& a = args.in;
  const long t = blockIdx.x;
  const int slot = a.slots[t], lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (slot < 0 || slot >= a.n_pages * a.page_size) return;
  const size_t page = slot / a.page_size, in_page = slot % a.page_size;
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < half; i += kRowThreads) {
    float c, s;
    turn(a.positions[t], a.freqs[i], a.gain, c, s);
    angles[i] = make_float2(c, s);
  }
  __syncthreads();
  // pair i: the channels that turn together, and behind the rotated part neighbours
  auto channels = [&](int i, int& i0, int& i1) {
    const bool apart = a.layout == THRIFT_ROPE_HALF && i < half;
    i0 = apart ? i : 2 * i, i1 = apart ? i + half : 2 * i + 1;
  };
  for (int h = wave; h < a.Hq; h += kRowWaves) {
    const uint16_t* x = a.q + t * a.qt + h * a.qh;
    uint16_t* y = a.q_out + ((size_t)t * a.Hq + h) * a.D;
    for (int i = lane; 2 * i < a.D; i += 64) {
      int i0, i1;
      channels(i, i0, i1);
      const uint16_t x0 = x[i0], x1 = x[i1];
      float y0, y1;
      if (i < half) rotate(T::to_float(x0), T::to_float(x1), angles[i].x, angles[i].y, y0, y1);
      y[i0] = i < half ? T::from_float(y0) : x0, y[i1] = i < half ? T::from_float(y1) : x1;
    }
  }
  for (int u = wave; u < 2 * a.Hkv; u += kRowWaves) {
    const bool key = u < a.Hkv;
    const int h = key ? u : u - a.Hkv;
    const uint16_t* x = key ? a.k + t * a.kt + h * a.kh : a.v + t * a.vt + h * a.vh;
    float y0[kPairs], y1[kPairs], top = 0.f;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      const int i = lane + 64 * e;
      y0[e] = y1[e] = 0.f;
      if (2 * i < a.D) {
        int i0, i1;
        channels(i, i0, i1);
        const float x0 = T::to_float(x[i0]), x1 = T::to_float(x[i1]);
        if (key && i < half) rotate(x0, x1, angles[i].x, angles[i].y, y0[e], y1[e]);
        else y0[e] = x0, y1[e] = x1;
        top = fmaxf(top, fmaxf(fabsf(finite_or_zero(y0[e])), fabsf(finite_or_zero(y1[e]))));
      }
    }
    const int exponent = e4m3_exponent(wave_max(top));
    const float inv = power_of_two(-exponent);
    const size_t row = (page * a.Hkv + h) * a.page_size + in_page;
    if (lane == 0) (key ? args.k_scales : args.v_scales)[row] = (uint8_t)(exponent + 127);
    uint8_t* codes = (key ? args.k_codes : args.v_codes) + row * a.D;
#pragma unroll
    for (int e = 0; e < kPairs; ++e) {
      const int i = lane + 64 * e;
      if (2 * i >= a.D) continue;
      int i0, i1;
      channels(i, i0, i1);
      const uint32_t both = e4m3_pair<false>(0, y0[e], y1[e], inv);
      codes[i0] = (uint8_t)both, codes[i1] = (uint8_t)(both >> 8);
    }
  }
}

// The chunks of one head as fp32, turned where `turned`.
template <typename T, int LAYOUT>
__device__ __forceinline__ void chunk_values(const Item<LAYOUT>& it, const v4i (&x)[2], const float2 (&cs)[8], bool turned, float (&y)[2][8]) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int d = 0; d < 4; ++d) y[c][2 * d] = T::to_float((uint16_t)x[c][d]), y[c][2 * d + 1] = T::to_float((uint16_t)((uint32_t)x[c][d] >> 16));
  if (!turned) return;
  if (LAYOUT == THRIFT_ROPE_HALF) {
    if (it.turned[0]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x0 = y[0][e], x1 = y[1][e];
        rotate(x0, x1, cs[e].x, cs[e].y, y[0][e], y[1][e]);
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (it.turned[c]) {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const float x0 = y[c][2 * d], x1 = y[c][2 * d + 1];
          rotate(x0, x1, cs[4 * c + d].x, cs[4 * c + d].y, y[c][2 * d], y[c][2 * d + 1]);
        }
      }
  }
}

// The same in 16-byte chunks, as the append to the 16-bit cache: the query heads of a row, then its key heads, then its value heads.  A head is
// D / 16 neighbouring lanes, a power of two of them, which find its largest magnitude between them.
template <typename T, int LAYOUT, bool STREAM>
__global__ void __launch_bounds__(kHeadThreads) paged_append8_items_kernel(PagedAppend8Args args, HeadShape z) {
  __shared__ float2 table[kAngles];
  const PagedAppendArgs& a = args.in;
  const int tid = threadIdx.x, half = a.rot / 2;
  const int first = (int)(blockIdx.x / z.splits) * z.tokens, split = blockIdx.x % z.splits;
  const int item = tid % z.items, rest = tid / z.items, local = rest % z.tokens, group = rest / z.tokens;
  const int t = first + local, turned = a.Hq + a.Hkv, heads = turned + a.Hkv;
  const int slot = group < z.lanes && t < a.T ? a.slots[t] : -1;
  const bool busy = slot >= 0 && slot < a.n_pages * a.page_size;
  const Item<LAYOUT> it(item, a.D, a.rot);
  const uint16_t *q = a.q + t * a.qt, *k = a.k + t * a.kt, *v = a.v + t * a.vt;
  const int shift = 31 - __builtin_clz(a.page_size);
  const size_t row0 = (((size_t)(slot >> shift) * a.Hkv) << shift) + (slot & (a.page_size - 1));
  uint16_t* q_out = a.q_out + (size_t)t * a.Hq * a.D;
  const int step = z.lanes * z.splits;
  int h = busy ? split * z.lanes + group : heads;
  auto load = [&](int i, v4i (&c)[2]) {
    const uint16_t* p = i < a.Hq ? q + i * a.qh : i < turned ? k + (i - a.Hq) * a.kh : v + (i - turned) * a.vh;
    c[0] = chunk_from<false>(p + it.at[0]), c[1] = chunk_from<false>(p + it.at[1]);
  };
  v4i c[2];
  if (h < heads) load(h, c);                 // on its way while the angles are formed
  for (int i = tid; i < z.tokens * half; i += kHeadThreads) {
    const int row = first + i / half;
    if (row >= a.T) break;
    float cs, sn;
    turn(a.positions[row], a.freqs[i % half], a.gain, cs, sn);
    table[i] = make_float2(cs, sn);
  }
  __syncthreads();
  float2 cs[8];
  if (busy) it.angles(table + local * half, cs);
  while (h < heads) {
    const int now = h;
    h += step;
    v4i next[2];
    if (h < heads) load(h, next);
    if (now < a.Hq) {
      uint16_t* p = q_out + (size_t)now * a.D;
      turn_item<T, LAYOUT>(it, c, cs);
      chunk_to<STREAM>(p + it.at[0], c[0]), chunk_to<STREAM>(p + it.at[1], c[1]);
    } else {
      const bool key = now < turned;
      float y[2][8], top = 0.f;
      chunk_values<T, LAYOUT>(it, c, cs, key, y);
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(finite_or_zero(y[i >> 3][i & 7])));
      for (int d = 1; d < z.items; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
      const int exponent = e4m3_exponent(top);
      const float inv = power_of_two(-exponent);
      const size_t row = row0 + ((size_t)(now - (key ? a.Hq : turned)) << shift);
      if (item == 0) (key ? args.k_scales : args.v_scales)[row] = (uint8_t)(exponent + 127);
      uint8_t* codes = (key ? args.k_codes : args.v_codes) + row * a.D;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v2i x;
#pragma unroll
        for (int d = 0; d < 2; ++d)
          x[d] = (int)e4m3_pair<true>(e4m3_pair<false>(0, y[i][4 * d], y[i][4 * d + 1], inv), y[i][4 * d + 2], y[i][4 * d + 3], inv);
        *reinterpret_cast<v2i*>(codes + it.at[i]) = x;
      }
    }
    c[0] = next[0], c[1] = next[1];
  }
}

// A workgroup takes as few tokens as still give every thread a head, mostly one, and goes over its heads two or three times.  The kernel is bound by
// memory; workgroups of eight tokens turn more heads per formed angle, but are a fraction of the number (eight / one, us): 72 / 60 for 8192 tokens of 64/8 heads
// (319 MB, 5.3 TB/s), 147 / 130 for 32768 of 32/8, 13.8 / 11.5 for 8192 of 16/2 heads of 64 channels, 7.2 / 7.8 for 1024 of 32/8.  72 registers, seven wavefronts per SIMD (fp16
// in the interleaved layout: 88 and five).  Reading past the caches takes 57 for the first, but 21 instead of 18 where the heads, 50 MB, were just written.
HeadShape shape_of(const PagedAppendArgs& a) {
  const int total = a.Hq + 2 * a.Hkv;
  HeadShape z = head_shape(a.T, total, a.D, a.rot);
  int tokens = 1;
  while (tokens < z.tokens && 2 * z.items * tokens * total <= kHeadThreads) tokens *= 2;
  z.tokens = tokens;
  z.lanes = kHeadThreads / (z.items * tokens);
  if (z.lanes > total) z.lanes = total;
  const long groups = ((long)a.T + tokens - 1) / tokens, most = (total + z.lanes - 1) / z.lanes, wanted = (2048 + groups - 1) / groups;
  z.splits = (int)(wanted < most ? wanted : most);
  return z;
}

template <typename T>
void launch_append8(const PagedAppend8Args& args, hipStream_t st) {
  const PagedAppendArgs& a = args.in;
  const uintptr_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.q_out;
  if (a.D % 16 != 0 || (a.D & (a.D - 1)) != 0 || a.rot % 16 != 0 || at % 16 != 0 || (((uintptr_t)args.k_codes | (uintptr_t)args.v_codes) & 7) != 0 ||
      ((a.q ? a.qt | a.qh : 0) | a.kt | a.kh | a.vt | a.vh) % 8 != 0) {
    paged_append8_kernel<T><<<dim3((unsigned)a.T), dim3(kRowThreads), 0, st>>>(args);
    return;
  }
  const HeadShape z = shape_of(a);
  const dim3 grid((unsigned)((a.T + z.tokens - 1) / z.tokens * z.splits)), block(kHeadThreads);
  const bool stream = fills_lines(a.D, a.rot, a.layout);
#define THRIFT_APPEND8(L_)                                                                    \
  if (stream) paged_append8_items_kernel<T, L_, true><<<grid, block, 0, st>>>(args, z);       \
  else paged_append8_items_kernel<T, L_, false><<<grid, block, 0, st>>>(args, z)
  if (a.layout == THRIFT_ROPE_HALF) { THRIFT_APPEND8(THRIFT_ROPE_HALF); }
  else { THRIFT_APPEND8(THRIFT_ROPE_INTERLEAVED); }
#undef THRIFT_APPEND8
}

}  // namespace

void launch_paged_append8(const PagedAppend8Args& a, thrift_dtype dt, hipStream_t st) {
  if (dt == THRIFT_F16) launch_append8<F16>(a, st);
  else launch_append8<BF16>(a, st);
}

}  // namespace thrift
