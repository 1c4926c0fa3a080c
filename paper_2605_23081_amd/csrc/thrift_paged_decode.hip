// Attention of one new token per sequence over a paged 16-bit cache.
//
// A row is one (sequence, KV head) with the G query heads of its group.  Its keys are walked in steps of 32, the heads a column each of
// 16 x 16 matrix tiles:
//   S = K Q^T      32 keys x 16 heads; operand K straight from memory, a lane reads 16 bytes of the row of its key
//   P = 2^(S - m)  in fp32, with the running maximum m of the head; sums in fp32
//   O^T += V^T P^T channels x heads.  A lane reads eight channels (four of 64) of every 128 in the rows of its eight keys and pairs the
//                  rows' halves up (one byte permute per two elements); matrix tile j holds channel j of every lane.  The eight keys are those whose
//                  scores the lane holds, so that P goes from S to the next product without leaving the lane.
// No tile passes through LDS.  P is split into two 16-bit pieces, high and low, for two products.  Rounded once, an fp32 output of bf16 inputs was off by
// 1.1e-4 (1000 tokens) to 3.9e-4 (30000) relative to its norm, with two pieces by 2.4e-7 and 7.5e-7, in the same time (8 x 16384-32768
// tokens, 64/8 heads: 129.0 and 129.1 us).  For fp16, the pieces are those of 2^15 P, so that a piece is a normal number down to 2^-29 of the largest;
// bf16 needs no scale, and its largest values would overflow under one.  The scale is a factor behind the exponential: folded into the
// maximum, m - 15 rounds to another number from 2^24 on, and the largest P to 2^16, which fp16 does not hold.
//
// The steps of all rows are counted through on the GPU from the lengths and cut into equal shares, one per workgroup, whatever the
// lengths are; a wavefront walks a quarter of it, or every fourth step where the share lies in one row.  It asks for the keys of its next step as soon as the scores of this one are
// formed, and for its values as soon as this one's are added, also where the next step is in another row; wavefronts wait for each
// other only at the end, where parts of one row that neighbours hold are joined through LDS.  A row inside one share is written by
// its workgroup; otherwise each share leaves a partial, and a second launch joins a row's partials in the order of the shares.
//
// Bound by memory for long caches: what is fetched are the keys and values of the lengths and nothing else (counters), 8.6 GB for 16 x 131072 tokens,
// 32/8 heads, in 1220 us (7.0 TB/s; a streaming read reaches 7.0-7.15), 775 MB for 8 x 16384-32768, 64/8 heads, in 123-128 us (6.0-6.3 TB/s).  Next to that the
// chain of latencies counts: lengths, sums, page, keys, values (7.0 us of kernel for 1 x 1000 tokens), and the second launch (2.4-5.5 us).
#include "thrift_device.h"
#include "thrift_launch.h"
#include "thrift_paged.h"

namespace thrift {

namespace {

constexpr int kThreads = 256;              // of the merge
// Wavefronts of a share.  256 channels: two, whose 64 KiB on their way are as much as four of 128 channels have (4 x 8192-16384 tokens, 32/8
// heads: 74.1 -> 70.2 us); 64 channels: eight with as much were slower than four (23.6 -> 25.1 us).
constexpr int waves_of(int D) { return D == 256 ? 2 : 4; }
constexpr int kStep = 32;                  // keys per step of a wavefront
constexpr float kLn2 = 0.6931471805599453f;
// One workgroup per CU: its four wavefronts have 64 KiB on their way, 16 MiB on the chip.  More of them ask for more than the memory takes at a
// time, and what waits in front of it is served unevenly (one / two / three per CU: 1220 / 1225 / 1265 us for 16 x 131072 tokens of 32/8 heads,
// 130 / 132 / 150 for 8 x 16384-32768 of 64/8).
constexpr int kShares = kCus;

// scalar loads: the lengths and the table do not change during the launch
typedef const __attribute__((address_space(4))) int32_t* scalar_ints;
__device__ __forceinline__ scalar_ints scalar(const int32_t* p) { return (scalar_ints)(uintptr_t)p; }

struct Mfma16F16 {
  static constexpr float kScale = 32768.f; // of P's pieces
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
};
struct Mfma16BF16 {
  static constexpr float kScale = 1.f;
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  }
};
template <typename T> struct Mma;
template <> struct Mma<F16> : Mfma16F16 {};
template <> struct Mma<BF16> : Mfma16BF16 {};

// largest / sum of the four lanes that are 16 apart, in all of them
__device__ __forceinline__ float over_groups_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return both_halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float over_groups_sum(float x) {
  uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = __float_as_uint(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  const auto t = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// Workspace: the row that every share leaves unfinished, and two partials per share: of a row that an earlier share has begun, and of
// that unfinished row.  O [D], then the maximum and the sum.
struct Space {
  int2* tail;                // [kShares] row (-1: none) and number of shares that it lies in
  float* part_o;             // [2*kShares][G][D]
  float* part_ml;            // [2*kShares][G][2]
};

struct Launch {
  Space w;
  int G, shift;
  float c;                   // softmax scale * log2(e)
};

// a step: which keys of which row
struct Step {
  int b, hk, t, len, steps;                // sequence, KV head, number in the row; the sequence's length and steps
};

__device__ __forceinline__ int length_of(const PagedDecodeArgs& a, const Launch& z, int n) { return min(a.max_pages << z.shift, max(0, n)); }
// len + 31 passes 31 bits at the longest lengths
__device__ __forceinline__ int steps_of(int len) { return (int)(((unsigned)len + kStep - 1) / kStep); }

// What a wavefront holds of a row, and its steps
template <typename T, int D, int NB>
struct Walk {
  static constexpr int KS = D / 32;        // 16-byte pieces of a key's row per lane
  static constexpr int VC = D / 16;        // channels of a value's row per lane
  static constexpr int NR = NB * (VC * 4 + 2);                   // registers of a state
  // the next row's queries are on their way during a step; 32 heads of 256 channels have no registers for that: with it they
  // take 161 us for 64 x 2048-4096 tokens of 64/2 heads, without it 83-90.  They are still short of 26 registers per lane, some of which are
  // reloaded inside the walk; no other form uses scratch memory.
  static constexpr bool kQueryAhead = NB * D < 512;
  static constexpr int kStream = 2;        // non-temporal: keys and values are read once
  int lane, col, grp;
  v4i q[NB][KS], q_next[NB][KS], k[2][KS];
  uint32_t v[8][VC / 2];
  v4f o[NB][VC];                           // kScale o [D] of one head, spread over the four lanes of its column: element r of tile j is channel(r, j)
  float m[NB], l[NB];                      // maximum; this lane's part of the sum
  // Loads of 16 keys go through a descriptor of their page's rows up to the length: what lies behind reads as 0 and is not fetched, and
  // a step that does not exist has none.
  __amdgpu_buffer_rsrc_t kd[2], vd[2];
  int page[2];                             // of a step that is described later: a load of its own in front of the loads

  __device__ __forceinline__ Walk() : lane(threadIdx.x & 63), col(lane & 15), grp(lane >> 4) {}
  __device__ __forceinline__ int channel(int r, int j) const { return (j >> 3) * 128 + (4 * grp + r) * min(VC, 8) + (j & 7); }

  __device__ __forceinline__ void look_up(const PagedDecodeArgs& a, const Launch& z, const Step& s) {
    const scalar_ints table = scalar(a.table + (size_t)s.b * a.max_pages);
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) page[sub] = table[min(a.max_pages - 1, (s.t * kStep + 16 * sub) >> z.shift)];
  }
  __device__ __forceinline__ void describe(const PagedDecodeArgs& a, const Launch& z, const Step& s, bool there) {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const int key = s.t * kStep + 16 * sub, rows = __builtin_amdgcn_readfirstlane(there ? min(16, max(0, s.len - key)) : 0);
      const int p = __builtin_amdgcn_readfirstlane(min(a.n_pages - 1, max(0, page[sub])));
      const size_t at = ((((size_t)p * a.Hkv + s.hk) << z.shift) + (key & ((1 << z.shift) - 1))) * D;
      kd[sub] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.k_pages + at), 0, rows * D * 2, 0x00020000);
      vd[sub] = __builtin_amdgcn_make_buffer_rsrc((void*)(a.v_pages + at), 0, rows * D * 2, 0x00020000);
    }
  }
  __device__ __forceinline__ void load_q(const PagedDecodeArgs& a, const Launch& z, const Step& s, bool there) {
    const uint16_t* qp = a.q + ((size_t)s.b * a.Hkv + s.hk) * z.G * D;
    const __amdgpu_buffer_rsrc_t qd = __builtin_amdgcn_make_buffer_rsrc((void*)qp, 0, there ? z.G * D * 2 : 0, 0x00020000);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < KS; ++e)
        q_next[nb][e] = __builtin_amdgcn_raw_buffer_load_b128(qd, (col + 16 * nb) * D * 2 + 64 * e + 16 * grp, 0, 0);
  }
  __device__ __forceinline__ void next_q() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < KS; ++e) q[nb][e] = q_next[nb][e];
  }
  __device__ __forceinline__ void load_k() {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int e = 0; e < KS; ++e) k[sub][e] = __builtin_amdgcn_raw_buffer_load_b128(kd[sub], col * D * 2 + 16 * grp + 64 * e, 0, kStream);
  }
  __device__ __forceinline__ void load_v() {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int from = 4 * grp * D * 2 + 2 * min(VC, 8) * col + (r & 3) * D * 2;
      if constexpr (VC == 4) {
        const v2i x = __builtin_amdgcn_raw_buffer_load_b64(vd[r >> 2], from, 0, kStream);
        v[r][0] = x[0], v[r][1] = x[1];
      } else {
#pragma unroll
        for (int e = 0; e < VC / 8; ++e) {
          const v4i x = __builtin_amdgcn_raw_buffer_load_b128(vd[r >> 2], from + 256 * e, 0, kStream);
#pragma unroll
          for (int d = 0; d < 4; ++d) v[r][4 * e + d] = x[d];
        }
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb] = -__FLT_MAX__, l[nb] = 0.f;   // a number: scores of -inf then have weight 0
#pragma unroll
      for (int j = 0; j < VC; ++j) o[nb][j] = v4f{0.f, 0.f, 0.f, 0.f};
    }
  }

  // One step, of which the row has `behind` keys from its first on; `ask` when the keys' registers are free
  template <typename F>
  __device__ __forceinline__ void step(float c, int behind, F ask) {
    // A score is rounded once, before the maximum: a fused s c - m would leave the largest one's rounding, units and more from 2^24 on
#pragma clang fp contract(off)
    float x[NB][8];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        v4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < KS; ++e) s = Mma<T>::mma(k[sub][e], q[nb][e], s);
#pragma unroll
        for (int r = 0; r < 4; ++r) x[nb][4 * sub + r] = s[r] * c;
      }
    ask();
    v4i high[NB], low[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (behind < kStep) {
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if ((r < 4 ? 0 : 12) + 4 * grp + r >= behind) x[nb][r] = -__builtin_inff();
      }
      const float (&y)[8] = x[nb];
      const float top = over_groups_max(fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7]))));
      if (__ballot(top > m[nb])) {
        const float grown = fmaxf(top, m[nb]), keep = fast_exp2(m[nb] - grown);
        m[nb] = grown;
        l[nb] *= keep;
#pragma unroll
        for (int j = 0; j < VC; ++j) o[nb][j] *= keep;
      }
      uint16_t hi[8], lo[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float p = fast_exp2(y[r] - m[nb]);
        l[nb] += p;
        const float scaled = p * Mma<T>::kScale;
        hi[r] = T::from_float(scaled);
        lo[r] = T::from_float(scaled - T::to_float(hi[r]));
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        high[nb][r] = (int)((uint32_t)hi[2 * r] | ((uint32_t)hi[2 * r + 1] << 16));
        low[nb][r] = (int)((uint32_t)lo[2 * r] | ((uint32_t)lo[2 * r + 1] << 16));
      }
    }
#pragma unroll
    for (int j = 0; j < VC; ++j) {
      v4i y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (int)__builtin_amdgcn_perm(v[2 * r + 1][j / 2], v[2 * r][j / 2], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        o[nb][j] = Mma<T>::mma(y, high[nb], o[nb][j]);
        o[nb][j] = Mma<T>::mma(y, low[nb], o[nb][j]);
      }
    }
  }

  // The state in LDS, a lane's registers in its column, and the addition of another
  __device__ __forceinline__ void give(float (*to)[64]) const {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float (*p)[64] = to + nb * (VC * 4 + 2);
#pragma unroll
      for (int j = 0; j < VC; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[4 * j + r][lane] = o[nb][j][r];
      p[4 * VC][lane] = m[nb], p[4 * VC + 1][lane] = l[nb];
    }
  }
  __device__ __forceinline__ void take(float (*from)[64]) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float (*p)[64] = from + nb * (VC * 4 + 2);
      const float other = p[4 * VC][lane], top = fmaxf(m[nb], other), k1 = fast_exp2(m[nb] - top), k2 = fast_exp2(other - top);
      m[nb] = top;
      l[nb] = l[nb] * k1 + p[4 * VC + 1][lane] * k2;
#pragma unroll
      for (int j = 0; j < VC; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[nb][j][r] = o[nb][j][r] * k1 + p[4 * j + r][lane] * k2;
    }
  }
  // The state as the row's result, or as a part of it in `slot`
  __device__ __forceinline__ void put(const PagedDecodeArgs& a, const Launch& z, const Step& s, bool whole, size_t slot) const {
    const size_t row = (size_t)s.b * a.Hkv + s.hk;
    constexpr float kUnscale = 1.f / Mma<T>::kScale;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int head = col + 16 * nb;
      const float sum = over_groups_sum(l[nb]), inv = whole ? kUnscale / sum : kUnscale;
      if (head >= z.G) continue;
      if (whole) {
        const size_t to = row * z.G + head;
        if (a.lse != nullptr && grp == 0) a.lse[to] = kLn2 * (m[nb] + __builtin_log2f(sum));
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < VC; j += 4)
            store_out4(a.out, a.out_dt, to * D + channel(r, j), o[nb][j][r] * inv, o[nb][j + 1][r] * inv, o[nb][j + 2][r] * inv, o[nb][j + 3][r] * inv);
      } else {
        const size_t to = slot * z.G + head;
        if (grp == 0) z.w.part_ml[2 * to] = m[nb], z.w.part_ml[2 * to + 1] = sum;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < VC; j += 4)
            *reinterpret_cast<v4f*>(z.w.part_o + to * D + channel(r, j)) = v4f{o[nb][j][r], o[nb][j + 1][r], o[nb][j + 2][r], o[nb][j + 3][r]} * inv;
      }
    }
  }
};

template <typename T, int D, int NB>
__global__ void __launch_bounds__(64 * waves_of(D), D * NB <= 128 ? 2 : 1) paged_decode_kernel(PagedDecodeArgs a, Launch z) {
  constexpr int kWaves = waves_of(D);
  using W = Walk<T, D, NB>;
  __shared__ float parts[kWaves][W::NR][64];                     // a wavefront's part of a row that an earlier one has begun
  __shared__ int ended[kWaves];            // whether the row ends with that part
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;

  // ---- this workgroup's share, steps u .. u_end - 1, and the first one's place ----
  int u = 0, u_end = 0, each = 0, window = 0, lens;         // lens: length of sequence window + lane
  Step cur;
  {
    int n = a.B, per, base = 0, b = 0;
    bool first = true;
    do {                                   // 64 parts of what is left; the part with step u; once more inside it
      per = (n + 63) / 64;
      int sum = 0;
      for (int i = 0; i < per; ++i) {
        const int at = lane * per + i;
        lens = b + at < a.B ? length_of(a, z, a.seqlens[b + at]) : 0;     // the last round's reach past its part: the sequences that follow
        if (at < n) sum += a.Hkv * steps_of(lens);
      }
      int incl = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int other = __shfl_up(incl, d);
        if (lane >= d) incl += other;
      }
      if (first) {
        const int total = __builtin_amdgcn_readlane(incl, 63);
        const int quarter = max(1, (total + kShares * kWaves - 1) / (kShares * kWaves));
        if (threadIdx.x == 0) z.w.tail[blockIdx.x] = make_int2(-1, 0);
        const long begin = (long)blockIdx.x * kWaves * quarter;
        if (begin >= total) return;        // the whole workgroup
        u = (int)begin, u_end = min(total, u + quarter * kWaves);
        each = quarter;
        first = false;
      }
      const int at = __builtin_ctzll(__ballot(base + incl > u));
      base += __builtin_amdgcn_readlane(incl - sum, at);
      window = b;
      b += at * per;
      n = min(per, n - at * per);
    } while (per > 1);                     // the last round has a sequence per lane: its lengths are kept
    // wavefront-uniform, and known to be: descriptors of loads are scalar
    u = __builtin_amdgcn_readfirstlane(u), u_end = __builtin_amdgcn_readfirstlane(u_end);
    window = __builtin_amdgcn_readfirstlane(window), base = __builtin_amdgcn_readfirstlane(base);
    cur.b = __builtin_amdgcn_readfirstlane(b);
    cur.len = __builtin_amdgcn_readlane(lens, cur.b - window);
    cur.steps = steps_of(cur.len);
    cur.hk = __builtin_amdgcn_readfirstlane((u - base) / cur.steps);
    cur.t = (u - base) - cur.hk * cur.steps;
  }
  auto advance = [&](Step& s) {            // there is a step behind
    if (++s.t < s.steps) return;
    s.t = 0;
    if (++s.hk < a.Hkv) return;
    s.hk = 0;
    while (true) {
      const unsigned long long later = __ballot(lens > 0 && lane > s.b - window);
      if (later != 0) {
        const int at = __builtin_ctzll(later);
        s.b = window + at, s.len = __builtin_amdgcn_readlane(lens, at);
        break;
      }
      window += 64, s.b = window - 1;
      lens = window + lane < a.B ? length_of(a, z, a.seqlens[window + lane]) : 0;
    }
    s.steps = steps_of(s.len);
  };

  W w;
  // ---- this wavefront's steps: every fourth where the share lies in one row, which keeps what the four read together, otherwise a quarter
  // of the share, which leaves them one meeting whatever number of rows there is ----
  const bool one_row = cur.t + (u_end - u) <= cur.steps;
  const int stride = one_row ? kWaves : 1;
  int skip = one_row ? wave : wave * each;
  u += skip;
  if (!one_row) u_end = min(u_end, u + each);
  while (skip > 0 && u < u_end) {
    const int room = cur.steps - cur.t;
    if (skip < room) {
      cur.t += skip;
      break;
    }
    skip -= room;
    cur.t = cur.steps - 1;
    advance(cur);
  }
  bool kept = false;                       // the state is the first part of a row that the next wavefronts have more of
  int begin = cur.t, first_u = u;          // this wavefront's first step of the row: in the row, and of all steps
  if (wave > 0 && lane == 0) ended[wave] = u < u_end ? 0 : -1;
  Step next = cur;
  bool more = false;                       // next is a step of this wavefront
  auto follow = [&]() {                    // next becomes the step behind, if there is one, and its pages are asked for
    u += stride;
    more = u < u_end;
    if (one_row) next.t += more ? kWaves : 0;
    else if (more) advance(next);
    w.look_up(a, z, next);
  };
  bool busy = u < u_end;
  if (busy) {
    w.look_up(a, z, cur);
    w.load_q(a, z, cur, true);
    w.describe(a, z, cur, true);
    w.load_k();
    w.load_v();
    w.clear();
    w.next_q();
    follow();
  }
  while (busy) {
    const bool turns = more && next.t == 0;                      // a row begins with the next step
    w.step(z.c, cur.len - cur.t * kStep, [&]() {
      w.describe(a, z, next, more);
      w.load_k();
      if (W::kQueryAhead) w.load_q(a, z, next, turns);
    });
    w.load_v();
    if (!more || turns) {                  // the row ends, or what this wavefront has of it
      const bool ends = cur.t + 1 == cur.steps;
      if (begin > 0 && wave > 0) {         // an earlier wavefront's row
        w.give(parts[wave]);
        if (ends && lane == 0) ended[wave] = 1;
      } else if (ends && !one_row) {
        w.put(a, z, cur, begin == 0, 2 * (size_t)blockIdx.x);
      } else {
        kept = true;
      }
      if (!more) break;
      w.clear();
      if (!W::kQueryAhead) w.load_q(a, z, next, true);
      w.next_q();
      begin = 0, first_u = u;
    }
    cur = next;
    follow();
  }
  __syncthreads();
  if (!kept) return;
  bool ends = cur.t + 1 == cur.steps;
  for (int i = wave + 1; i < kWaves && (one_row || !ends); ++i) {
    if (ended[i] < 0) break;
    w.take(parts[i]);
    ends |= ended[i] > 0;
  }
  w.put(a, z, cur, begin == 0 && ends, 2 * (size_t)blockIdx.x + (begin == 0 ? 1 : 0));
  // the state began with the row's first step, at each * kWaves * (shares so far) + what this share has of other rows; the rest of the
  // row's steps fill the shares behind
  if (begin == 0 && !ends && lane == 0) {
    const int share = each * kWaves, here = min(share - (first_u - (int)blockIdx.x * share), cur.steps);
    z.w.tail[blockIdx.x] = make_int2(cur.b * a.Hkv + cur.hk, 1 + (cur.steps - here + share - 1) / share);
  }
}

// One workgroup per row, for short caches: what it reads first (length, pages, query) does not depend on each other, and there is nothing to
// join afterwards.  Wavefronts take every fourth step (eight instead of four gained nothing); at the end each joins some channels of all
// of them.
constexpr int kRowWaves = 4;
template <typename T, int D>
__global__ void __launch_bounds__(64 * kRowWaves, 1) paged_decode_rows_kernel(PagedDecodeArgs a, Launch z) {
  using Rows = Walk<T, D, 1>;
  constexpr int W = kRowWaves;
  constexpr int VC = Rows::VC;
  __shared__ float parts[W][Rows::NR][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Step cur;
  cur.b = blockIdx.x / a.Hkv, cur.hk = blockIdx.x - cur.b * a.Hkv, cur.t = wave;
  const int n = scalar(a.seqlens)[cur.b];
  Rows w;
  w.look_up(a, z, cur);
  w.load_q(a, z, cur, true);
  cur.len = length_of(a, z, n), cur.steps = steps_of(cur.len);
  const size_t row0 = (size_t)blockIdx.x * z.G;                  // the group's first row of out
  if (cur.len == 0) {
    for (int i = threadIdx.x; i < z.G * D / 4; i += 64 * W) store_out4(a.out, a.out_dt, row0 * D + 4 * (size_t)i, 0.f, 0.f, 0.f, 0.f);
    if (a.lse != nullptr && (int)threadIdx.x < z.G) a.lse[row0 + threadIdx.x] = -__builtin_inff();
    return;
  }
  const int active = min(W, cur.steps);                          // wavefronts with a step
  if (wave < active) {
    w.describe(a, z, cur, true);
    w.load_k();
    w.load_v();
    w.clear();
    w.next_q();
    while (true) {
      Step next = cur;
      next.t += W;
      const bool more = next.t < cur.steps;
      w.look_up(a, z, next);
      w.step(z.c, cur.len - cur.t * kStep, [&]() {
        w.describe(a, z, next, more);
        w.load_k();
      });
      if (!more) break;
      w.load_v();
      cur.t = next.t;
    }
    w.give(parts[wave]);
  }
  __syncthreads();
  // four channels of every lane's head at a time
  if (w.col >= z.G) return;
  float top = -__FLT_MAX__, l = 0.f, weight[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    weight[i] = i < active ? parts[i][4 * VC][lane] : -__FLT_MAX__;
    top = fmaxf(top, weight[i]);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    weight[i] = i < active ? fast_exp2(weight[i] - top) : 0.f;
    if (i < active) {
#pragma unroll
      for (int g = 0; g < 4; ++g) l += weight[i] * parts[i][4 * VC + 1][w.col + 16 * g];
    }
  }
  const float inv = 1.f / (Mma<T>::kScale * l);
  const size_t to = row0 + w.col;
  if (a.lse != nullptr && threadIdx.x == w.col) a.lse[to] = kLn2 * (top + __builtin_log2f(l));
  for (int u = wave; u < VC; u += W) {
    const int r = u & 3, j = 4 * (u >> 2);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < active) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += weight[i] * parts[i][4 * (j + e) + r][lane];
      }
    store_out4(a.out, a.out_dt, to * D + w.channel(r, j), x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  }
}

// One workgroup per share and head of a group: joins the partials of the row that the share leaves unfinished.  Threads take four channels
// of every kParts-th partial with a running maximum of their own, so that a partial's maximum, sum and channels are asked
// for together.  Sequences without tokens become 0.
template <int D>
__global__ void __launch_bounds__(kThreads) paged_merge_kernel(PagedDecodeArgs a, Launch z) {
  constexpr int kQuads = D / 4, kParts = kThreads / kQuads, kAhead = 4;
  __shared__ float2 ml[kParts];
  __shared__ __align__(16) v4f sums[kParts][kQuads];
  const int tid = threadIdx.x, first = blockIdx.x / z.G, g = blockIdx.x % z.G;
  const int quad = tid % kQuads, part = tid / kQuads;
  const int2 tail = z.w.tail[first];
  // partial w of the row that begins in share `first`
  auto slot = [&](int w) { return (size_t)(2 * (first + w) + (w == 0 ? 1 : 0)) * z.G + g; };
  // the first kParts of them before it is known how many there are, or whether there are any
  const size_t ahead = slot(min(part, kShares - 1 - first));
  const v4f x0 = *reinterpret_cast<const v4f*>(z.w.part_o + ahead * D + 4 * quad);
  const float2 y0 = *reinterpret_cast<const float2*>(z.w.part_ml + 2 * ahead);
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    if (a.seqlens[b] > 0) continue;
    for (int i = tid; i < a.Hq * kQuads; i += kThreads) store_out4(a.out, a.out_dt, (size_t)b * a.Hq * D + 4 * (size_t)i, 0.f, 0.f, 0.f, 0.f);
    if (a.lse != nullptr)
      for (int h = tid; h < a.Hq; h += kThreads) a.lse[(size_t)b * a.Hq + h] = -__builtin_inff();
  }
  const int n = tail.y;
  if (tail.x < 0) return;
  const size_t at = (size_t)tail.x * z.G + g;
  v4f o = {0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  if (part < n) o = x0, m = y0.x, l = y0.y;
  for (int i0 = part + kParts; i0 < n; i0 += kParts * kAhead) {
    v4f x[kAhead];
    float2 y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int w = min(n - 1, i0 + i * kParts);
      const size_t s = slot(w);
      x[i] = *reinterpret_cast<const v4f*>(z.w.part_o + s * D + 4 * quad);
      y[i] = *reinterpret_cast<const float2*>(z.w.part_ml + 2 * s);
      if (i0 + i * kParts >= n) y[i] = make_float2(-__builtin_inff(), 0.f);
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) top = fmaxf(top, y[i].x);
    const float keep = fast_exp2(m - top);
    m = top, l *= keep, o *= keep;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float k = fast_exp2(y[i].x - top);
      l += k * y[i].y, o += k * x[i];
    }
  }
  if (quad == 0) ml[part] = make_float2(m, l);
  sums[part][quad] = o;
  __syncthreads();
  if (part != 0) return;
  float top = ml[0].x, sum = 0.f;
#pragma unroll
  for (int i = 1; i < kParts; ++i) top = fmaxf(top, ml[i].x);
  o = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const float k = fast_exp2(ml[i].x - top);
    sum += k * ml[i].y, o += k * sums[i][quad];
  }
  const float inv = 1.f / sum;
  store_out4(a.out, a.out_dt, at * D + 4 * quad, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (a.lse != nullptr && tid == 0) a.lse[at] = kLn2 * (top + __builtin_log2f(sum));
}

// A CU takes about 40 GB/s from memory, so that a row of its own costs it 6.4 us for 256 KiB of keys and values; where the block table has room for no
// more, that is less than the search for a share and the second launch.  Shares / rows, us, 32/8 heads of 128 channels: 10.3 / 6.3 for 1 x 256,
// 10.7 / 5.7 for 16 x 50-100, 12.8 / 10.7 for 16 x 250-500, 54.3 / 54.6 for 256 x 125-500; beyond: 10.3 / 12.5 for 1 x 1000, 15.2 / 17.8 for
// 16 x 500-1000.  64 channels: 14.0 / 11.5 for 64 x 125-500; 256 channels: 12.5 / 16.2 for 4 x 250-500, 16/16 heads.
// With more than four rows per CU the shares are as fast (33.8 / 33.7 for 256 x 63-250) or faster (160 / 226 for 4096 x 15-60).
constexpr long kRowBytes = 256 << 10, kRowMost = 4 * kCus;
bool by_rows(int B, int Hq, int Hkv, int max_pages, int page_size, int D) {
  return Hq / Hkv <= 16 && (long)max_pages * page_size * D * 4 <= kRowBytes && (long)B * Hkv <= kRowMost;
}

template <typename T>
void launch(const PagedDecodeArgs& a, const Launch& z, hipStream_t st) {
  if (by_rows(a.B, a.Hq, a.Hkv, a.max_pages, a.page_size, a.D)) {
    const dim3 rows((unsigned)((long)a.B * a.Hkv)), block(64 * kRowWaves);
    if (a.D == 64) paged_decode_rows_kernel<T, 64><<<rows, block, 0, st>>>(a, z);
    else if (a.D == 128) paged_decode_rows_kernel<T, 128><<<rows, block, 0, st>>>(a, z);
    else paged_decode_rows_kernel<T, 256><<<rows, block, 0, st>>>(a, z);
    return;
  }
  const dim3 grid(kShares), merge(kShares * z.G), block(kThreads);
#define THRIFT_PAGED(D_)                                                                     \
  if (z.G <= 16) paged_decode_kernel<T, D_, 1><<<grid, dim3(64 * waves_of(D_)), 0, st>>>(a, z);                \
  else paged_decode_kernel<T, D_, 2><<<grid, dim3(64 * waves_of(D_)), 0, st>>>(a, z);                          \
  paged_merge_kernel<D_><<<merge, block, 0, st>>>(a, z)
  if (a.D == 64) { THRIFT_PAGED(64); }
  else if (a.D == 128) { THRIFT_PAGED(128); }
  else { THRIFT_PAGED(256); }
#undef THRIFT_PAGED
}

constexpr size_t kTailBytes = kShares * sizeof(int2);

}  // namespace

size_t paged_decode_workspace(int B, int Hq, int Hkv, int max_pages, int page_size, int D) {
  if (by_rows(B, Hq, Hkv, max_pages, page_size, D)) return 0;
  return kTailBytes + 2 * (size_t)kShares * (Hq / Hkv) * (D + 2) * sizeof(float);
}

void launch_paged_decode(const PagedDecodeArgs& a, hipStream_t st) {
  Launch z;
  z.G = a.Hq / a.Hkv;
  z.shift = __builtin_ctz(a.page_size);
  z.c = a.scale * 1.4426950408889634f;
  char* w = (char*)a.workspace;
  z.w.tail = (int2*)w;
  z.w.part_o = (float*)(w + kTailBytes);
  z.w.part_ml = z.w.part_o + 2 * (size_t)kShares * z.G * a.D;
  if (a.dt == THRIFT_F16) launch<F16>(a, z, st);
  else launch<BF16>(a, z, st);
}

}  // namespace thrift
