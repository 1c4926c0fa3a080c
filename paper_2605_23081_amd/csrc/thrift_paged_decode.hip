// Attention of one new token per sequence over a paged 16-bit cache.
//
// A row is one (sequence, KV head) with the G query heads of its group.  Its keys are walked in steps of 32, the heads a column each of
// 16 x 16 matrix tiles:
//   S = K Q^T      32 keys x 16 heads; operand K straight from memory, a lane reads 16 bytes of the row of its key
//   P = 2^(S - m)  in fp32, with the running maximum m of the head; sums in fp32
//   O^T += V^T P^T channels x heads.  A lane reads the channels D/16 c .. of the rows of its eight keys and pairs the rows' halves
//                  up (one byte permute per two elements); matrix tile j holds channel j of every lane.  The eight keys are those whose
//                  scores the lane holds, so that P goes from S to the next product without leaving the lane.
// No tile passes through LDS and nothing waits for a barrier inside the walk.  P is split into two 16-bit pieces, high and low,
// for two products: rounding it once would cost an output of 16 bits as much accuracy again as the output's own rounding.
// P is scaled by 2^15, so that an fp16 piece is a normal number down to 2^-29 of the largest.
//
// The steps of all rows are counted through on the GPU from the lengths and cut into equal shares, one per workgroup, whatever the
// lengths are.  In a workgroup the steps of a row go to the four wavefronts in turn; their states are joined in LDS when the row
// or the share ends.  A row inside one share is written by its workgroup; otherwise each share leaves a partial, and a second launch
// joins a row's partials in the order of the shares.
#include "thrift_device.h"
#include "thrift_launch.h"
#include "thrift_paged.h"

namespace thrift {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kStep = 32;                  // keys per step of a wavefront
constexpr int kLeastShare = kWaves;        // steps
constexpr float kShift = 15.f;

// scalar loads: the lengths and the table do not change during the launch
typedef const __attribute__((address_space(4))) int32_t* scalar_ints;
__device__ __forceinline__ scalar_ints scalar(const int32_t* p) { return (scalar_ints)(uintptr_t)p; }

struct Mfma16F16 {
  static __device__ __forceinline__ v4f mma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
  }
};
struct Mfma16BF16 {
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

// Workspace: [0] steps per share, then the first step of every row, then the partials (two per share): O [D], then m - 15 and the sum.
struct Space {
  int* share;
  int* row_start;            // [B*Hkv]
  float* part_o;             // [2*shares][G][D]
  float* part_ml;            // [2*shares][G][2]
};

struct Launch {
  Space w;
  int G, shift, shares;
  float c;                   // softmax scale * log2(e)
};

// The state of one head: o [D] spread over the four lanes of the head, m (less 15) and this lane's part of the sum
template <int NB, int VC>
struct State {
  v4f o[NB][VC];
  float m[NB], l[NB];
};

// workgroups per CU that the registers allow
constexpr int resident(int D, int NB) { return D == 64 ? (NB == 1 ? 4 : 3) : D == 128 ? (NB == 1 ? 3 : 2) : (NB == 1 ? 2 : 1); }

template <typename T, int D, int NB>
__global__ void __launch_bounds__(kThreads, resident(D, NB)) paged_decode_kernel(PagedDecodeArgs a, Launch z) {
  constexpr int KS = D / 32;               // 16-byte pieces of a key's row per lane
  constexpr int VC = D / 16;               // channels of a value's row per lane
  constexpr int NR = NB * (VC * 4 + 2);    // registers of a state
  __shared__ __align__(16) float joined[2][NR][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, grp = lane >> 4;
  const scalar_ints seqlens = scalar(a.seqlens);
  const int capacity = a.max_pages << z.shift;
  auto length = [&](int n) { return min(capacity, max(0, n)); };
  auto steps_of = [&](int len) { return (len + kStep - 1) / kStep; };

  // ---- this workgroup's share: total, first step, and the sequence it lies in ----
  int u, u_end, b = 0, left;               // left: steps of the sequence in front of u
  {
    int n = a.B, base = 0, total = 0;
    u = 0; u_end = 0;
    bool first = true;
    do {
      const int per = (n + 63) / 64;
      int sum = 0;
      for (int i = 0; i < per; ++i) {
        const int at = lane * per + i;
        if (at < n) sum += a.Hkv * steps_of(length(a.seqlens[b + at]));
      }
      int incl = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int other = __shfl_up(incl, d);
        if (lane >= d) incl += other;
      }
      if (first) {
        total = __builtin_amdgcn_readlane(incl, 63);
        const int share = max(kLeastShare, (total + z.shares - 1) / z.shares);
        if (blockIdx.x == 0 && tid == 0) z.w.share[0] = share;
        const long from = (long)blockIdx.x * share;
        if (from >= total) return;
        u = (int)from;
        u_end = min(total, u + share);
        first = false;
      }
      const int at = __builtin_ctzll(__ballot(base + incl > u));
      base += __builtin_amdgcn_readlane(incl - sum, at);
      b += at * per;
      n = min(per, n - at * per);
    } while (n > 1);
    left = u - base;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  int len = length(seqlens[b]), steps = steps_of(len);
  int hk = left / steps, t = left - hk * steps;

  while (true) {
    // ---- one segment: steps t .. t_end - 1 of row (b, hk) ----
    const int t_end = min(steps, t + (u_end - u));
    const scalar_ints table = scalar(a.table + (size_t)b * a.max_pages);
    const size_t row = (size_t)b * a.Hkv + hk;
    if (t == 0 && tid == 0) z.w.row_start[row] = u;

    v4i q[NB][KS];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int head = col + 16 * nb;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        q[nb][s] = head < z.G ? *reinterpret_cast<const v4i*>(a.q + (row * z.G + head) * D + 32 * s + 8 * grp) : v4i{0, 0, 0, 0};
    }
    State<NB, VC> st;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      st.m[nb] = -__builtin_inff(), st.l[nb] = 0.f;
#pragma unroll
      for (int j = 0; j < VC; ++j) st.o[nb][j] = v4f{0.f, 0.f, 0.f, 0.f};
    }

    // element offset of the 16 keys from key on
    auto place = [&](int key) {
      const int page = min(a.n_pages - 1, max(0, table[min(a.max_pages - 1, key >> z.shift)]));
      return ((((size_t)page * a.Hkv + hk) << z.shift) + (key & ((1 << z.shift) - 1))) * D;
    };
    for (int i = t + wave; i < t_end; i += kWaves) {
      const int key0 = i * kStep;
      v4i k[2][KS];
      uint32_t v[8][VC / 2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const size_t at = place(key0 + 16 * sub);
        const uint16_t* kp = a.k_pages + at + col * D + 8 * grp;
        const uint16_t* vp = a.v_pages + at + 4 * grp * D + VC * col;
#pragma unroll
        for (int s = 0; s < KS; ++s) k[sub][s] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(kp + 32 * s));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (VC == 4) {
            const v2i x = __builtin_nontemporal_load(reinterpret_cast<const v2i*>(vp + r * D));
            v[4 * sub + r][0] = x[0], v[4 * sub + r][1] = x[1];
          } else {
#pragma unroll
            for (int e = 0; e < VC / 8; ++e) {
              const v4i x = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(vp + r * D + 8 * e));
#pragma unroll
              for (int d = 0; d < 4; ++d) v[4 * sub + r][4 * e + d] = x[d];
            }
          }
        }
      }
      const bool tail = key0 + kStep > len;
      v4i high[NB], low[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float x[8];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          v4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < KS; ++e) s = Mma<T>::mma(k[sub][e], q[nb][e], s);
#pragma unroll
          for (int r = 0; r < 4; ++r) x[4 * sub + r] = s[r] * z.c;
        }
        if (tail) {
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (key0 + (r < 4 ? 0 : 12) + 4 * grp + r >= len) x[r] = -__builtin_inff();
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = over_groups_max(top) - kShift;
        if (__ballot(top > st.m[nb])) {
          const float m = fmaxf(top, st.m[nb]), keep = fast_exp2(st.m[nb] - m);
          st.m[nb] = m;
          st.l[nb] *= keep;
#pragma unroll
          for (int j = 0; j < VC; ++j) st.o[nb][j] *= keep;
        }
        uint16_t hi[8], lo[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float p = fast_exp2(x[r] - st.m[nb]);
          st.l[nb] += p;
          hi[r] = T::from_float(p);
          lo[r] = T::from_float(p - T::to_float(hi[r]));
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          high[nb][r] = (int)((uint32_t)hi[2 * r] | ((uint32_t)hi[2 * r + 1] << 16));
          low[nb][r] = (int)((uint32_t)lo[2 * r] | ((uint32_t)lo[2 * r + 1] << 16));
        }
      }
      if (tail) {                          // 0 times whatever lies past the length would not be 0
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (key0 + (r < 4 ? 0 : 12) + 4 * grp + r >= len) {
#pragma unroll
            for (int d = 0; d < VC / 2; ++d) v[r][d] = 0;
          }
      }
#pragma unroll
      for (int j = 0; j < VC; ++j) {
        v4i x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = (int)__builtin_amdgcn_perm(v[2 * r + 1][j / 2], v[2 * r][j / 2], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          st.o[nb][j] = Mma<T>::mma(x, high[nb], st.o[nb][j]);
          st.o[nb][j] = Mma<T>::mma(x, low[nb], st.o[nb][j]);
        }
      }
    }

    // ---- join the wavefronts: 2 into 0 and 3 into 1, then 1 into 0 ----
    auto give = [&](float (*to)[64]) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float (*p)[64] = to + nb * (VC * 4 + 2);
#pragma unroll
        for (int j = 0; j < VC; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) p[4 * j + r][lane] = st.o[nb][j][r];
        p[4 * VC][lane] = st.m[nb], p[4 * VC + 1][lane] = st.l[nb];
      }
    };
    auto take = [&](float (*from)[64]) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float (*p)[64] = from + nb * (VC * 4 + 2);
        const float m2 = p[4 * VC][lane], m = fmaxf(st.m[nb], m2);
        const float k1 = st.m[nb] == m ? 1.f : fast_exp2(st.m[nb] - m), k2 = m2 == -__builtin_inff() ? 0.f : fast_exp2(m2 - m);
        st.m[nb] = m;
        st.l[nb] = st.l[nb] * k1 + p[4 * VC + 1][lane] * k2;
#pragma unroll
        for (int j = 0; j < VC; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) st.o[nb][j][r] = st.o[nb][j][r] * k1 + p[4 * j + r][lane] * k2;
      }
    };
    if (wave >= 2) give(joined[wave - 2]);
    __syncthreads();
    if (wave < 2) take(joined[wave]);
    if (wave == 1) give(joined[1]);
    __syncthreads();
    if (wave == 0) {
      take(joined[1]);
      const bool whole = t == 0 && t_end == steps;
      const int slot = 2 * (int)blockIdx.x + (t == 0 ? 1 : 0);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int head = col + 16 * nb;
        const float l = over_groups_sum(st.l[nb]), inv = 1.f / l;
        if (head >= z.G) continue;
        if (whole) {
          const size_t at = row * z.G + head;
          if (a.lse != nullptr && grp == 0) a.lse[at] = 0.6931471805599453f * (st.m[nb] + __builtin_log2f(l));
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VC; j += 4)
              store_out4(a.out, a.out_dt, at * D + (4 * grp + r) * VC + j, st.o[nb][j][r] * inv, st.o[nb][j + 1][r] * inv, st.o[nb][j + 2][r] * inv, st.o[nb][j + 3][r] * inv);
        } else {
          const size_t at = (size_t)slot * z.G + head;
          if (grp == 0) z.w.part_ml[2 * at] = st.m[nb], z.w.part_ml[2 * at + 1] = l;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < VC; j += 4)
              *reinterpret_cast<v4f*>(z.w.part_o + at * D + (4 * grp + r) * VC + j) = v4f{st.o[nb][j][r], st.o[nb][j + 1][r], st.o[nb][j + 2][r], st.o[nb][j + 3][r]};
        }
      }
    }
    u += t_end - t;
    if (u >= u_end) return;
    t = 0;
    if (++hk == a.Hkv) {
      hk = 0;
      do len = length(seqlens[++b]); while (len == 0);       // u < u_end: there is a sequence with tokens behind
      steps = steps_of(len);
    }
    __syncthreads();                       // wavefront 0 has read what the next segment overwrites
  }
}

// One workgroup per (sequence, query head): joins the partials of a row that several shares have; rows without tokens become 0.
template <int D>
__global__ void __launch_bounds__(256) paged_merge_kernel(PagedDecodeArgs a, Launch z) {
  constexpr int kQuads = D / 4, kParts = 256 / kQuads;      // float4 columns; partials side by side
  __shared__ float scale_of[256];
  __shared__ float top_of[4], sum_of[4];
  __shared__ __align__(16) v4f sums[kParts][kQuads];
  const int tid = threadIdx.x, b = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, hk = h / z.G;
  const int len = min(a.max_pages << z.shift, max(0, a.seqlens[b])), steps = (len + kStep - 1) / kStep;
  const size_t at = (size_t)b * a.Hq + h;
  const int quad = tid % kQuads, part = tid / kQuads;
  if (len == 0) {
    if (part == 0) store_out4(a.out, a.out_dt, at * D + 4 * quad, 0.f, 0.f, 0.f, 0.f);
    if (a.lse != nullptr && tid == 0) a.lse[at] = -__builtin_inff();
    return;
  }
  const int share = z.w.share[0], u = z.w.row_start[(size_t)b * a.Hkv + hk];
  const int first = u / share, n = (u + steps - 1) / share - first + 1;
  if (n == 1) return;                                       // inside one share: written already
  auto slot = [&](int i) { return (size_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * z.G + (h - hk * z.G); };
  // the largest maximum of all partials
  float top = -__builtin_inff();
  for (int i = tid; i < n; i += 256) top = fmaxf(top, z.w.part_ml[2 * slot(i)]);
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) top_of[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
  v4f o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int i0 = 0; i0 < n; i0 += 256) {
    if (i0 > 0) __syncthreads();
    if (i0 + tid < n) {
      const size_t s = slot(i0 + tid);
      const float k = fast_exp2(z.w.part_ml[2 * s] - top);
      scale_of[tid] = k;
      l += k * z.w.part_ml[2 * s + 1];
    }
    __syncthreads();
    const int count = min(256, n - i0);
    for (int i = part; i < count; i += kParts) o += scale_of[i] * *reinterpret_cast<const v4f*>(z.w.part_o + slot(i0 + i) * D + 4 * quad);
  }
  for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
  if ((tid & 63) == 0) sum_of[tid >> 6] = l;
  sums[part][quad] = o;
  __syncthreads();
  if (part != 0) return;
  l = (sum_of[0] + sum_of[1]) + (sum_of[2] + sum_of[3]);
  for (int i = 1; i < kParts; ++i) o += sums[i][quad];
  const float inv = 1.f / l;
  store_out4(a.out, a.out_dt, at * D + 4 * quad, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (a.lse != nullptr && tid == 0) a.lse[at] = 0.6931471805599453f * (top + __builtin_log2f(l));
}

int shares_of(int D, int G) { return kCus * resident(D, G > 16 ? 2 : 1); }

template <typename T>
void launch(const PagedDecodeArgs& a, const Launch& z, hipStream_t st) {
  const dim3 grid(z.shares), merge((unsigned)((long)a.B * a.Hq)), block(kThreads);
#define THRIFT_PAGED(D_)                                                                     \
  if (z.G <= 16) paged_decode_kernel<T, D_, 1><<<grid, block, 0, st>>>(a, z);                \
  else paged_decode_kernel<T, D_, 2><<<grid, block, 0, st>>>(a, z);                          \
  paged_merge_kernel<D_><<<merge, dim3(256), 0, st>>>(a, z)
  if (a.D == 64) { THRIFT_PAGED(64); }
  else if (a.D == 128) { THRIFT_PAGED(128); }
  else { THRIFT_PAGED(256); }
#undef THRIFT_PAGED
}

size_t aligned(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t paged_decode_workspace(int B, int Hq, int Hkv, int, int, int D) {
  const size_t G = Hq / Hkv, slots = 2 * (size_t)shares_of(D, (int)G);
  return 256 + aligned((size_t)B * Hkv * sizeof(int)) + aligned(slots * G * D * sizeof(float)) + aligned(slots * G * 2 * sizeof(float));
}

void launch_paged_decode(const PagedDecodeArgs& a, hipStream_t st) {
  Launch z;
  z.G = a.Hq / a.Hkv;
  z.shift = __builtin_ctz(a.page_size);
  z.shares = shares_of(a.D, z.G);
  z.c = a.scale * 1.4426950408889634f;
  char* w = (char*)a.workspace;
  z.w.share = (int*)w; w += 256;
  z.w.row_start = (int*)w; w += aligned((size_t)a.B * a.Hkv * sizeof(int));
  z.w.part_o = (float*)w; w += aligned(2 * (size_t)z.shares * z.G * a.D * sizeof(float));
  z.w.part_ml = (float*)w;
  if (a.dt == THRIFT_F16) launch<F16>(a, z, st);
  else launch<BF16>(a, z, st);
}

}  // namespace thrift
