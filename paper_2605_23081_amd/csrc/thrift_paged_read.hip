// Tokens of a paged cache as dense rows.
#include "thrift_e4m3.h"
#include "thrift_paged.h"

namespace thrift {

namespace {

constexpr int kReadThreads = 256;
constexpr long kMostGroups = 1L << 22;    // of a launch, which has less than 2^32 threads: workgroups of larger ones go on behind the last
// Above this many bytes of keys and values, written and read, the rows are written past the caches; the pages are read through them
constexpr long kStreamBytes = 128L << 20;

template <bool STREAM, typename V>
__device__ __forceinline__ void store(V* p, V x) {
  if (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}

// A number as T, at most T's largest; NaN stays
template <typename T>
__device__ __forceinline__ uint32_t within(float x) {
  const float most = T::to_float(T::kLargest);
  return T::from_float(x > most ? most : x < -most ? -most : x);
}
// Eight codes, in the first two registers, times a scale
template <typename T>
__device__ __forceinline__ v4i chunk_values(v4i codes, float scale) {
  v4i y;
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const float2 lo = e4m3_values<false>((uint32_t)codes[d], scale), hi = e4m3_values<true>((uint32_t)codes[d], scale);
    y[2 * d] = (int)(within<T>(lo.x) | (within<T>(lo.y) << 16)), y[2 * d + 1] = (int)(within<T>(hi.x) | (within<T>(hi.y) << 16));
  }
  return y;
}

// One element of K and of V per thread, for what cannot be moved in 16-byte chunks.
template <typename T, bool CODES>
__global__ void __launch_bounds__(kReadThreads) paged_read_kernel(PagedReadArgs a) {
  const size_t all = (size_t)a.B * a.Hkv * a.N * a.D;
  for (size_t i = (size_t)blockIdx.x * kReadThreads + threadIdx.x; i < all; i += (size_t)gridDim.x * kReadThreads) {
    const int c = (int)(i % a.D);
    const size_t row = i / a.D;
    const int n = (int)(row % a.N), h = (int)(row / a.N % a.Hkv), b = (int)(row / a.N / a.Hkv);
    const int len = min(a.max_pages * a.page_size, a.seqlens[b]);
    const long p = (long)n + (a.first ? max(0, a.first[b]) : 0);
    uint16_t k = 0, v = 0;
    if (p < len) {
      const int page = a.table[(size_t)b * a.max_pages + p / a.page_size];
      if (page >= 0 && page < a.n_pages) {
        const size_t at = ((size_t)page * a.Hkv + h) * a.page_size + p % a.page_size;
        if (CODES) {
          k = (uint16_t)within<T>(e4m3_values<false>(((const uint8_t*)a.k_pages)[at * a.D + c], scale_of(a.k_scales[at])).x);
          v = (uint16_t)within<T>(e4m3_values<false>(((const uint8_t*)a.v_pages)[at * a.D + c], scale_of(a.v_scales[at])).x);
        } else {
          k = ((const uint16_t*)a.k_pages)[at * a.D + c], v = ((const uint16_t*)a.v_pages)[at * a.D + c];
        }
      }
    }
    a.k_out[i] = k, a.v_out[i] = v;
  }
}

// In chunks of eight channels: a workgroup takes `rows` tokens of one head, about kItems chunks of K and as many of V.  Bound by memory: 30720 tokens of
// 8 heads of 128 channels, 252 MB, in 45 us (5.5 TB/s), 5 x 750-3001 of 16 heads from codes in 24 (6.6), 1000 tokens of 8 heads in 3.6 in a graph.  Two chunks of each
// per thread; one takes 69 instead of 67 us for 60000 tokens from codes, four 4.5 for the 1000 tokens.  Rows through the caches: 52 instead of 45 for the first; codes past them:
// 33 instead of 26 for the second, whose pages the cache in front of the memory still holds.
constexpr int kAhead = 2, kItems = kReadThreads * kAhead;
struct ReadShape {
  int chunks, rows, parts;                  // of a token's head; of a workgroup; workgroups per head
  uint32_t groups;                          // workgroups' shares in all
  uint32_t magic;                           // 2^32 / chunks, rounded up: i / chunks is the high word of their product for i < 2^16 (0 for one chunk)
};

template <typename T, bool CODES, bool STREAM>
__global__ void __launch_bounds__(kReadThreads) paged_read_chunks_kernel(PagedReadArgs a, ReadShape z) {
  const int shift = 31 - __builtin_clz(a.page_size);
  // Once but for more than kMostGroups; below 2^31 of them, so that the sum stays below 2^32
  for (uint32_t group = blockIdx.x; group < z.groups; group += gridDim.x) {
    const int head = group / z.parts, n0 = (group - head * z.parts) * z.rows, b = head / a.Hkv, h = head - b * a.Hkv;
    const int len = min(a.max_pages << shift, a.seqlens[b]), first = a.first ? max(0, a.first[b]) : 0;
    const int count = min(z.rows, a.N - n0) * z.chunks;
    const int32_t* table = a.table + (size_t)b * a.max_pages;
    v4i k[kAhead], v[kAhead];
    uint32_t ks[kAhead], vs[kAhead];
    size_t at[kAhead];
    bool there[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = min(threadIdx.x + u * kReadThreads, (unsigned)count - 1);
      const int row = z.magic ? (int)__umulhi((uint32_t)i, z.magic) : i, c = i - row * z.chunks;
      const long p = (long)first + n0 + row;
      there[u] = p < len;
      const int page = there[u] ? table[p >> shift] : -1;
      there[u] = page >= 0 && page < a.n_pages;
      const size_t from = (((size_t)page * a.Hkv + h) << shift) + (p & (a.page_size - 1));
      at[u] = ((size_t)head * a.N + n0 + row) * a.D + 8 * c;
      k[u] = v[u] = v4i{0, 0, 0, 0};
      ks[u] = vs[u] = 0;
      if (there[u]) {
        if (CODES) {
          const v2i x = *(const v2i*)((const uint8_t*)a.k_pages + from * a.D + 8 * c), y = *(const v2i*)((const uint8_t*)a.v_pages + from * a.D + 8 * c);
          k[u] = v4i{x[0], x[1], 0, 0}, v[u] = v4i{y[0], y[1], 0, 0};
          ks[u] = a.k_scales[from], vs[u] = a.v_scales[from];
        } else {
          k[u] = *(const v4i*)((const uint16_t*)a.k_pages + from * a.D + 8 * c);
          v[u] = *(const v4i*)((const uint16_t*)a.v_pages + from * a.D + 8 * c);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if ((int)threadIdx.x + u * kReadThreads >= count) break;
      if (CODES) k[u] = chunk_values<T>(k[u], scale_of(ks[u])), v[u] = chunk_values<T>(v[u], scale_of(vs[u]));
      store<STREAM>((v4i*)(a.k_out + at[u]), k[u]);
      store<STREAM>((v4i*)(a.v_out + at[u]), v[u]);
    }
  }
}

template <typename T, bool CODES>
void launch(const PagedReadArgs& a, hipStream_t st) {
  const uintptr_t out = (uintptr_t)a.k_out | (uintptr_t)a.v_out, in = (uintptr_t)a.k_pages | (uintptr_t)a.v_pages;
  if (a.D % 8 != 0 || out % 16 != 0 || in % (CODES ? 8 : 16) != 0) {
    const long groups = ((long)a.B * a.Hkv * a.N * a.D + kReadThreads - 1) / kReadThreads;
    paged_read_kernel<T, CODES><<<dim3((unsigned)(groups < kMostGroups ? groups : kMostGroups)), dim3(kReadThreads), 0, st>>>(a);
    return;
  }
  ReadShape z;
  z.chunks = a.D / 8;
  z.rows = kItems / z.chunks;
  if (z.rows > a.N) z.rows = a.N;
  z.parts = (int)(((long)a.N + z.rows - 1) / z.rows);
  z.magic = z.chunks == 1 ? 0u : (uint32_t)((0x100000000ull + z.chunks - 1) / z.chunks);
  const long groups = (long)a.B * a.Hkv * z.parts;          // at most B * Hkv * N
  z.groups = (uint32_t)groups;
  const dim3 grid((unsigned)(groups < kMostGroups ? groups : kMostGroups)), block(kReadThreads);
  if ((long)a.B * a.Hkv * a.N * a.D * 8 > kStreamBytes) paged_read_chunks_kernel<T, CODES, true><<<grid, block, 0, st>>>(a, z);
  else paged_read_chunks_kernel<T, CODES, false><<<grid, block, 0, st>>>(a, z);
}

}  // namespace

void launch_paged_read(const PagedReadArgs& a, thrift_dtype dt, hipStream_t st) {
  if (a.k_scales == nullptr) launch<F16, false>(a, st);
  else if (dt == THRIFT_F16) launch<F16, true>(a, st);
  else launch<BF16, true>(a, st);
}

}  // namespace thrift
