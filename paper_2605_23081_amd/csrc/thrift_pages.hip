// Pages of the paged 16-bit cache: block tables and slots from the lengths on the device, return of pages, and the write of
// new tokens with the rotation of their queries and keys.
#include "thrift_paged.h"
#include "thrift_rotary.h"

namespace thrift {

namespace {

constexpr int kMapThreads = 256;
constexpr int kMapPerThread = kMapMaxSeqs / kMapThreads;

// Exclusive prefix sums of at most kMapMaxSeqs counts over the workgroup, saturating at `cap`: counts and cap are not negative and below
// 2^31, so that a sum of two fits 32 unsigned bits, and min(a + b, cap) is associative.  count(b) is asked for once;
// prefix[0 .. B] is written.
template <typename F>
__device__ __forceinline__ void prefix_sums(int B, uint32_t cap, uint32_t* prefix, uint32_t* wave_sums, F count) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (B + kMapThreads - 1) / kMapThreads;
  uint32_t mine[kMapPerThread], sum = 0;
#pragma unroll
  for (int i = 0; i < kMapPerThread; ++i) {
    const int b = tid * per + i;
    mine[i] = (i < per && b < B) ? min(count(b), cap) : 0u;
    sum = min(sum + mine[i], cap);
  }
  uint32_t incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t other = __shfl_up(incl, d);
    if (lane >= d) incl = min(incl + other, cap);
  }
  if (lane == 63) wave_sums[wave] = incl;
  __syncthreads();
  uint32_t before = __shfl_up(incl, 1);
  if (lane == 0) before = 0;
  uint32_t front = 0;
  for (int w = 0; w < wave; ++w) front = min(front + wave_sums[w], cap);
  before = min(before + front, cap);
#pragma unroll
  for (int i = 0; i < kMapPerThread; ++i) {
    const int b = tid * per + i;
    if (i < per && b < B) {
      prefix[b] = before;
      before = min(before + mine[i], cap);
      if (b == B - 1) prefix[B] = before;
    }
  }
  __syncthreads();
}

// The largest b in [0, B) with prefix[b] <= x, for x < prefix[B]: the sequence that owns item x (sequences without items own none).
__device__ __forceinline__ int owner(const uint32_t* prefix, int B, uint32_t x) {
  int lo = 0, hi = B;                                  // prefix[lo] <= x < prefix[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Every workgroup forms the prefix sums of all sequences for itself (a few microseconds of one CU each, side by side, instead of a launch
// in front) and then takes its share of the rows, of the new pages and of the sequences.
__global__ void __launch_bounds__(kMapThreads) page_map_kernel(PageMapArgs a) {
  __shared__ uint32_t row0[kMapMaxSeqs + 1];           // first row of every sequence
  __shared__ uint32_t page0[kMapMaxSeqs + 1];          // new pages of the sequences in front
  __shared__ uint32_t wave_sums[kMapThreads / 64];
  const int tid = threadIdx.x, P = a.page_size;
  const int shift = 31 - __builtin_clz(P);
  const uint32_t capacity = (uint32_t)a.max_pages << shift;
  const uint32_t avail = (uint32_t)min(a.free_capacity, max(0, a.free_count[0]));
  auto length = [&](int b) { return min(capacity, (uint32_t)max(0, a.seqlens[b])); };
  auto pages = [&](uint32_t tokens) { return (tokens + P - 1) >> shift; };
  prefix_sums(a.B, (uint32_t)a.rows, row0, wave_sums, [&](int b) { return (uint32_t)max(0, a.new_lens[b]); });
  auto fitting = [&](int b, uint32_t len) { return min(row0[b + 1] - row0[b], capacity - len); };
  auto wanted = [&](int b, uint32_t len) { return pages(len + fitting(b, len)) - pages(len); };
  prefix_sums(a.B, 0x7fffffffu, page0, wave_sums, [&](int b) { return wanted(b, length(b)); });
  // tokens of sequence b that have a place: page i of all new pages exists for i < avail
  auto granted = [&](int b) { return min(page0[b + 1], avail) - min(page0[b], avail); };
  auto placed = [&](int b, uint32_t len) { return min(fitting(b, len), ((pages(len) + granted(b)) << shift) - len); };
  // page i of all new pages
  auto taken = [&](uint32_t i) { return a.free_pages[avail - 1 - i]; };

  const uint32_t stride = gridDim.x * kMapThreads, first = blockIdx.x * kMapThreads + tid;
  for (uint32_t r = first; r < (uint32_t)a.rows; r += stride) {
    int slot = -1, position = 0;
    if (r < row0[a.B]) {
      const int b = owner(row0, a.B, r);
      const uint32_t len = length(b), i = r - row0[b], p = len + i, j = p >> shift, old = pages(len);
      position = (int)p;
      if (i < placed(b, len)) {
        // a page of this call comes from the stack: the table's entry is being written by another thread
        const int page = j < old ? a.table[(size_t)b * a.max_pages + j] : taken(page0[b] + (j - old));
        if (page >= 0 && page < a.n_pages) slot = (page << shift) + (int)(p & (P - 1));
      }
    }
    a.slots[r] = slot;
    a.positions[r] = position;
  }
  const uint32_t total = min(page0[a.B], avail);
  for (uint32_t i = first; i < total; i += stride) {
    const int b = owner(page0, a.B, i);
    a.table[(size_t)b * a.max_pages + pages(length(b)) + (i - page0[b])] = taken(i);
  }
  for (uint32_t b = first; b <= (uint32_t)a.B; b += stride) {
    a.starts[b] = (int)row0[b];
    if (b < (uint32_t)a.B) {
      const uint32_t len = length(b);
      a.seqlens_out[b] = (int)(len + placed(b, len));
    } else {
      a.free_count_out[0] = (int)(avail - total);
    }
  }
}

__global__ void __launch_bounds__(kMapThreads) page_release_kernel(PageReleaseArgs a) {
  __shared__ uint32_t page0[kMapMaxSeqs + 1];          // pages put back by the sequences in front
  __shared__ uint32_t wave_sums[kMapThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = a.page_size;
  const int shift = 31 - __builtin_clz(P);
  const uint32_t capacity = (uint32_t)a.max_pages << shift;
  const uint32_t have = (uint32_t)min(a.free_capacity, max(0, a.free_count[0]));
  auto held = [&](int b) { return (min(capacity, (uint32_t)max(0, a.seqlens[b])) + P - 1) >> shift; };
  auto valid = [&](int page) { return page >= 0 && page < a.n_pages; };
  // pages whose entries name none are not put back: a sequence's count is that of its good entries
  for (int b = wave; b < a.B; b += kMapThreads / 64) {
    uint32_t n = 0;
    if (a.drop[b] != 0)
      for (uint32_t j = lane; j < held(b); j += 64) n += valid(a.table[(size_t)b * a.max_pages + j]);
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if (lane == 0) page0[b] = n;
  }
  __syncthreads();
  prefix_sums(a.B, 0x7fffffffu, page0, wave_sums, [&](int b) { return page0[b]; });
  for (int b = wave; b < a.B; b += kMapThreads / 64) {
    const bool drop = a.drop[b] != 0;
    const uint32_t n = drop ? held(b) : 0u;
    uint32_t at = have + page0[b];
    for (uint32_t j0 = 0; j0 < n; j0 += 64) {
      const int page = j0 + lane < n ? a.table[(size_t)b * a.max_pages + j0 + lane] : -1;
      const unsigned long long good = __ballot(valid(page));
      const uint32_t to = at + __popcll(good & ((1ull << lane) - 1));
      if (valid(page) && to < (uint32_t)a.free_capacity) a.free_pages[to] = page;
      at += __popcll(good);
    }
    if (lane == 0) a.seqlens_out[b] = drop ? 0 : a.seqlens[b];
  }
  if (tid == 0) a.free_count_out[0] = (int)min((uint32_t)a.free_capacity, have + page0[a.B]);
}

constexpr int kAppendRowThreads = 128;

// One workgroup per row, a thread per pair or channel; cos and sin are formed once for all heads.
template <typename T>
__global__ void __launch_bounds__(kAppendRowThreads) paged_append_kernel(PagedAppendArgs a) {
  const long t = blockIdx.x;
  const int slot = a.slots[t];
  if (slot < 0 || slot >= a.n_pages * a.page_size) return;
  const size_t page = slot / a.page_size, in_page = slot % a.page_size;
  const size_t to = (page * a.Hkv * a.page_size + in_page) * a.D, head = (size_t)a.page_size * a.D;
  const int half = a.rot / 2, position = half ? a.positions[t] : 0;
  for (int i = threadIdx.x; i < half + (a.D - a.rot); i += kAppendRowThreads) {
    float c = 1.f, s = 0.f;
    if (i < half) turn(position, a.freqs[i], a.gain, c, s);
    auto turn_head = [&](const uint16_t* x, uint16_t* y) {
      if (i >= half) {
        y[half + i] = x[half + i];
        return;
      }
      const int i0 = a.layout == THRIFT_ROPE_HALF ? i : 2 * i, i1 = a.layout == THRIFT_ROPE_HALF ? i + half : 2 * i + 1;
      float y0, y1;
      rotate(T::to_float(x[i0]), T::to_float(x[i1]), c, s, y0, y1);
      y[i0] = T::from_float(y0);
      y[i1] = T::from_float(y1);
    };
    if (a.q != nullptr)
      for (int h = 0; h < a.Hq; ++h) turn_head(a.q + t * a.qt + h * a.qh, a.q_out + ((size_t)t * a.Hq + h) * a.D);
    for (int h = 0; h < a.Hkv; ++h) turn_head(a.k + t * a.kt + h * a.kh, a.k_pages + to + h * head);
  }
  for (int h = 0; h < a.Hkv; ++h)
    for (int i = threadIdx.x; i < a.D; i += kAppendRowThreads) a.v_pages[to + h * head + i] = a.v[t * a.vt + h * a.vh + i];
}

// The same in 16-byte chunks (thrift_rotary.h): the query heads of a row, then its key heads, then its value heads, which are copied.
template <typename T, int LAYOUT>
__global__ void __launch_bounds__(kHeadThreads) paged_append_items_kernel(PagedAppendArgs a, HeadShape z) {
  __shared__ float2 table[kAngles];
  const int tid = threadIdx.x, half = a.rot / 2;
  const int first = (int)(blockIdx.x / z.splits) * z.tokens, split = blockIdx.x % z.splits;
  const int item = tid % z.items, rest = tid / z.items, local = rest % z.tokens, group = rest / z.tokens;
  const int t = first + local, turned = a.Hq + a.Hkv, heads = turned + a.Hkv;
  const int slot = group < z.lanes && t < a.T ? a.slots[t] : -1;
  const bool busy = slot >= 0 && slot < a.n_pages * a.page_size;
  const Item<LAYOUT> it(item, a.D, a.rot);
  const uint16_t *q = a.q + t * a.qt, *k = a.k + t * a.kt, *v = a.v + t * a.vt;
  const int shift = 31 - __builtin_clz(a.page_size);
  const size_t head = (size_t)a.D << shift;                         // elements of a head in a page
  const size_t to = (size_t)(slot >> shift) * a.Hkv * head + (size_t)(slot & (a.page_size - 1)) * a.D;
  uint16_t* q_out = a.q_out + (size_t)t * a.Hq * a.D;
  const int step = z.lanes * z.splits;
  int h = busy ? split * z.lanes + group : heads;
  auto load = [&](int i, v4i (&c)[2]) {
    const uint16_t* p = i < a.Hq ? q + i * a.qh : i < turned ? k + (i - a.Hq) * a.kh : v + (i - turned) * a.vh;
    c[0] = *reinterpret_cast<const v4i*>(p + it.at[0]), c[1] = *reinterpret_cast<const v4i*>(p + it.at[1]);
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
    uint16_t* p = h < a.Hq ? q_out + (size_t)h * a.D : h < turned ? a.k_pages + to + (h - a.Hq) * head : a.v_pages + to + (h - turned) * head;
    const bool value = h >= turned;
    h += step;
    v4i next[2];
    if (h < heads) load(h, next);
    if (!value) turn_item<T, LAYOUT>(it, c, cs);
    *reinterpret_cast<v4i*>(p + it.at[0]) = c[0], *reinterpret_cast<v4i*>(p + it.at[1]) = c[1];
    c[0] = next[0], c[1] = next[1];
  }
}

template <typename T>
void launch_append(const PagedAppendArgs& a, hipStream_t st) {
  const uintptr_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.q_out | (uintptr_t)a.k_pages | (uintptr_t)a.v_pages;
  if (a.D % 16 != 0 || a.rot % 16 != 0 || at % 16 != 0 || ((a.q ? a.qt | a.qh : 0) | a.kt | a.kh | a.vt | a.vh) % 8 != 0) {
    paged_append_kernel<T><<<dim3((unsigned)a.T), dim3(kAppendRowThreads), 0, st>>>(a);
    return;
  }
  const HeadShape z = head_shape(a.T, a.Hq + 2 * a.Hkv, a.D, a.rot);
  const dim3 grid((unsigned)((a.T + z.tokens - 1) / z.tokens * z.splits)), block(kHeadThreads);
  if (a.layout == THRIFT_ROPE_HALF) paged_append_items_kernel<T, THRIFT_ROPE_HALF><<<grid, block, 0, st>>>(a, z);
  else paged_append_items_kernel<T, THRIFT_ROPE_INTERLEAVED><<<grid, block, 0, st>>>(a, z);
}

}  // namespace

void launch_page_map(const PageMapArgs& a, hipStream_t st) {
  const long items = a.rows > a.B ? a.rows : a.B;
  const long blocks = (items + kMapThreads - 1) / kMapThreads;
  page_map_kernel<<<dim3((unsigned)(blocks < 256 ? blocks : 256)), dim3(kMapThreads), 0, st>>>(a);
}

void launch_page_release(const PageReleaseArgs& a, hipStream_t st) {
  page_release_kernel<<<dim3(1), dim3(kMapThreads), 0, st>>>(a);
}

void launch_paged_append(const PagedAppendArgs& a, thrift_dtype dt, hipStream_t st) {
  if (dt == THRIFT_F16) launch_append<F16>(a, st);
  else launch_append<BF16>(a, st);
}

}  // namespace thrift
