// Pages of the paged 16-bit cache: block tables and slots from the lengths on the device, return of pages, and the write of
// new tokens with the rotation of their queries and keys.
//
// The map is bound by latency: 5.5 us of kernel for 256 sequences with a token each, 5.6 for 64 with 262144 rows (2 MB), 6.0-6.3 with the call.  So is the
// release: 8.7 us of kernel for 12 of 256 sequences of up to 1024 pages, 14.6-15 with the call, whose host part passes through ctypes.  The append is
// bound by memory: it reads and writes every element once (counters), 8192 rows of 64/8 heads in 72 us (4.7 TB/s), 32768 of 32/8 in 157
// (5.1; a copy: 6.5); a decode step's rows take the launch (3.7 us of kernel, 4.5 with the call).
#include "thrift_paged.h"
#include "thrift_rotary.h"

namespace thrift {

namespace {

constexpr int kMapThreads = 256;
constexpr int kMapRows = 4;                            // neighbouring rows of a thread

// Exclusive prefix sums of two counts per sequence over the workgroup, at most kMapMaxSeqs sequences.  The first saturates at `cap`: counts and
// cap are below 2^31, so that a sum of two fits 32 unsigned bits, and min(a + b, cap) is associative.  The second may not pass
// 2^31 (saturated there as well).  PER: sequences of a thread at most.  count(b) is asked for once; x[0 .. B] and y[0 .. B] are written.
template <int PER, typename F>
__device__ __forceinline__ void prefix_sums(int B, uint32_t cap, uint32_t* x, uint32_t* y, uint2* wave_sums, F count) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = PER == 1 ? 1 : (B + kMapThreads - 1) / kMapThreads;
  auto add = [&](uint2 a, uint2 b) { return make_uint2(min(a.x + b.x, cap), min(a.y + b.y, 0x7fffffffu)); };
  uint2 mine[PER], sum = make_uint2(0, 0);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = tid * per + i;
    mine[i] = i < per && b < B ? count(b) : make_uint2(0, 0);
    mine[i].x = min(mine[i].x, cap);
    sum = add(sum, mine[i]);
  }
  uint2 incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint2 other = make_uint2(__shfl_up(incl.x, d), __shfl_up(incl.y, d));
    if (lane >= d) incl = add(incl, other);
  }
  if (lane == 63) wave_sums[wave] = incl;
  __syncthreads();
  uint2 before = make_uint2(__shfl_up(incl.x, 1), __shfl_up(incl.y, 1));
  if (lane == 0) before = make_uint2(0, 0);
  for (int w = 0; w < wave; ++w) before = add(before, wave_sums[w]);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = tid * per + i;
    if (i < per && b < B) {
      x[b] = before.x, y[b] = before.y;
      before = add(before, mine[i]);
      if (b == B - 1) x[B] = before.x, y[B] = before.y;
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

// Every workgroup forms the prefix sums of all sequences for itself (side by side instead of a launch in front) and then takes its
// share of the rows, of the new pages and of the sequences.  The pages are counted as if no row were cut off; where rows are, the
// first sequence they are cut off from ends the count (`last_page`).  Bounded by its chain of latencies: lengths, sums, the
// search for a row's sequence, its page.
template <int PER>
__global__ void __launch_bounds__(kMapThreads) page_map_kernel(PageMapArgs a) {
  __shared__ uint32_t row0[kMapMaxSeqs + 1];           // first row of every sequence
  __shared__ uint32_t page0[kMapMaxSeqs + 1];          // new pages of the sequences in front
  __shared__ uint32_t lens[kMapMaxSeqs];
  __shared__ uint2 wave_sums[kMapThreads / 64];
  __shared__ uint32_t cut_page;
  const int tid = threadIdx.x, P = a.page_size;
  const int shift = 31 - __builtin_clz(P);
  const uint32_t capacity = (uint32_t)a.max_pages << shift, rows = (uint32_t)a.rows;
  const uint32_t avail = (uint32_t)min(a.free_capacity, max(0, a.free_count[0]));
  auto pages = [&](uint32_t tokens) { return (tokens + P - 1) >> shift; };
  if (tid == 0) cut_page = 0xffffffffu;
  prefix_sums<PER>(a.B, rows, row0, page0, wave_sums, [&](int b) {
    const uint32_t len = min(capacity, (uint32_t)max(0, a.seqlens[b])), fresh = (uint32_t)max(0, a.new_lens[b]);
    lens[b] = len;
    return make_uint2(fresh, pages(len + min(fresh, capacity - len)) - pages(len));
  });
  auto fitting = [&](int b) { return min(row0[b + 1] - row0[b], capacity - lens[b]); };
  if (row0[a.B] == rows) {                             // rows may have been cut off
    for (int b = tid; b < a.B; b += kMapThreads)
      if (row0[b] < rows && row0[b + 1] == rows) cut_page = page0[b] + pages(lens[b] + fitting(b)) - pages(lens[b]);
    __syncthreads();
  }
  const uint32_t last_page = min(cut_page, avail);     // page i of all new pages exists for i < last_page
  // tokens of sequence b that have a place
  auto placed = [&](int b) {
    const uint32_t granted = min(page0[b + 1], last_page) - min(page0[b], last_page);
    return min(fitting(b), ((pages(lens[b]) + granted) << shift) - lens[b]);
  };
  // page i of all new pages
  auto taken = [&](uint32_t i) { return a.free_pages[avail - 1 - i]; };

  const uint32_t threads = gridDim.x * kMapThreads, first = blockIdx.x * kMapThreads + tid;
  const bool chunks = (((uintptr_t)a.slots | (uintptr_t)a.positions) & 15) == 0;
  for (uint32_t r0 = first * kMapRows; r0 < rows; r0 += threads * kMapRows) {
    int slot[kMapRows], position[kMapRows];
    int b = r0 < row0[a.B] ? owner(row0, a.B, r0) : a.B;
    uint32_t have = b < a.B ? placed(b) : 0;
#pragma unroll
    for (int e = 0; e < kMapRows; ++e) {
      const uint32_t r = r0 + e;
      slot[e] = -1, position[e] = 0;
      if (b < a.B && r >= row0[b + 1]) {
        do ++b; while (b < a.B && r >= row0[b + 1]);
        have = b < a.B ? placed(b) : 0;
      }
      if (b < a.B) {
        const uint32_t len = lens[b], i = r - row0[b], p = len + i, j = p >> shift, old = pages(len);
        position[e] = (int)p;
        if (i < have) {
          // a page of this call comes from the stack: the table's entry is being written by another thread
          const int page = j < old ? a.table[(size_t)b * a.max_pages + j] : taken(page0[b] + (j - old));
          if (page >= 0 && page < a.n_pages) slot[e] = (page << shift) + (int)(p & (P - 1));
        }
      }
    }
    if (chunks && r0 + kMapRows <= rows) {
      *reinterpret_cast<int4*>(a.slots + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      *reinterpret_cast<int4*>(a.positions + r0) = make_int4(position[0], position[1], position[2], position[3]);
    } else {
#pragma unroll
      for (int e = 0; e < kMapRows; ++e)
        if (r0 + e < rows) a.slots[r0 + e] = slot[e], a.positions[r0 + e] = position[e];
    }
  }
  const uint32_t total = min(page0[a.B], last_page);
  for (uint32_t i = first; i < total; i += threads) {
    const int b = owner(page0, a.B, i);
    a.table[(size_t)b * a.max_pages + pages(lens[b]) + (i - page0[b])] = taken(i);
  }
  for (uint32_t b = first; b <= (uint32_t)a.B; b += threads) {
    a.starts[b] = (int)row0[b];
    if (b < (uint32_t)a.B) a.seqlens_out[b] = (int)(lens[b] + placed(b));
    else a.free_count_out[0] = (int)(avail - total);
  }
}

constexpr int kReleaseThreads = 1024;

// One workgroup: most sequences stay, so those that end are listed first, in order; a wavefront then takes every 16th of them, once to
// count its pages and once to put them on the stack behind those of the sequences in front.
__global__ void __launch_bounds__(kReleaseThreads) page_release_kernel(PageReleaseArgs a) {
  constexpr int kWaves = kReleaseThreads / 64;
  __shared__ int ending[kMapMaxSeqs];
  __shared__ uint32_t to_stack[kMapMaxSeqs];           // pages that go back, then their sums in front
  __shared__ uint32_t wave_sums[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = a.page_size;
  const int shift = 31 - __builtin_clz(P);
  const uint32_t capacity = (uint32_t)a.max_pages << shift;
  const uint32_t have = (uint32_t)min(a.free_capacity, max(0, a.free_count[0]));
  const unsigned long long below = (1ull << lane) - 1;
  // 16 wavefronts' counts to the sum in front of this one's, and of all
  auto sums = [&](uint32_t mine, uint32_t& front, uint32_t& all) {
    __syncthreads();
    if (lane == 0) wave_sums[wave] = mine;
    __syncthreads();
    front = all = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) front += wave_sums[w];
      all += wave_sums[w];
    }
  };
  uint32_t n = 0, front, all;
  for (int b0 = 0; b0 < a.B; b0 += kReleaseThreads) {
    const int b = b0 + tid;
    const bool drop = b < a.B && a.drop[b] != 0;
    if (b < a.B) a.seqlens_out[b] = drop ? 0 : a.seqlens[b];
    const unsigned long long who = __ballot(drop);
    sums((uint32_t)__popcll(who), front, all);
    if (drop) ending[n + front + __popcll(who & below)] = b;
    n += all;
  }
  __syncthreads();
  auto held = [&](int b) { return (min(capacity, (uint32_t)max(0, a.seqlens[b])) + P - 1) >> shift; };
  // entries that name no page are not put back
  auto page_of = [&](int b, uint32_t j, uint32_t pages) {
    const int page = j < pages ? a.table[(size_t)b * a.max_pages + j] : -1;
    return page < a.n_pages ? page : -1;
  };
  for (uint32_t i = wave; i < n; i += kWaves) {
    const int b = ending[i];
    const uint32_t pages = held(b);
    uint32_t good = 0;
    for (uint32_t j0 = 0; j0 < pages; j0 += 64) good += __popcll(__ballot(page_of(b, j0 + lane, pages) >= 0));
    if (lane == 0) to_stack[i] = good;
  }
  __syncthreads();
  uint32_t total = 0;
  for (uint32_t i0 = 0; i0 < n; i0 += kReleaseThreads) {
    const uint32_t i = i0 + tid, mine = i < n ? to_stack[i] : 0u;
    uint32_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t other = __shfl_up(incl, d);
      if (lane >= d) incl += other;
    }
    sums(__shfl(incl, 63), front, all);
    if (i < n) to_stack[i] = total + front + incl - mine;
    total += all;
  }
  __syncthreads();
  for (uint32_t i = wave; i < n; i += kWaves) {
    const int b = ending[i];
    const uint32_t pages = held(b);
    uint32_t at = have + to_stack[i];
    for (uint32_t j0 = 0; j0 < pages; j0 += 64) {
      const int page = page_of(b, j0 + lane, pages);
      const unsigned long long good = __ballot(page >= 0);
      const uint32_t to = at + __popcll(good & below);
      if (page >= 0 && to < (uint32_t)a.free_capacity) a.free_pages[to] = page;
      at += __popcll(good);
    }
  }
  if (tid == 0) a.free_count_out[0] = (int)min((uint32_t)a.free_capacity, have + total);
}

constexpr int kAppendRowThreads = 128;

// One workgroup per row, a thread per pair or channel; cos and sin are formed once for all heads.  For what cannot be moved in 16-byte
// chunks; where it can, the kernel below is faster (8192 rows of 64/8 heads: 134 us here, 78 there with cached stores as well; 208 here with 20 of
// 128 channels turned).
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
template <typename T, int LAYOUT, bool STREAM>
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
    uint16_t* p = h < a.Hq ? q_out + (size_t)h * a.D : h < turned ? a.k_pages + to + (h - a.Hq) * head : a.v_pages + to + (h - turned) * head;
    const bool value = h >= turned;
    h += step;
    v4i next[2];
    if (h < heads) load(h, next);
    if (!value) turn_item<T, LAYOUT>(it, c, cs);
    chunk_to<STREAM>(p + it.at[0], c[0]), chunk_to<STREAM>(p + it.at[1], c[1]);
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
  // Written past the caches where a store fills lines: 78.4 -> 71.8 us for 8192 rows of 64/8 heads of 128 channels, 167.7 -> 157.0 for 32768 of 32/8;
  // with 64 channels turned by halves 78.1 cached, 82.4 past the caches, with none 46.1 and 54.0 (8192 rows of 32/8)
  const bool stream = fills_lines(a.D, a.rot, a.layout);
#define THRIFT_APPEND(L_)                                                                    \
  if (stream) paged_append_items_kernel<T, L_, true><<<grid, block, 0, st>>>(a, z);          \
  else paged_append_items_kernel<T, L_, false><<<grid, block, 0, st>>>(a, z)
  if (a.layout == THRIFT_ROPE_HALF) { THRIFT_APPEND(THRIFT_ROPE_HALF); }
  else { THRIFT_APPEND(THRIFT_ROPE_INTERLEAVED); }
#undef THRIFT_APPEND
}

}  // namespace

void launch_page_map(const PageMapArgs& a, hipStream_t st) {
  const long items = a.rows / kMapRows > a.B ? a.rows / kMapRows : a.B;
  const long blocks = (items + kMapThreads - 1) / kMapThreads;
  const dim3 grid((unsigned)(blocks < 256 ? blocks : 256)), block(kMapThreads);
  if (a.B <= kMapThreads) page_map_kernel<1><<<grid, block, 0, st>>>(a);
  else page_map_kernel<kMapMaxSeqs / kMapThreads><<<grid, block, 0, st>>>(a);
}

void launch_page_release(const PageReleaseArgs& a, hipStream_t st) {
  page_release_kernel<<<dim3(1), dim3(kReleaseThreads), 0, st>>>(a);
}

void launch_paged_append(const PagedAppendArgs& a, thrift_dtype dt, hipStream_t st) {
  if (dt == THRIFT_F16) launch_append<F16>(a, st);
  else launch_append<BF16>(a, st);
}

}  // namespace thrift
