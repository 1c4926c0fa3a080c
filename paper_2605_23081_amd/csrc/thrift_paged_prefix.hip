// Attention of one new token per sequence where sequences start with the same pages.
//
// Three launches.  The first takes the common tokens: a group's members times the G query heads of a KV head are the rows of a product with
// the group's keys, and with P and its values, so that these are read once per tile of rows instead of once per sequence.  The second
// walks every sequence's own tokens (thrift_paged_walk.h).  The third joins what the two left of every row, and writes the results.
//
// Common tokens.  A tile is at most kTile rows of one group and KV head, a wavefront has 32 of them in the columns of 32 x 32 matrix
// tiles and walks blocks of 64 keys:
//   S = K Q^T      64 keys x 32 rows;  r: a reference of the row, P = 2^(S c - r) <= 2^15
//   O^T += V^T P^T channels x 32 rows; a lane's part of S is its operand P, without passing through LDS or other lanes
// K and V of a block lie in LDS for all wavefronts, V is transposed by the reads.  They come by LDS DMA, three blocks ahead.  With at most half a tile of rows, wavefronts take half a block's keys each, two to a row.
//   8-bit pages come through registers, two blocks ahead, and are converted on their way to LDS, once for all wavefronts: values and, for bf16 queries, keys times their scales, which bf16
// holds exactly; for fp16 queries keys without, and the scales, in LDS too, are factors of the scores.
//   P is rounded to 16 bits once, unlike in the walk of own tokens: two pieces would be half as many matrix instructions again, which
// bound this kernel for large groups.  Sums are those of the unrounded P.
//   The reference is the row's largest score so far where that has grown by more than fp16 (or 8 binades, bf16) would hold, so that O is rarely
// multiplied; for fp16 it lies 7 binades lower, which keeps P normal down to 2^-21 of the largest.  Scores from 2^20 on are rounded before r is
// taken off, as in the walk: a fused difference would be off by binades.
//   The blocks of all tiles are counted through on the GPU and cut into equal shares, one per workgroup and CU, a full tile's at twice the
// price.  The part of a tile that has its first block is written to the rows' places, any other is the first of its share and is
// written to the share's slot.
#include "thrift_paged_walk.h"
#include "thrift_tile.h"

namespace thrift {

namespace {

constexpr int kBlock = 64;                             // keys
constexpr int kPrefixShares = kCus;
// Wavefronts of a workgroup.  256 channels: four, with all registers that two have otherwise.
constexpr int prefix_waves(int D) { return D == 256 ? 4 : 8; }
constexpr int tile_rows(int D) { return 32 * prefix_waves(D); }

struct Prefix {
  float *home_o, *home_ml;                             // [B*Hq][D], [B*Hq][2]: parts with a tile's first block
  int4* home_span;                                     // [B*Hq]: first share with more of the row's tile, how many, the row in the tile
  float *slot_o, *slot_ml;                             // [kPrefixShares][tile_rows][D], [..][2]
};

struct PrefixLaunch {
  Prefix p;
  Launch own;
};

// Two numbers rounded to 16 bits, the first in the lower half
template <typename T>
__device__ __forceinline__ uint32_t pack16(float x, float y) {
  if constexpr (std::is_same_v<T, F16>) return __builtin_bit_cast(uint32_t, v2h{(_Float16)x, (_Float16)y});
  else return __builtin_bit_cast(uint32_t, v2bf{(__bf16)x, (__bf16)y});
}

template <typename T> struct Reference;                // how far below the largest score the reference lies, and how far one may pass it
template <> struct Reference<F16> { static constexpr float kBelow = 7.f, kMost = 15.f; };
template <> struct Reference<BF16> { static constexpr float kBelow = 0.f, kMost = 8.f; };

constexpr int kMaxSeqs = kMapMaxSeqs, kMaxGroups = kMapMaxSeqs;

template <typename T, int D, bool C8>
struct Tiles {
  using P = std::conditional_t<C8, BF16, T>;
  static constexpr bool kScaled = C8 && std::is_same_v<T, F16>;             // keys lie in LDS without their scales
  static constexpr int kWaves = prefix_waves(D), kThreads = 64 * kWaves, kTile = tile_rows(D);
  static constexpr int kRow = 2 * D;                                        // bytes of a row in LDS
  static constexpr int kSide = kBlock * kRow, kSlot = 2 * kSide;
  static constexpr int kRing = C8 || D == 256 ? 2 : 4;                      // blocks in LDS
  static constexpr int kChunks = kBlock * D / 8 / kThreads;                 // 16-byte chunks of K, and of V, of a thread
  static constexpr int kRowsOf = 512 / D;                                   // rows of a wavefront's chunk
  static_assert(kChunks * kWaves * kRowsOf == kBlock, "");

  struct Shared {
    char stage[kRing][kSlot];
    float scales[kScaled ? kRing : 1][kScaled ? kBlock : 1];
    float ml[kWaves / 2][2][64];
    int count[kMaxGroups];                             // members of every group
    uint16_t group[kMaxSeqs];                          // of every sequence; 0xffff: none
    int list[kTile + 1];                               // members that have rows in the tile
    long sums[kWaves];
    int waves[kWaves];
    long start_base;
    int start_group;
  };

  // A block of codes on its way
  struct Block {
    v2i k[kChunks], v[kChunks];
    uint32_t ks[kChunks], vs[kChunks];
  };
};

__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// One tile's rows in a wavefront: 32 of them
template <typename T, int D, bool C8, int PARTS>
struct Rows {
  using L = Tiles<T, D, C8>;
  using P = typename L::P;
  static constexpr int NT = 2 / PARTS;                 // 32-key halves of a block
  v8s q[D / 16];
  v16f s[NT];                                          // scores of a block,
  v4i p[NT][2];                                        // and P
  v16f o[D / 32];
  float r, l;                                          // reference, this lane's part of the sum
  bool large;                                          // of the wavefront: some reference from 2^20 on

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][i] = 0.f;
    r = -__FLT_MAX__, l = 0.f, large = false;
  }

  // The products with a block in LDS; part: which half of its keys, of PARTS.  Operands are asked for a phase ahead of the products that take them: fences
  // keep the compiler from putting every read in front of its use.
  __device__ __forceinline__ void scores(const char* slot, int part) {
    const int lane = threadIdx.x & 63, half = lane >> 5, row = lane & 31;
    // Chunk x of a K row lies at x ^ (row & 7): eight neighbouring rows at one chunk fill all banks
    const char* k0 = slot + (32 * part + row) * L::kRow;
    const uint32_t swizzled = 16u * (half ^ (row & 7));
    constexpr int kPiece = D / 16 < 8 ? D / 16 : 8, kPieces = NT * D / 16 / kPiece;       // K operands in flight, and of a block
    v8s k[2][kPiece];
    auto read_k = [&](int i) {
#pragma unroll
      for (int x = 0; x < kPiece; ++x) {
        const int t = i * kPiece / (D / 16), e = i * kPiece % (D / 16) + x;
        k[i & 1][x] = *reinterpret_cast<const v8s*>(k0 + 32 * t * L::kRow + ((swizzled ^ (32u * (e & 3))) + 128u * (e >> 2)));
      }
    };
    read_k(0);
    fence();
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      if (i + 1 < kPieces) {
        read_k(i + 1);
        fence();
      }
#pragma unroll
      for (int x = 0; x < kPiece; ++x) {
        const int t = i * kPiece / (D / 16), e = i * kPiece % (D / 16) + x;
        if (e == 0) {
#pragma unroll
          for (int j = 0; j < 16; ++j) s[t][j] = 0.f;
        }
        s[t] = T::mfma(k[i & 1][x], q[e], s[t]);
      }
    }
  }

  // Scores to P, with the reference and the sum; `valid` keys of the block are there
  __device__ __forceinline__ void soften(const float* scales, int part, int valid, float c) {
    const int half = (threadIdx.x & 63) >> 5;
    // register i of half t: key 32 t + 8 (i / 4) + 4 half + i % 4
    if constexpr (L::kScaled) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const v4f f = *reinterpret_cast<const v4f*>(scales + 32 * (part + t) + 2 * i + 4 * half);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][i + e] *= f[e];
        }
    }
    if (valid < kBlock) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * (part + t) + 8 * (i >> 2) + 4 * half + (i & 3) >= valid) s[t][i] = -__builtin_inff();
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
    top = both_halves_max(top) * c;
    if (__ballot(top - r > Reference<P>::kMost)) {
      // a score past 2^20 and its difference to a reference are no longer exact in one fused step
      const bool far = fabsf(top) >= 0x1p20f && fabsf(top) < __builtin_inff();
      const float next = top > r ? (far ? top : top - Reference<P>::kBelow) : r;
      const float raised = fmaxf(next, r), keep = fast_exp2(r - raised);
      r = raised, l *= keep;
#pragma unroll
      for (int n = 0; n < D / 32; ++n) o[n] *= keep;
      large = __ballot(fabsf(r) >= 0x1p20f && r > -__FLT_MAX__) != 0;
    }
    float f = c, off = r;
    if (large) {
#pragma clang fp contract(off)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = s[t][i] * c;
          s[t][i] = x - r;
        }
      f = 1.f, off = 0.f;
    }
    float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float x = fast_exp2(__builtin_fmaf(s[t][i], f, -off)), y = fast_exp2(__builtin_fmaf(s[t][i + 1], f, -off));
        sums[i & 2] += x, sums[(i & 2) + 1] += y;
        p[t][i >> 3][(i & 7) >> 1] = (int)pack16<P>(x, y);
      }
    l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
  }

  __device__ __forceinline__ void multiply(const char* slot, int part) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    // V operands: slots 8 half + e of step u of half t are keys 32 t + 16 u + 8 (e / 4) + 4 half + e % 4, as P's registers are.  A group of 16 lanes
    // reads four keys x 16 channels and gets four keys of a channel per lane
    const int i16 = lane & 15, g = (lane >> 4) & 1, key = 4 * half + (i16 >> 2);
    typedef v4s __attribute__((address_space(3))) * lds_v4s_ptr;
    const char* v0 = slot + L::kSide + (32 * part + key) * L::kRow;
    const uint32_t at = (32u * g + 8u * (i16 & 3)) ^ v_swizzle(key);
    constexpr int kWide = D / 32 < 4 ? D / 32 : 4, kSteps = 2 * NT * (D / 32) / kWide;     // channel tiles of a phase; phases
    v4s v[2][kWide][2];
    auto read_v = [&](int i) {
#pragma unroll
      for (int x = 0; x < kWide; ++x) {
        const int tu = i * kWide / (D / 32), n = i * kWide % (D / 32) + x;
        const char* from = v0 + 16 * tu * L::kRow + ((at ^ (64u * (n & 3))) + 256u * (n >> 2));
        v[i & 1][x][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(from));
        v[i & 1][x][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(from + 8 * L::kRow));
      }
    };
    read_v(0);
    fence();
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i + 1 < kSteps) {
        read_v(i + 1);
        fence();
      }
#pragma unroll
      for (int x = 0; x < kWide; ++x) {
        const int tu = i * kWide / (D / 32), n = i * kWide % (D / 32) + x;
        o[n] = P::mfma(__builtin_shufflevector(v[i & 1][x][0], v[i & 1][x][1], 0, 1, 2, 3, 4, 5, 6, 7), __builtin_bit_cast(v8s, p[tu >> 1][tu & 1]), o[n]);
      }
      fence();
    }
  }

  // Bytes that a V row's offsets are swizzled by: four neighbouring rows at one 64-byte piece fill all banks
  static __device__ __forceinline__ uint32_t v_swizzle(int row) { return D == 64 ? 64u * ((row >> 1) & 1) : 64u * (row & 3); }
};

template <typename T, int D, bool C8>
__global__ void __launch_bounds__(64 * prefix_waves(D)) prefix_kernel(PagedDecodeArgs a, PrefixLaunch z) {
  using L = Tiles<T, D, C8>;
  __shared__ __align__(16) typename L::Shared sh;
  constexpr int kWaves = L::kWaves, kThreads = L::kThreads, kTile = L::kTile;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = z.own.G, shift = z.own.shift, capacity = a.max_pages << shift, n_groups = z.own.groups.n;

  // ---- members of the groups, and this workgroup's share ----
  for (int g = tid; g < n_groups; g += kThreads) sh.count[g] = 0;
  __syncthreads();
  for (int b = tid; b < a.B; b += kThreads) {
    const int n = common_tokens(z.own.groups, capacity, shift, b, min(capacity, max(0, a.seqlens[b])));
    const int g = n > 0 ? z.own.groups.of[b] : 0xffff;
    sh.group[b] = (uint16_t)g;
    if (n > 0) atomicAdd(&sh.count[g], 1);
  }
  __syncthreads();
  auto tokens_of = [&](int g) { return min(capacity, max(0, z.own.groups.lens[g])) >> shift << shift; };
  auto blocks_of = [&](int tokens) { return (int)(((unsigned)tokens + kBlock - 1) / kBlock); };
  auto weight_of = [&](int rows) { return rows == 0 ? 0 : rows > kTile / 2 ? 2 : 1; };      // of a tile's block
  auto price = [&](int g) -> long {
    const int n = sh.count[g];
    if (n == 0) return 0;
    const int rows = n * G, full = rows / kTile;
    return (long)a.Hkv * (2 * full + weight_of(rows - full * kTile)) * blocks_of(tokens_of(g));
  };
  const int per = (n_groups + kThreads - 1) / kThreads;
  long sum = 0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < n_groups) sum += price(tid * per + i);
  long incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long other = __shfl_up(incl, d);
    if (lane >= d) incl += other;
  }
  if (lane == 63) sh.sums[wave] = incl;
  __syncthreads();
  long base = incl - sum, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) base += sh.sums[w];
    total += sh.sums[w];
  }
  const long each = (total + 2 * kPrefixShares - 1) / (2 * kPrefixShares) * 2;              // even: every share inside a tile has a block of it
  long u = (long)blockIdx.x * each;
  if (u >= total) return;                              // the whole workgroup
  const long u_end = min(total, u + each);
  if (base <= u && u < base + sum) {
    int g = tid * per;
    for (long p = price(g); base + p <= u; p = price(g)) base += p, ++g;
    sh.start_group = g, sh.start_base = base;
  }
  __syncthreads();
  int g = __builtin_amdgcn_readfirstlane(sh.start_group);
  long g_base = sh.start_base;
  int listed_group = -1, listed_tile = -1;

  while (true) {
    // ---- the piece of a tile that begins at u ----
    const int members = sh.count[g], tokens = __builtin_amdgcn_readfirstlane(tokens_of(g)), blocks = blocks_of(tokens), rows = members * G, full = rows / kTile;
    const long tile_price = 2L * a.Hkv * blocks;
    const long into = u - g_base;
    const int tile = (int)min((long)full, into / tile_price), weight = tile < full ? 2 : weight_of(rows - full * kTile);
    const long in_tile = into - tile * tile_price;
    const int hk = (int)(in_tile / ((long)weight * blocks));
    const long unit = g_base + tile * tile_price + (long)hk * weight * blocks;            // where the blocks of this KV head begin
    const long end = min(u_end, unit + (long)weight * blocks);
    const int t0 = (int)((u - unit + weight - 1) / weight), t1 = (int)((end - unit + weight - 1) / weight);
    const int row0 = tile * kTile, tile_rows = min(kTile, rows - row0);

    // ---- the tile's members, in the order of the batch ----
    if (listed_group != g || listed_tile != tile) {
      const int m0 = row0 / G, m1 = (row0 + tile_rows - 1) / G;
      const int chunk = (a.B + kThreads - 1) / kThreads * 64, from = wave * chunk, to = min(a.B, from + chunk);
      int n = 0;
      for (int b0 = from; b0 < to; b0 += 64) n += __popcll(__ballot(b0 + lane < to && sh.group[b0 + lane] == g));
      __syncthreads();                                 // nobody reads the list in front
      if (lane == 0) sh.waves[wave] = n;
      __syncthreads();
      int at = 0;
      for (int w = 0; w < wave; ++w) at += sh.waves[w];
      for (int b0 = from; b0 < to; b0 += 64) {
        const bool mine = b0 + lane < to && sh.group[b0 + lane] == g;
        const unsigned long long who = __ballot(mine);
        const int i = at + __popcll(who & ((1ull << lane) - 1));
        if (mine && i >= m0 && i <= m1) sh.list[i - m0] = b0 + lane;
        at += __popcll(who);
      }
      listed_group = g, listed_tile = tile;
    }
    __syncthreads();

    auto piece = [&](auto parts) {
      constexpr int PARTS = decltype(parts)::value;
      Rows<T, D, C8, PARTS> w;
      const int part = PARTS == 1 ? 0 : wave & 1, rows_at = 32 * (PARTS == 1 ? wave : wave >> 1);
      const bool busy = rows_at < tile_rows;           // of the wavefront; the others bring blocks alone
      const int row = rows_at + (lane & 31), mine = min(row, tile_rows - 1);
      const int member = (row0 + mine) / G - row0 / G, head = (row0 + mine) % G;
      const size_t home = (size_t)sh.list[member] * a.Hq + hk * G + head;                 // of out
      {
        const uint16_t* from = a.q + home * D + 8 * (lane >> 5);
#pragma unroll
        for (int e = 0; e < D / 16; ++e) w.q[e] = *reinterpret_cast<const v8s*>(from + 16 * e);
        // they arrive here: a wait inside the walk would be one for the blocks on their way
#pragma unroll
        for (int e = 0; e < D / 16; ++e) asm volatile("" : "+v"(w.q[e]));
      }
      w.clear();

      // blocks on their way: the rows that this wavefront brings.  Common tokens are whole pages, so that all rows of a chunk are there or none;
      // LDS gets other rows of the block for those (P is 0 there), or, from codes, zeros
      const int my_row = lane * 8 / D, my_chunk = lane % (D / 8);
      auto first_row = [&](int i) { return (i * kWaves + wave) * L::kRowsOf; };
      auto key_of = [&](int t, int i) {                // 31 bits are passed behind the end, where nothing is read
        const unsigned key = (unsigned)t * kBlock + first_row(i);
        return C8 || key < (unsigned)tokens ? key : (unsigned)t * kBlock + first_row(i) % 16;
      };
      // a lane has the page of one chunk of one block, from block page_t on: no scalar loads in the walk, whose results would be waited for with the
      // reads of LDS
      constexpr int kPages = 64 / L::kChunks;
      const int32_t* table = a.table + (size_t)__builtin_amdgcn_readfirstlane(sh.list[0]) * a.max_pages;
      int pages, page_t = t0 - kPages;
      auto row_at = [&](int t, int i) {
        if (t >= page_t + kPages) {
          page_t = t;
          const unsigned at = min((unsigned)a.max_pages - 1, key_of(t + lane / L::kChunks, lane % L::kChunks) >> shift);
          pages = min(a.n_pages - 1, max(0, table[at]));
        }
        const int p = __builtin_amdgcn_readlane(pages, (t - page_t) * L::kChunks + i);
        return (((size_t)p * a.Hkv + hk) << shift) + (key_of(t, i) & ((1u << shift) - 1));
      };
      constexpr int kRing = L::kRing;
      auto step = [&](int t, int s) {
        if (!busy) return;
        w.scores(sh.stage[s], part);
        w.soften(sh.scales[L::kScaled ? s : 0], part, tokens - t * kBlock, z.own.c);
        w.multiply(sh.stage[s], part);
      };
      auto next_slot = [&](int s) { return s + 1 == kRing ? 0 : s + 1; };
      if constexpr (C8) {
        auto load = [&](typename L::Block& x, int t) {
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i) {
            const bool there = t < t1 && (int)key_of(t, i) < tokens;
            const size_t at = row_at(t, i);
            const auto kd = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.k_pages + at * D), 0, there ? L::kRowsOf * D : 0, 0x00020000);
            const auto vd = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)a.v_pages + at * D), 0, there ? L::kRowsOf * D : 0, 0x00020000);
            const auto ksd = __builtin_amdgcn_make_buffer_rsrc((void*)(a.k_scales + at), 0, there ? L::kRowsOf : 0, 0x00020000);
            const auto vsd = __builtin_amdgcn_make_buffer_rsrc((void*)(a.v_scales + at), 0, there ? L::kRowsOf : 0, 0x00020000);
            x.k[i] = __builtin_amdgcn_raw_buffer_load_b64(kd, 8 * lane, 0, 0), x.v[i] = __builtin_amdgcn_raw_buffer_load_b64(vd, 8 * lane, 0, 0);
            x.ks[i] = __builtin_amdgcn_raw_buffer_load_b8(ksd, my_row, 0, 0), x.vs[i] = __builtin_amdgcn_raw_buffer_load_b8(vsd, my_row, 0, 0);
          }
        };
        auto write = [&](const typename L::Block& x, int s) {
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i) {
            const int r = first_row(i) + my_row;
            char *k = sh.stage[s] + r * L::kRow + 16 * (my_chunk ^ (r & 7)), *v = sh.stage[s] + L::kSide + r * L::kRow + ((16u * my_chunk) ^ Rows<T, D, C8, 1>::v_swizzle(r));
            *reinterpret_cast<v4i*>(k) = widen_chunk<T>(x.k[i], L::kScaled ? 1.f : scale_of(x.ks[i]));
            *reinterpret_cast<v4i*>(v) = widen_chunk<BF16>(x.v[i], scale_of(x.vs[i]));
            if constexpr (L::kScaled)
              if (my_chunk == 0) sh.scales[s][r] = scale_of(x.ks[i]);
          }
        };
        typename L::Block x, y;
        load(x, t0);
        load(y, t0 + 1);
        write(x, 0);
        lds_barrier();
        for (int t = t0; t < t1; t += 2) {
          load(x, t + 2);
          step(t, 0);
          write(y, 1);
          lds_barrier();
          if (t + 1 == t1) break;
          load(y, t + 3);
          step(t + 1, 1);
          write(x, 0);
          lds_barrier();
        }
      } else {
        // LDS is written in the order of the lanes: a lane reads the chunk that belongs in its place
        constexpr int kLoads = 2 * L::kChunks;
        const int r0 = first_row(0) + my_row;          // first_row(i) is the same but for multiples of eight
        const uint32_t k_off = my_row * L::kRow + 16 * (my_chunk ^ (r0 & 7)), v_off = my_row * L::kRow + ((16u * my_chunk) ^ Rows<T, D, C8, 1>::v_swizzle(r0));
        auto load = [&](int t, int s) {
          if (t >= t1) return;
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i) {
            const size_t at = row_at(t, i) * L::kRow;
            const uint32_t to = lds_address(sh.stage[s]) + first_row(i) * L::kRow;
            dma_b128((const char*)a.k_pages + at, k_off, to);
            dma_b128((const char*)a.v_pages + at, v_off, to + L::kSide);
          }
        };
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) load(t0 + i, i);
        for (int t = t0, s = 0; t < t1; ++t, s = next_slot(s)) {
          // block t is here: those behind it that are on their way may stay so
          if (kRing > 3 && t + 2 < t1) vm_wait<2 * kLoads>();
          else if (kRing > 2 && t + 1 < t1) vm_wait<kLoads>();
          else vm_wait<0>();
          lds_barrier();
          load(t + kRing - 1, s == 0 ? kRing - 1 : s - 1);
          step(t, s);
        }
      }

      // ---- both halves of a row's keys, and its place ----
      float l = w.l;
      {
        const uint32_t bits = __float_as_uint(l);
        const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
        l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
      }
      if constexpr (PARTS == 2) {
        lds_barrier();                                 // nobody reads the last block any more
        float(*mail)[64] = reinterpret_cast<float(*)[64]>(sh.stage) + (wave >> 1) * (D / 2);
        if (part == 1 && busy) {
#pragma unroll
          for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) mail[16 * n + i][lane] = w.o[n][i];
          sh.ml[wave >> 1][0][lane] = w.r, sh.ml[wave >> 1][1][lane] = l;
        }
        lds_barrier();
        if (part == 0 && busy) {
          const float other = sh.ml[wave >> 1][0][lane], top = fmaxf(w.r, other), k1 = fast_exp2(w.r - top), k2 = fast_exp2(other - top);
          w.r = top, l = l * k1 + sh.ml[wave >> 1][1][lane] * k2;
#pragma unroll
          for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) w.o[n][i] = w.o[n][i] * k1 + mail[16 * n + i][lane] * k2;
        }
      }
      if (busy && row < tile_rows && (PARTS == 1 || part == 0)) {
        const size_t slot = (size_t)blockIdx.x * kTile + row, to = t0 == 0 ? home : slot;
        float *to_o = t0 == 0 ? z.p.home_o : z.p.slot_o, *to_ml = t0 == 0 ? z.p.home_ml : z.p.slot_ml;
        const int half = lane >> 5;
        if (half == 0) {
          to_ml[2 * to] = w.r, to_ml[2 * to + 1] = l;
          // the last block lies in the share of its price's place
          if (t0 == 0) z.p.home_span[home] = make_int4((int)blockIdx.x + 1, (int)((unit + (long)weight * (blocks - 1)) / each) - (int)blockIdx.x, row, 0);
        }
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<v4f*>(to_o + to * D + 32 * n + 8 * i + 4 * half) = v4f{w.o[n][4 * i], w.o[n][4 * i + 1], w.o[n][4 * i + 2], w.o[n][4 * i + 3]};
      }
    };
    if (weight == 2) piece(std::integral_constant<int, 1>{});
    else piece(std::integral_constant<int, 2>{});

    u = end;
    if (u >= u_end) break;
    __syncthreads();                                   // the stage is free again
    if (u - g_base >= price(g)) {                      // the next group with members
      g_base += price(g);
      int next = g + 1;
      while (true) {
        const unsigned long long some = __ballot(next + lane < n_groups && sh.count[min(next + lane, n_groups - 1)] > 0);
        if (some != 0) {
          next += __builtin_ctzll(some);
          break;
        }
        next += 64;
      }
      g = __builtin_amdgcn_readfirstlane(next);
    }
  }
}

// One workgroup per sequence and query head: joins the parts of its common and its own tokens in the order of the tokens.  Threads take four channels of
// every kParts-th part.
template <int D, int kShares>
__global__ void __launch_bounds__(256) prefix_merge_kernel(PagedDecodeArgs a, PrefixLaunch z) {
  constexpr int kQuads = D / 4, kParts = 256 / kQuads, kTile = tile_rows(D);
  __shared__ float2 ml[kParts];
  __shared__ __align__(16) v4f sums[kParts][kQuads];
  const int tid = threadIdx.x, quad = tid % kQuads, part = tid / kQuads;
  const size_t at = blockIdx.x;
  const int b = (int)(at / a.Hq), h = (int)(at % a.Hq), hk = h / z.own.G, gh = h % z.own.G, shift = z.own.shift, capacity = a.max_pages << shift;
  const int len = min(capacity, max(0, a.seqlens[b])), common = common_tokens(z.own.groups, capacity, shift, b, len);
  if (len == 0) {
    if (part == 0) store_out4(a.out, a.out_dt, at * D + 4 * quad, 0.f, 0.f, 0.f, 0.f);
    if (a.lse != nullptr && tid == 0) a.lse[at] = -__builtin_inff();
    return;
  }
  const int4 span = common > 0 ? z.p.home_span[at] : make_int4(0, -1, 0, 0);
  const int2 own = len > common ? z.own.own_span[(size_t)b * a.Hkv + hk] : make_int2(0, -1);
  const int n1 = span.y + 1, n = n1 + own.y + 1;
  v4f o = {0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  for (int i = part; i < n; i += kParts) {
    const float *from_o, *from_ml;
    size_t row;
    if (i < n1) {
      row = i == 0 ? at : (size_t)(span.x + i - 1) * kTile + span.z;
      from_o = i == 0 ? z.p.home_o : z.p.slot_o, from_ml = i == 0 ? z.p.home_ml : z.p.slot_ml;
    } else {
      const int j = i - n1;
      row = j == 0 ? at : (size_t)(own.x + j - 1) * z.own.G + gh;
      from_o = j == 0 ? z.own.own_o : z.own.w.part_o, from_ml = j == 0 ? z.own.own_ml : z.own.w.part_ml;
    }
    const v4f x = *reinterpret_cast<const v4f*>(from_o + row * D + 4 * quad);
    const float2 y = *reinterpret_cast<const float2*>(from_ml + 2 * row);
    const float top = fmaxf(m, y.x), k1 = fast_exp2(m - top), k2 = fast_exp2(y.x - top);
    m = top, l = l * k1 + y.y * k2, o = o * k1 + x * k2;
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

// Workspace, all parts 16-byte aligned
struct Layout {
  size_t home_o, home_ml, home_span, slot_o, slot_ml, own_o, own_ml, own_span, part_o, part_ml, total;
};
Layout layout_of(bool codes, int B, int Hq, int Hkv, int D) {
  Layout y;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 15) & ~(size_t)15;
    return here;
  };
  const size_t rows = (size_t)B * Hq, slots = (size_t)kPrefixShares * tile_rows(D), parts = (size_t)shares_of(codes) * (Hq / Hkv);
  y.home_o = take(rows * D * 4), y.home_ml = take(rows * 8), y.home_span = take(rows * 16);
  y.slot_o = take(slots * D * 4), y.slot_ml = take(slots * 8);
  y.own_o = take(rows * D * 4), y.own_ml = take(rows * 8), y.own_span = take((size_t)B * Hkv * 8);
  y.part_o = take(parts * D * 4), y.part_ml = take(parts * 8);
  y.total = at;
  return y;
}

template <typename T, int D, bool C8>
void launch(const PagedPrefixArgs& args, hipStream_t st) {
  const PagedDecodeArgs& a = args.d;
  const Layout y = layout_of(C8, a.B, a.Hq, a.Hkv, D);
  char* w = (char*)a.workspace;
  PrefixLaunch z;
  z.own = launch_of(a, C8, a.workspace);
  z.own.groups = Groups{args.group_of, args.group_lens, args.n_groups};
  z.own.w.tail = nullptr;
  z.own.w.part_o = (float*)(w + y.part_o), z.own.w.part_ml = (float*)(w + y.part_ml);
  z.own.own_o = (float*)(w + y.own_o), z.own.own_ml = (float*)(w + y.own_ml), z.own.own_span = (int2*)(w + y.own_span);
  z.p.home_o = (float*)(w + y.home_o), z.p.home_ml = (float*)(w + y.home_ml), z.p.home_span = (int4*)(w + y.home_span);
  z.p.slot_o = (float*)(w + y.slot_o), z.p.slot_ml = (float*)(w + y.slot_ml);
  prefix_kernel<T, D, C8><<<dim3(kPrefixShares), dim3(64 * prefix_waves(D)), 0, st>>>(a, z);
  const dim3 grid(shares_of(C8)), block(64 * waves_of(D));
  if (z.own.G <= 16) paged_decode_kernel<T, D, 1, C8, true><<<grid, block, 0, st>>>(a, z.own);
  else paged_decode_kernel<T, D, 2, C8, true><<<grid, block, 0, st>>>(a, z.own);
  prefix_merge_kernel<D, shares_of(C8)><<<dim3((unsigned)((long)a.B * a.Hq)), dim3(256), 0, st>>>(a, z);
}
template <typename T, bool C8>
void launch(const PagedPrefixArgs& a, hipStream_t st) {
  if (a.d.D == 64) launch<T, 64, C8>(a, st);
  else if (a.d.D == 128) launch<T, 128, C8>(a, st);
  else launch<T, 256, C8>(a, st);
}

}  // namespace

size_t paged_prefix_workspace(int bits, int B, int Hq, int Hkv, int n_groups, int max_pages, int page_size, int D) {
  return layout_of(bits == 8, B, Hq, Hkv, D).total;
}

void launch_paged_prefix(const PagedPrefixArgs& a, int bits, hipStream_t st) {
  if (bits == 8 && a.d.dt == THRIFT_F16) launch<F16, true>(a, st);
  else if (bits == 8) launch<BF16, true>(a, st);
  else if (a.d.dt == THRIFT_F16) launch<F16, false>(a, st);
  else launch<BF16, false>(a, st);
}

}  // namespace thrift
