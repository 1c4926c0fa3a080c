// Attention of one new token per sequence where sequences start with the same pages.
//
// Three launches.  The first takes the common tokens: a group's members times the G query heads of a KV head are the rows of a product with
// the group's keys, and with P and its values, so that these are read once per tile of rows instead of once per sequence.  The second
// walks every sequence's own tokens (thrift_paged_walk.h).  The third joins what the two left of every row, and writes the results.
//
// Common tokens.  A tile is at most kTile rows of one group and KV head, a wavefront has 32 of them in the columns of 32 x 32 matrix
// tiles and walks blocks of 64 keys:
//   S = K Q^T      64 keys x 32 rows;  r: a reference of the row, P = 2^(S c - r)
//   O^T += V^T P^T channels x 32 rows; a lane's part of S is its operand P, without passing through LDS or other lanes
// K and V of a block lie in LDS for all wavefronts, V is transposed by the reads.  They lie in a ring of four blocks, with a barrier for every second one (256 channels: a ring of two), where LDS DMA brings them.
// With at most half a tile of rows, wavefronts take half a block's keys each, two to a row.
//   8-bit pages come through registers and are converted on their way, once for all wavefronts: values and, for bf16 queries, keys times their scales,
// which bf16 holds exactly; for fp16 queries keys without, and the scales, in LDS too, are factors of the scores.
//   P is two 16-bit pieces, high and low, for two products, as in the walk of own tokens: what a result holds does not depend on which tokens are common.  Rounded once, results were
// off by 1.1e-3 of their norm (bf16; 1.5e-4 fp16) and 64 x 32768 tokens of 64/8 heads took 107 us instead of 134.  The pieces take the registers of their scores.
//   What bounds it: for large groups instructions.  64 x 32768 tokens of 64/8 heads are 103 GFLOP with the second piece, 52 us at the 2.0 PFLOP/s that matrix instructions reach on all
// CUs; a score's exponential, sum, two roundings and maximum next to them cost as much again (a vector instruction beside matrix instructions takes 0.9 ns of a
// SIMD).  The common keys and values are 134 MB, read from memory once, by both tiles of a KV head.  For small groups the three launches do.
//   The reference is raised where the row's largest score so far has passed it by as much as P may hold (fp16: 2^15, bf16: 1, so that sums of values near the
// end of its range stay finite), and then lies some binades from that score, so that O is rarely multiplied: 7 below for fp16, which keeps P normal down to
// 2^-21 of the largest, 8 above for bf16.  Scores from 2^20 on are rounded before r is taken off, as in the walk: a fused difference would be off by binades.
//   Tiles are cut into parts of equal numbers of blocks on the GPU, so that there is one for every CU: a tile's first part is written to its rows' places, the
// others to slots.
#include "thrift_paged_walk.h"
#include "thrift_tile.h"

namespace thrift {

namespace {

constexpr int kBlock = 64;                             // keys
constexpr int kPrefixShares = kCus;
// What a block costs for a tile of rows, and for half a one at most, where two wavefronts share its keys.  From codes, 96 x 16384 tokens: 79.5 us in all, with 2 : 1
// 83, with 5 : 3 79
constexpr int kPriceFull = 3, kPriceHalf = 2;
// Wavefronts of a workgroup.  256 channels: four, with all registers that two have otherwise.
constexpr int prefix_waves(int D) { return D == 256 ? 4 : 8; }
constexpr int tile_rows(int D) { return 32 * prefix_waves(D); }

struct Prefix {
  float *home_o, *home_ml;                             // [B*Hq][D], [B*Hq][2]: a tile's first part
  int4* home_span;                                     // [B*Hq]: first slot with more of the row's tile, how many, the row in the tile
  float *slot_o, *slot_ml;                             // [kPrefixShares][tile_rows][D], [..][2]: the other parts
};

// Groups of sequences that start with the same pages
struct Groups {
  const int32_t* of;         // [B]
  const int32_t* lens;       // [n]
  int n;
};
struct PrefixLaunch {
  Prefix p;
  Groups groups;
  int32_t* common;           // [B] tokens in front of every sequence that the first launch takes
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
template <> struct Reference<BF16> { static constexpr float kBelow = -8.f, kMost = 0.f; };

constexpr int kMaxSeqs = kMapMaxSeqs, kMaxGroups = kMapMaxSeqs;
// A group whose common tokens, but for one member's, are fewer than this together is left alone: a part of a tile costs as much in front of and behind its walk as
// reading about so many tokens
constexpr int kLeastShared = 512;


template <typename T, int D, bool C8>
struct Tiles {
  using P = std::conditional_t<C8, BF16, T>;
  static constexpr bool kScaled = C8 && std::is_same_v<T, F16>;             // keys lie in LDS without their scales
  static constexpr int kWaves = prefix_waves(D), kThreads = 64 * kWaves, kTile = tile_rows(D);
  static constexpr int kRow = 2 * D;                                        // bytes of a row in LDS
  static constexpr int kSide = kBlock * kRow;                               // bytes of a block of K or V
  static constexpr int kRing = D == 256 ? 2 : 4;                      // blocks of K, and of V, in LDS
  static constexpr int kChunks = kBlock * D / 8 / kThreads;                 // 16-byte chunks of K, and of V, of a thread
  static constexpr int kRowsOf = 512 / D;                                   // rows of a wavefront's chunk
  static_assert(kChunks * kWaves * kRowsOf == kBlock, "");

  struct Shared {
    union {
      struct {
        char k[kRing][kSide], v[kRing][kSide];
      };
      char stage[8192 * kWaves];                       // of results
    };
    float scales[kScaled ? kRing : 1][kScaled ? kBlock : 1];
    float ml[kWaves / 2][2][64];
    int count[kMaxGroups];                             // members of every group
    uint16_t group[kMaxSeqs];                          // of every sequence; 0xffff: none
    int list[kTile + 1];                               // members that have rows in the tile
    uint3 sums[kWaves];
    int waves[kWaves];
    uint32_t start_share, start_unit;
    int start_group;
  };

  // K or V of a block of codes on its way
  struct Block {
    v2i codes[kChunks];
    uint32_t scales[kChunks];
  };
};

// The lane's number, formed where it stands
__device__ __forceinline__ int lane_here() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// One tile's rows in a wavefront: 32 of them.
//
// A step has the scores of block t in `s`.  It forms P of block t between the products of the queries with the keys of block t + 1, and the largest of
// those scores between the products of P with the values of block t: matrix and vector instructions take turns in one stream, held in place by
// fences, and reads of LDS run some products ahead.  Without that the two kinds hardly overlapped, neither within a wavefront nor between the two of a SIMD.
template <typename T, int D, bool C8, int PARTS>
struct Rows {
  using L = Tiles<T, D, C8>;
  using P = typename L::P;
  static constexpr int NT = 2 / PARTS;                 // 32-key halves of a block
  static constexpr int kKeys = NT * D / 16, kValues = 2 * NT * (D / 32);    // products with the keys and with the values of a block
  static constexpr int kAhead = 4;                     // reads ahead of their products
  typedef v16f Scores[NT];
  v8s q[D / 16];
  v16f o[D / 32];
  float r, l, top;                                     // reference, this lane's part of the sum, largest score of the next block
  bool large;                                          // of the wavefront: some reference from 2^20 on
  int part, half, row;                                 // which half of a block's keys, of PARTS; of the lane

  __device__ __forceinline__ void clear(int which) {
    part = which, half = (threadIdx.x & 63) >> 5, row = threadIdx.x & 31;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][i] = 0.f;
    r = -__FLT_MAX__, l = 0.f, large = false;
  }

  // Operand i of the keys: half i / (D / 16) of the block.  Chunk x of a K row lies at x ^ (row & 7): eight neighbouring rows at one chunk fill all banks
  struct KeyReader {
    const char* from;
    uint32_t swizzled;
    __device__ __forceinline__ v8s operator()(int i) const {
      const int t = i / (D / 16), e = i % (D / 16);
      return *reinterpret_cast<const v8s*>(from + 32 * t * L::kRow + ((swizzled ^ (32u * (e & 3))) + 128u * (e >> 2)));
    }
  };
  __device__ __forceinline__ KeyReader keys_in(const char* k) const { return KeyReader{k + (32 * part + row) * L::kRow, 16u * (half ^ (row & 7))}; }
  __device__ __forceinline__ void product(Scores& n, int i, v8s k) const {
    if (i % (D / 16) == 0) {
#pragma unroll
      for (int j = 0; j < 16; ++j) n[i / (D / 16)][j] = 0.f;
    }
    n[i / (D / 16)] = T::mfma(k, q[i % (D / 16)], n[i / (D / 16)]);
  }

  // The scores of a block, where nothing else is to be done
  __device__ __forceinline__ void scores(Scores& n, const char* k, const float* scales, int valid, float c) {
    const KeyReader key = keys_in(k);
#pragma unroll
    for (int i = 0; i < kKeys; ++i) product(n, i, key(i));
    settle(n, scales, valid);
    float x = n[0][0];
#pragma unroll
    for (int i = 1; i < 16 * NT; ++i) x = fmaxf(x, n[i >> 4][i & 15]);
    top = both_halves_max(x) * c;
  }

  // Scales of the keys, where K lies in LDS without them; `valid` keys of the block are there.  Register i of half t: key 32 t + 8 (i / 4) + 4 half + i % 4
  __device__ __forceinline__ void settle(Scores& n, const float* scales, int valid) const {
    if constexpr (L::kScaled) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const v4f f = *reinterpret_cast<const v4f*>(scales + 32 * (part + t) + 2 * i + 4 * half);
#pragma unroll
          for (int e = 0; e < 4; ++e) n[t][i + e] *= f[e];
        }
    }
    if (valid < kBlock) {
      // The lane's number is asked for here, and the rest are constants: keys of registers, or what they start from, would be formed in front of the walk and kept through it
      const int there = valid - 32 * part - 4 * (lane_here() >> 5);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * t + 8 * (i >> 2) + (i & 3) >= there) n[t][i] = -__builtin_inff();
    }
  }

  // k: K of block t + 1 (whatever LDS holds there behind the last one), with its scales and keys; v: V of block t; ask(): between the two series of products
  template <typename F>
  __device__ __forceinline__ void step(Scores& s, Scores& n, const char* k, const float* scales, int valid, const char* v, float c, F ask) {
    if (__ballot(top - r > Reference<P>::kMost)) {
      // a score past 2^20 and its difference to a reference are no longer exact in one fused step
      const bool far = fabsf(top) >= 0x1p20f && fabsf(top) < __builtin_inff();
      const float next = top > r ? (far ? top : top - Reference<P>::kBelow) : r;
      const float raised = fmaxf(next, r), keep = fast_exp2(r - raised);
      r = raised, l *= keep;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) o[i] *= keep;
      large = __ballot(fabsf(r) >= 0x1p20f && r > -__FLT_MAX__) != 0;
    }
    float f = c, off = r;
    if (large) {
#pragma clang fp contract(off)
#pragma unroll
      for (int i = 0; i < 16 * NT; ++i) {
        const float x = s[i >> 4][i & 15] * c;
        s[i >> 4][i & 15] = x - r;
      }
      f = 1.f, off = 0.f;
    }

    // V operands: slots 8 half + e of step u of half t are keys 32 t + 16 u + 8 (e / 4) + 4 half + e % 4, as P's registers are.  A group of 16 lanes
    // reads four keys x 16 channels and gets four keys of a channel per lane
    typedef v4s __attribute__((address_space(3))) * lds_v4s_ptr;
    const int i16 = row & 15, key_row = 4 * half + (i16 >> 2);
    const char* v0 = v + (32 * part + key_row) * L::kRow;
    const uint32_t v_at = (32u * (row >> 4) + 8u * (i16 & 3)) ^ v_swizzle(key_row);
    v4s value[kAhead + 1][2];
    auto read_value = [&](int i) {
      const int tu = i / (D / 32), n = i % (D / 32);
      const char* from = v0 + 16 * tu * L::kRow + ((v_at ^ (64u * (n & 3))) + 256u * (n >> 2));
      value[i % (kAhead + 1)][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(from));
      value[i % (kAhead + 1)][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)(from + 8 * L::kRow));
    };
    const KeyReader key = keys_in(k);
    v8s operand[kAhead + 1];
    v4i p[NT][2], low[NT][2];
    float sums[4] = {0.f, 0.f, 0.f, 0.f};
    // elements 2 i and 2 i + 1 of the lane's P
    auto pair = [&](int i) {
      const int t = i >> 3, e = 2 * i & 15;
      const float x = fast_exp2(__builtin_fmaf(s[t][e], f, -off)), y = fast_exp2(__builtin_fmaf(s[t][e + 1], f, -off));
      sums[e & 2] += x, sums[(e & 2) + 1] += y;
      const uint32_t high = pack16<P>(x, y);
      p[t][e >> 3][(e & 7) >> 1] = (int)high;
      low[t][e >> 3][(e & 7) >> 1] = (int)pack16<P>(x - P::to_float((uint16_t)high), y - P::to_float((uint16_t)(high >> 16)));
      // here and not behind the branch on `valid`, to where the compiler takes them otherwise, away from the products
      asm volatile("" : "+v"(p[t][e >> 3][(e & 7) >> 1]), "+v"(low[t][e >> 3][(e & 7) >> 1]), "+v"(sums[e & 2]), "+v"(sums[(e & 2) + 1]));
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) operand[i] = key(i);
    fence();
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      product(n, i, operand[i % (kAhead + 1)]);
      if (i + kAhead < kKeys) operand[(i + kAhead) % (kAhead + 1)] = key(i + kAhead);
      else read_value(i + kAhead - kKeys);
#pragma unroll
      for (int x = 8 * NT * i / kKeys; x < 8 * NT * (i + 1) / kKeys; ++x) pair(x);
      fence();
    }
    l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
    ask();
    settle(n, scales, valid);
    float most = n[0][0];
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const int tu = i / (D / 32), tile = i % (D / 32), at = i % (kAhead + 1);
      const v8s channels = __builtin_shufflevector(value[at][0], value[at][1], 0, 1, 2, 3, 4, 5, 6, 7);
      o[tile] = P::mfma(channels, __builtin_bit_cast(v8s, p[tu >> 1][tu & 1]), o[tile]);
      o[tile] = P::mfma(channels, __builtin_bit_cast(v8s, low[tu >> 1][tu & 1]), o[tile]);
      if (i + kAhead < kValues) read_value(i + kAhead);
#pragma unroll
      for (int x = 16 * NT * i / kValues; x < 16 * NT * (i + 1) / kValues; ++x) most = fmaxf(most, n[x >> 4][x & 15]);
      fence();
    }
    top = both_halves_max(most) * c;
  }

  // What a V row's offsets are swizzled by: of eight neighbouring rows, four at one 64-byte piece, or all at one 32-byte piece, fill all banks
  static __device__ __forceinline__ uint32_t v_swizzle(int row) { return 64u * (D == 64 ? (row >> 1) & 1 : row & 3) + 32u * ((row >> 2) & 1); }
};

template <typename T, int D, bool C8>
__global__ void __launch_bounds__(64 * prefix_waves(D)) prefix_kernel(PagedDecodeArgs a, PrefixLaunch z) {
  using L = Tiles<T, D, C8>;
  __shared__ __align__(16) typename L::Shared sh;
  constexpr int kWaves = L::kWaves, kThreads = L::kThreads, kTile = L::kTile;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = z.own.G, shift = z.own.shift, capacity = a.max_pages << shift, n_groups = z.groups.n;
  auto tokens_of = [&](int g) { return min(capacity, max(0, z.groups.lens[g])) >> shift << shift; };
  auto blocks_of = [&](int tokens) { return (int)(((unsigned)tokens + kBlock - 1) / kBlock); };

  // ---- members of the groups ----
  for (int g = tid; g < n_groups; g += kThreads) sh.count[g] = 0;
  __syncthreads();
  for (int b = tid; b < a.B; b += kThreads) {
    int g = z.groups.of[b];
    const int len = min(capacity, max(0, a.seqlens[b]));
    if ((unsigned)g < (unsigned)n_groups) {
      const int n = tokens_of(g);
      if (n == 0 || len < n) g = 0xffff;
    } else {
      g = 0xffff;
    }
    sh.group[b] = (uint16_t)g;
    if (g != 0xffff) atomicAdd(&sh.count[g], 1);
  }
  __syncthreads();
  for (int g = tid; g < n_groups; g += kThreads) {
    const int n = sh.count[g];
    if (n > 0 && (long)(n - 1) * tokens_of(g) < kLeastShared) sh.count[g] = 0;
  }
  __syncthreads();
  if (blockIdx.x == 0)                                 // for the launches behind
    for (int b = tid; b < a.B; b += kThreads) {
      const int g = sh.group[b];
      z.common[b] = g != 0xffff && sh.count[g] > 0 ? tokens_of(g) : 0;
    }

  // ---- parts of tiles: a unit is a tile of a KV head, and has as many parts of equal numbers of blocks as its price asks for ----
  // At most one per member, KV head and block, and a group has two members at least; with pages of 16 tokens a block may have no more.  Four per member, KV head
  // and 64 tokens are below 2^32 for the sizes that are taken (B * Hkv * tokens / 32 below 2^30)
  struct Units {
    int full, rest, blocks;                            // full tiles, the price of a block of the other one (0: there is none), blocks
    uint32_t units, price;
  };
  auto units_of = [&](int g) {
    Units x = {0, 0, 0, 0, 0};
    const int rows = sh.count[g] * G;
    if (rows == 0) return x;
    x.blocks = blocks_of(tokens_of(g)), x.full = rows / kTile;
    const int left = rows - x.full * kTile;
    x.rest = left == 0 ? 0 : left > kTile / 2 ? kPriceFull : kPriceHalf;
    x.units = (uint32_t)a.Hkv * (x.full + (left > 0)), x.price = (uint32_t)a.Hkv * (kPriceFull * x.full + x.rest) * x.blocks;
    return x;
  };
  const int per = (n_groups + kThreads - 1) / kThreads, g0 = tid * per, g1 = min(n_groups, g0 + per);
  // sums over the workgroup of three numbers of every thread: of the threads in front, and of all
  struct Three { uint32_t v[3]; };
  auto sums_of = [&](const Three& x, Three& front, Three& all) {
    Three incl = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const uint32_t other = __shfl_up(incl.v[i], d);
        if (lane >= d) incl.v[i] += other;
      }
    __syncthreads();
    if (lane == 63) sh.sums[wave] = make_uint3(incl.v[0], incl.v[1], incl.v[2]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) front.v[i] = incl.v[i] - x.v[i], all.v[i] = 0;
    for (int w = 0; w < kWaves; ++w) {
      const uint3 sum = sh.sums[w];
      const Three y = {{sum.x, sum.y, sum.z}};
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        if (w < wave) front.v[i] += y.v[i];
        all.v[i] += y.v[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) all.v[i] = __builtin_amdgcn_readfirstlane(all.v[i]);
  };
  Three mine = {{0, 0, 0}}, front, all;
  for (int g = g0; g < g1; ++g) {
    const Units x = units_of(g);
    mine.v[0] += x.price, mine.v[1] += x.units;
  }
  sums_of(mine, front, all);
  const uint32_t total = all.v[0], all_units = all.v[1];
  if (total == 0) return;                              // the whole workgroup
  // The price of a part.  Parts of total / 256 where they come to 256 at most, as they do where units are alike; otherwise larger ones, so that with at most 128 units every workgroup
  // gets one part at most.  The parts behind a unit's first are fewer than the slots in any case: their prices sum up to less than `total`.
  auto over = [](uint32_t x, uint32_t y) { return x / y + (x % y != 0); };
  const uint32_t tight = over(total, kPrefixShares), loose = over(total, all_units < kPrefixShares / 2 ? kPrefixShares - all_units : kPrefixShares / 2);
  auto parts_of = [&](int price_of_block, int blocks, uint32_t each) { return (int)min((uint32_t)blocks, over((uint32_t)price_of_block * blocks, each)); };
  auto shares_of_group = [&](const Units& x, uint32_t each) -> uint32_t {
    if (x.units == 0) return 0;
    return (uint32_t)a.Hkv * (x.full * parts_of(kPriceFull, x.blocks, each) + (x.rest ? parts_of(x.rest, x.blocks, each) : 0));
  };
  mine.v[0] = mine.v[2] = 0;
  for (int g = g0; g < g1; ++g) {
    const Units x = units_of(g);
    mine.v[0] += shares_of_group(x, tight), mine.v[2] += shares_of_group(x, loose);
  }
  sums_of(mine, front, all);
  const bool fits = all.v[0] <= kPrefixShares;
  const uint32_t each = fits ? tight : loose, all_shares = fits ? all.v[0] : all.v[2], share_front = fits ? front.v[0] : front.v[2], unit_front = front.v[1];
  const uint32_t shares = fits ? mine.v[0] : mine.v[2];

  for (uint32_t share = blockIdx.x; share < all_shares; share += kPrefixShares) {
    // ---- the part of a tile that this share is ----
    __syncthreads();                                   // LDS is free again
    if (share_front <= share && share < share_front + shares) {
      uint32_t at = share_front, unit = unit_front;
      for (int g = g0; g < g1; ++g) {
        const Units x = units_of(g);
        const uint32_t n = shares_of_group(x, each);
        if (share < at + n) {
          sh.start_group = g, sh.start_share = at, sh.start_unit = unit;
          break;
        }
        at += n, unit += x.units;
      }
    }
    __syncthreads();
    const int g = __builtin_amdgcn_readfirstlane(sh.start_group), members = __builtin_amdgcn_readfirstlane(sh.count[g]);
    const int tokens = __builtin_amdgcn_readfirstlane(tokens_of(g)), blocks = blocks_of(tokens);
    const int rows = members * G, full = rows / kTile, n_full = parts_of(kPriceFull, blocks, each);
    uint32_t rel = share - __builtin_amdgcn_readfirstlane(sh.start_share), unit = __builtin_amdgcn_readfirstlane(sh.start_unit);
    const bool wide = rel < (uint32_t)a.Hkv * full * n_full || rows - full * kTile > kTile / 2;
    int tile = full, parts = n_full;
    if (rel >= (uint32_t)a.Hkv * full * n_full) {
      rel -= (uint32_t)a.Hkv * full * n_full, unit += (uint32_t)a.Hkv * full;
      parts = wide ? n_full : parts_of(kPriceHalf, blocks, each);
    } else {
      tile = rel / ((uint32_t)n_full * a.Hkv);
      rel -= (uint32_t)tile * n_full * a.Hkv, unit += (uint32_t)tile * a.Hkv;
    }
    const int hk = rel / (uint32_t)parts, number = rel - hk * parts;
    unit += hk;
    const int t0 = (int)((uint64_t)number * blocks / parts), t1 = (int)((uint64_t)(number + 1) * blocks / parts);
    const uint32_t slot_of_part = share - unit - 1;    // parts behind the first of their unit, counted through
    const int row0 = tile * kTile, tile_rows = min(kTile, rows - row0);

    // ---- the tile's members, in the order of the batch ----
    {
      const int m0 = row0 / G, m1 = (row0 + tile_rows - 1) / G;
      const int chunk = (a.B + kThreads - 1) / kThreads * 64, from = wave * chunk, to = min(a.B, from + chunk);
      int n = 0;
      for (int b0 = from; b0 < to; b0 += 64) n += __popcll(__ballot(b0 + lane < to && sh.group[b0 + lane] == g));
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
    }
    __syncthreads();

    auto piece = [&](auto halves) {
      constexpr int PARTS = decltype(halves)::value;
      Rows<T, D, C8, PARTS> w;
      const int part = PARTS == 1 ? 0 : wave & 1, rows_at = 32 * (PARTS == 1 ? wave : wave >> 1);
      const bool busy = rows_at < tile_rows;           // of the wavefront; the others bring blocks alone
      const int row = rows_at + (lane & 31), mine = min(row, tile_rows - 1);
      const int member = (row0 + mine) / G - row0 / G, head = (row0 + mine) % G;
      const size_t home = (size_t)sh.list[member] * a.Hq + hk * G + head;                 // of out
      auto ask = [&]() {
        const uint16_t* from = a.q + home * D + 8 * (lane >> 5);
#pragma unroll
        for (int e = 0; e < D / 16; ++e) w.q[e] = *reinterpret_cast<const v8s*>(from + 16 * e);
      };
      w.clear(part);

      // blocks on their way: the rows that this wavefront brings.  Common tokens are whole pages, so that all rows of a chunk are there or none;
      // LDS gets other rows of the block for those (P is 0 there), or, from codes, zeros
      const int my_row = lane * 8 / D, my_chunk = lane % (D / 8);
      auto first_row = [&](int i) { return (i * kWaves + wave) * L::kRowsOf; };
      auto key_of = [&](int t, int i) {                // 31 bits are passed behind the end, where nothing is read
        const unsigned key = (unsigned)t * kBlock + first_row(i);
        return C8 || key < (unsigned)tokens ? key : (unsigned)t * kBlock + first_row(i) % 16;
      };
      // A lane has the place of one chunk of one block in the pages, from block place_t on: no scalar loads in the walk, whose results would be waited for with the
      // reads of LDS, and few scalar instructions.  The window moves on with K of a block t and then begins at t - 1: the forms ask for V of t - 1 in front of K of t, or
      // behind it where a side at a time is on its way, and never for an earlier block
      constexpr int kPlaces = 64 / L::kChunks;
      const int32_t* table = a.table + (size_t)__builtin_amdgcn_readfirstlane(sh.list[0]) * a.max_pages;
      size_t place;
      int place_t;
      auto look_up = [&](int t) {
        place_t = t;
        const unsigned key = key_of(t + lane / L::kChunks, lane % L::kChunks);
        const int p = min(a.n_pages - 1, max(0, table[min((unsigned)a.max_pages - 1, key >> shift)]));
        place = ((((size_t)p * a.Hkv + hk) << shift) + (key & ((1u << shift) - 1))) * (C8 ? 1 : L::kRow);
      };
      auto place_of = [&](int t, int i) {              // bytes, or rows of codes
        if (t >= place_t + kPlaces) look_up(t - 1);
        const int at = (t - place_t) * L::kChunks + i;
        return (size_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)place, at) | (size_t)(uint32_t)__builtin_amdgcn_readlane((int)(place >> 32), at) << 32;
      };
      constexpr int kRing = L::kRing;
      look_up(t0);                                     // both on their way together
      ask();
      // The walk: K is brought one block ahead of V, since a step reads K of block t + 1 and V of block t.  begin(): until K of the first block is in LDS; bring(t): at
      // the start of step t, until K of t + 1 and V of t are; ask_for(t): inside it, what is to come.
      const float c = z.own.c;
      auto arrive = [&]() {                            // the queries, here: a wait inside the walk would be one for the blocks on their way
#pragma unroll
        for (int e = 0; e < D / 16; ++e) asm volatile("" : "+v"(w.q[e]));
      };
      auto slot = [&](int t) { return (unsigned)(t - t0) % kRing; };
      auto scales_of = [&](int t) { return sh.scales[L::kScaled ? slot(t) : 0]; };
      auto keys_from = [&](int t) { return (int)((unsigned)tokens - (unsigned)t * kBlock); };         // 31 bits are passed behind the last block
      auto walk = [&](auto begin, auto bring, auto ask_for) {
        begin();
        if (t0 == t1) return;
        if (!busy) {
          for (int t = t0; t < t1; ++t) bring(t), ask_for(t);
          return;
        }
        typename Rows<T, D, C8, PARTS>::Scores x, y;
        w.scores(x, sh.k[0], scales_of(t0), keys_from(t0), c);
        auto step = [&](int t, auto& s, auto& n) {
          bring(t);
          w.step(s, n, sh.k[slot(t + 1)], scales_of(t + 1), keys_from(t + 1), sh.v[slot(t)], c, [&]() { ask_for(t); });
        };
        for (int t = t0; t < t1; t += 2) {
          step(t, x, y);
          if (t + 1 == t1) break;
          step(t + 1, y, x);
        }
      };
      if constexpr (C8) {
        auto load = [&](typename L::Block& x, const void* pages, const uint8_t* scales, int t) {
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i) {
            const bool there = t < t1 && (int)key_of(t, i) < tokens;
            const size_t at = there ? place_of(t, i) : 0;
            const auto codes = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)pages + at * D), 0, there ? L::kRowsOf * D : 0, 0x00020000);
            const auto bytes = __builtin_amdgcn_make_buffer_rsrc((void*)(scales + at), 0, there ? L::kRowsOf : 0, 0x00020000);
            x.codes[i] = __builtin_amdgcn_raw_buffer_load_b64(codes, 8 * lane, 0, 0), x.scales[i] = __builtin_amdgcn_raw_buffer_load_b8(bytes, my_row, 0, 0);
          }
        };
        // rows of a thread's chunks are the same but for multiples of eight, and so are their places in a row
        constexpr int kApart = kWaves * L::kRowsOf;
        static_assert(L::kChunks == 1 || kApart % 8 == 0, "");
        const int r0 = first_row(0) + my_row;
        const uint32_t k_off = r0 * L::kRow + 16 * (my_chunk ^ (r0 & 7)), v_off = r0 * L::kRow + ((16u * my_chunk) ^ Rows<T, D, C8, 1>::v_swizzle(r0));
        auto write_k = [&](const typename L::Block& x, int s) {
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i) {
            *reinterpret_cast<v4i*>(sh.k[s] + k_off + i * kApart * L::kRow) = widen_chunk<T>(x.codes[i], L::kScaled ? 1.f : scale_of(x.scales[i]));
            if constexpr (L::kScaled)
              if (my_chunk == 0) sh.scales[s][r0 + i * kApart] = scale_of(x.scales[i]);
          }
        };
        auto write_v = [&](const typename L::Block& x, int s) {
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i)
            *reinterpret_cast<v4i*>(sh.v[s] + v_off + i * kApart * L::kRow) = widen_chunk<BF16>(x.codes[i], scale_of(x.scales[i]));
        };
        typename L::Block k, v;
        auto load_k = [&](typename L::Block& x, int t) { load(x, a.k_pages, a.k_scales, t); };
        auto load_v = [&](typename L::Block& x, int t) { load(x, a.v_pages, a.v_scales, t); };
        if constexpr (kRing == 4) {
          // As below, a barrier for every second step (96 x 16384 tokens of 32/8 heads: 82.5 us in all with one for every step, now 79.5); a step
          // writes K of t + 3 and V of t + 2
          walk(
              [&]() {
                typename L::Block k1, v1, k2;
                load_k(k, t0), load_v(v, t0), load_k(k1, t0 + 1), load_v(v1, t0 + 1), load_k(k2, t0 + 2);
                arrive();
                write_k(k, 0), write_v(v, 0), write_k(k1, 1), write_v(v1, 1), write_k(k2, 2);
                load_v(v, t0 + 2), load_k(k, t0 + 3);
                lds_barrier();
              },
              [&](int t) {
                if (((t - t0) & 1) == 0) lds_barrier();      // the first of them: K of t0 is read, whose place K of t0 + 4 gets in the next step
                write_v(v, slot(t + 2)), write_k(k, slot(t + 3));
                load_v(v, t + 3), load_k(k, t + 4);
              },
              [](int) {});
        } else if constexpr (L::kScaled) {
          // One side at a time: K of t + 2 is written inside step t, where K of t is read, and the registers then take V of t + 1.  256 channels, 64 x 32768 tokens of 64/8 heads:
          // 350 us instead of 380 with fp16 queries, which spill registers with both sides on their way, but 352 instead of 335 with bf16
          walk(
              [&]() {
                typename L::Block k1;
                load_k(k, t0), load_k(k1, t0 + 1), load_v(v, t0);
                arrive();
                write_k(k, 0), write_k(k1, 1), write_v(v, 0);
                load_k(k, t0 + 2);
                lds_barrier();
              },
              [&](int t) {
                if (t != t0) write_v(k, slot(t)), load_k(k, t + 2);
                lds_barrier();
              },
              [&](int t) { write_k(k, slot(t + 2)), load_v(k, t + 1); });
        } else {
          walk(
              [&]() {
                load_k(k, t0), load_v(v, t0);
                arrive();
                write_k(k, 0);
                load_k(k, t0 + 1);
                lds_barrier();
              },
              [&](int t) {
                write_k(k, slot(t + 1)), write_v(v, slot(t));
                load_v(v, t + 1), load_k(k, t + 2);
                lds_barrier();
              },
              [](int) {});
        }
      } else {
        // LDS is written in the order of the lanes: a lane reads the chunk that belongs in its place
        const int r0 = first_row(0) + my_row;          // first_row(i) is the same but for multiples of eight
        const uint32_t k_off = my_row * L::kRow + 16 * (my_chunk ^ (r0 & 7)), v_off = my_row * L::kRow + ((16u * my_chunk) ^ Rows<T, D, C8, 1>::v_swizzle(r0));
        auto load = [&](const void* pages, uint32_t off, const char* to, int t) {
          if (t >= t1) return;
#pragma unroll
          for (int i = 0; i < L::kChunks; ++i) dma_b128((const char*)pages + place_of(t, i), off, lds_address(to) + first_row(i) * L::kRow);
        };
        // waits until of the sides of blocks that were asked for, the last n at most are still on their way
        auto wait = [&](int n) {
          if (n >= 4) vm_wait<4 * L::kChunks>();
          else if (n == 3) vm_wait<3 * L::kChunks>();
          else if (n == 2) vm_wait<2 * L::kChunks>();
          else if (n == 1) vm_wait<L::kChunks>();
          else vm_wait<0>();
        };
        auto load_k = [&](int t) { load(a.k_pages, k_off, sh.k[slot(t)], t); };
        auto load_v = [&](int t) { load(a.v_pages, v_off, sh.v[slot(t)], t); };
        if constexpr (kRing == 4) {
          // Two blocks at a time: a wait and a barrier for every second step, with the next two blocks on their way for a step and a half (64 x 32768 tokens, 64/8 heads: 138 us
          // in all with one for every step, now 135).  Two steps read K of t + 1 and t + 2 and V of t and t + 1; the places of all before are free
          walk(
              [&]() {
                load_k(t0);
                arrive();
                load_v(t0), load_k(t0 + 1), load_v(t0 + 1), load_k(t0 + 2);
                wait(min(2, t1 - 1 - t0) + min(2, t1 - t0));
                lds_barrier();
              },
              [&](int t) {
                if ((t - t0) & 1) return;
                wait(0);
                lds_barrier();
              },
              [&](int t) {
                if ((t - t0) & 1) return;
                load_v(t + 2), load_k(t + 3), load_v(t + 3), load_k(t + 4);
              });
        } else {
          walk(
              [&]() {
                load_k(t0);
                arrive();
                load_k(t0 + 1), load_v(t0);
                wait(min(1, t1 - 1 - t0) + min(1, t1 - t0));
                lds_barrier();
              },
              [&](int t) {
                wait(0);
                lds_barrier();
              },
              [&](int t) { load_v(t + 1), load_k(t + 2); });
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
        float(*mail)[64] = reinterpret_cast<float(*)[64]>(sh.k) + (wave >> 1) * (D / 2);   // K's blocks and V's behind them
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
      // Rows leave through LDS, where each wavefront has a place: lanes hold 16 bytes of 32 rows at a time, memory takes whole rows (2.4 us for
      // the 33 MB of parts of 64 x 32768 tokens, 64/8 heads)
      lds_barrier();                                   // nobody reads a block, or another wavefront's part, any more
      if (busy && (PARTS == 1 || part == 0)) {
        int me = lane;                                 // not known to be the lane: places would be formed in front of the walk and kept in registers through it
        asm volatile("" : "+v"(me));
        const int half = me >> 5;
        const size_t slot = (size_t)slot_of_part * kTile + row, to = number == 0 ? home : slot;
        float *to_o = number == 0 ? z.p.home_o : z.p.slot_o, *to_ml = number == 0 ? z.p.home_ml : z.p.slot_ml;
        if (half == 0 && row < tile_rows) {
          to_ml[2 * to] = w.r, to_ml[2 * to + 1] = l;
          if (number == 0) z.p.home_span[home] = make_int4((int)(slot_of_part + 1), parts - 1, row, 0);
        }
        // 64 channels of the 32 rows at a time; chunk x of a row lies at x ^ (row & 15)
        char* mine_lds = sh.stage + wave * 8192;
#pragma unroll
        for (int c0 = 0; c0 < D / 32; c0 += 2) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<v4f*>(mine_lds + 256 * (me & 31) + 16 * ((8 * n + 2 * i + half) ^ (me & 15))) =
                  v4f{w.o[c0 + n][4 * i], w.o[c0 + n][4 * i + 1], w.o[c0 + n][4 * i + 2], w.o[c0 + n][4 * i + 3]};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 4 * i + (me >> 4);
            const v4f x = *reinterpret_cast<const v4f*>(mine_lds + 256 * r + 16 * ((me ^ r) & 15));
            const size_t at = (size_t)(uint32_t)__shfl((int)(uint32_t)to, r) | (size_t)(uint32_t)__shfl((int)(to >> 32), r) << 32;
            if (rows_at + r < tile_rows) *reinterpret_cast<v4f*>(to_o + at * D + 32 * c0 + 4 * (me & 15)) = x;
          }
        }
      }
    };
    if (wide) piece(std::integral_constant<int, 1>{});
    else piece(std::integral_constant<int, 2>{});
  }
}

// One workgroup per sequence and query head: joins the parts of its common and its own tokens in the order of the tokens.  Threads take four channels of
// every kParts-th part, several at a time.  Where parts are is asked for together with the lengths, whether it was written or not.
template <int D, int kShares>
__global__ void __launch_bounds__(256) prefix_merge_kernel(PagedDecodeArgs a, PrefixLaunch z) {
  constexpr int kQuads = D / 4, kParts = 256 / kQuads, kTile = tile_rows(D), kAhead = 3;
  __shared__ float2 ml[kParts];
  __shared__ __align__(16) v4f sums[kParts][kQuads];
  const int tid = threadIdx.x, quad = tid % kQuads, part = tid / kQuads;
  const size_t at = blockIdx.x;
  const int b = (int)(at / a.Hq), h = (int)(at % a.Hq), hk = h / z.own.G, gh = h % z.own.G, shift = z.own.shift, capacity = a.max_pages << shift;
  int4 span = z.p.home_span[at];
  int2 own = z.own.own_span[(size_t)b * a.Hkv + hk];
  const int len = min(capacity, max(0, a.seqlens[b])), common = z.common[b];
  if (len == 0) {
    if (part == 0) store_out4(a.out, a.out_dt, at * D + 4 * quad, 0.f, 0.f, 0.f, 0.f);
    if (a.lse != nullptr && tid == 0) a.lse[at] = -__builtin_inff();
    return;
  }
  if (common == 0) span.y = -1;
  if (len == common) own.y = -1;
  const int n1 = span.y + 1, n = n1 + own.y + 1;
  v4f o = {0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  for (int i0 = part; i0 < n; i0 += kParts * kAhead) {
    v4f x[kAhead];
    float2 y[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int i = min(n - 1, i0 + e * kParts), j = i - n1;
      const bool first = i < n1;
      const size_t row = i == 0 || j == 0 ? at : first ? (size_t)(span.x + i - 1) * kTile + span.z : (size_t)(own.x + j - 1) * z.own.G + gh;
      const float* from_o = first ? (i == 0 ? z.p.home_o : z.p.slot_o) : j == 0 ? z.own.own_o : z.own.w.part_o;
      const float* from_ml = first ? (i == 0 ? z.p.home_ml : z.p.slot_ml) : j == 0 ? z.own.own_ml : z.own.w.part_ml;
      x[e] = *reinterpret_cast<const v4f*>(from_o + row * D + 4 * quad);
      y[e] = *reinterpret_cast<const float2*>(from_ml + 2 * row);
      if (i0 + e * kParts >= n) y[e] = make_float2(-__builtin_inff(), 0.f);
    }
    float top = m;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) top = fmaxf(top, y[e].x);
    const float keep = fast_exp2(m - top);
    m = top, l *= keep, o *= keep;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const float k = fast_exp2(y[e].x - top);
      l += k * y[e].y, o += k * x[e];
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

// Workspace, all parts 16-byte aligned
struct Layout {
  size_t home_o, home_ml, home_span, slot_o, slot_ml, own_o, own_ml, own_span, part_o, part_ml, common, total;
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
  y.common = take((size_t)B * 4);
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
  z.groups = Groups{args.group_of, args.group_lens, args.n_groups};
  z.common = (int32_t*)(w + y.common), z.own.common = z.common;
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

// Where the block table has room for less than this altogether, every sequence is walked by itself: what is saved is then no more than what the tiles cost in front of and
// behind their walks.  Tiles / by itself, us, 32/8 heads of 128 channels where not said: 21.4 / 16.0 for 6 x 2000 tokens (room for 52 MB), 19.7 / 14.2 for 8 x 500 of
// 16/16 (40), 29.1 / 27.0 for 4 x 8192 (138), 23.9 / 26.4 for 16 x 2000 (139), 20.9 / 27.0 for 32 x 500 of 16/16 (159), 29.6 / 88.7 for 16 x 8192; from codes
// 31.1 / 14.7 for 6 x 2000.
constexpr long kAloneBytes = 128L << 20;
static bool by_itself(int bits, int B, int Hkv, int max_pages, int page_size, int D) {
  return (long)B * Hkv * max_pages * page_size <= kAloneBytes / (bits == 8 ? 2 * (D + 1) : 4 * D);
}

size_t paged_prefix_workspace(int bits, int B, int Hq, int Hkv, int n_groups, int max_pages, int page_size, int D) {
  if (by_itself(bits, B, Hkv, max_pages, page_size, D))
    return (bits == 8 ? paged_decode8_workspace : paged_decode_workspace)(B, Hq, Hkv, max_pages, page_size, D);
  return layout_of(bits == 8, B, Hq, Hkv, D).total;
}

void launch_paged_prefix(const PagedPrefixArgs& a, int bits, hipStream_t st) {
  if (by_itself(bits, a.d.B, a.d.Hkv, a.d.max_pages, a.d.page_size, a.d.D)) {
    if (bits == 8) launch_paged_decode8(a.d, st);
    else launch_paged_decode(a.d, st);
  } else if (bits == 8 && a.d.dt == THRIFT_F16) launch<F16, true>(a, st);
  else if (bits == 8) launch<BF16, true>(a, st);
  else if (a.d.dt == THRIFT_F16) launch<F16, false>(a, st);
  else launch<BF16, false>(a, st);
}

}  // namespace thrift
