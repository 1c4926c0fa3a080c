// Host-side launch interface of rotary positions and of the paged cache in 16 and 8 bits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "thrift.h"

namespace thrift {

constexpr int kRopeMaxDim = 1024;         // channels of a head

struct RopeSide {             // the query heads or the key heads of a call
  const uint16_t* x;
  uint16_t* y;
  long xb, xh, xn, yb, yh, yn;   // elements from one batch entry, head and token to the next
  int heads;                  // 0: the side is absent
};
struct RopeArgs {
  RopeSide side[2];
  const int32_t* positions;   // nullable: token n is at position n
  const double* freqs;        // [rot/2] radians per position
  long positions_stride;
  int B, N, D, rot, layout;
  float gain, sign;           // sign -1: the transposed rotation
};
void launch_rope(const RopeArgs& a, thrift_dtype dt, hipStream_t st);

constexpr int kMapMaxSeqs = 4096;         // sequences whose prefix sums one workgroup holds in LDS
struct PageMapArgs {
  const int32_t* seqlens;     // [B]
  const int32_t* new_lens;    // [B]
  int32_t* table;             // [B,max_pages]
  const int32_t* free_pages;  // [free_capacity]
  const int32_t* free_count;  // [1]
  int32_t* slots;             // [rows]
  int32_t* positions;         // [rows]
  int32_t* starts;            // [B+1]
  int32_t* seqlens_out;       // [B]
  int32_t* free_count_out;    // [1]
  int B, page_size, n_pages, max_pages, free_capacity, rows;
};
void launch_page_map(const PageMapArgs& a, hipStream_t st);

struct PageReleaseArgs {
  const int32_t* seqlens;
  const int32_t* drop;
  const int32_t* table;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* seqlens_out;
  int32_t* free_count_out;
  int B, page_size, n_pages, max_pages, free_capacity;
};
void launch_page_release(const PageReleaseArgs& a, hipStream_t st);

struct PagedAppendArgs {
  const uint16_t *q, *k, *v;  // q nullable
  uint16_t* q_out;            // [T,Hq,D]
  long qt, qh, kt, kh, vt, vh;   // elements from one token and head to the next
  const int32_t* slots;       // [T]
  const int32_t* positions;   // [T]
  const double* freqs;
  uint16_t* k_pages;          // [n_pages,Hkv,page_size,D]
  uint16_t* v_pages;
  int T, Hq, Hkv, D, rot, layout, n_pages, page_size;
  float gain;
};
void launch_paged_append(const PagedAppendArgs& a, thrift_dtype dt, hipStream_t st);

struct PagedAppend8Args {
  PagedAppendArgs in;         // but for its pages
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;   // [n_pages,Hkv,page_size,D] and [n_pages,Hkv,page_size]
};
void launch_paged_append8(const PagedAppend8Args& a, thrift_dtype dt, hipStream_t st);

struct PagedReadArgs {
  const void *k_pages, *v_pages;                  // 16-bit elements, or codes
  const uint8_t *k_scales, *v_scales;             // nullptr: 16-bit pages
  const int32_t* table;       // [B,max_pages]
  const int32_t* first;       // nullable [B]
  const int32_t* seqlens;     // [B]
  uint16_t *k_out, *v_out;    // [B,Hkv,N,D]
  int B, Hkv, N, D, n_pages, max_pages, page_size;
};
void launch_paged_read(const PagedReadArgs& a, thrift_dtype dt, hipStream_t st);   // dt: of what 8-bit pages become

struct PagedDecodeArgs {
  const uint16_t* q;          // [B,Hq,D]
  const void* k_pages;        // [n_pages,Hkv,page_size,D] 16-bit elements, or codes
  const void* v_pages;
  const uint8_t* k_scales;    // [n_pages,Hkv,page_size] of codes
  const uint8_t* v_scales;
  const int32_t* table;       // [B,max_pages]
  const int32_t* seqlens;     // [B]
  void* out;                  // [B,Hq,D]
  float* lse;                 // nullable [B,Hq]
  void* workspace;
  int B, Hq, Hkv, D, n_pages, max_pages, page_size;
  float scale;                // softmax scale (already defaulted)
  thrift_dtype dt, out_dt;
};
size_t paged_decode_workspace(int B, int Hq, int Hkv, int max_pages, int page_size, int D);   // 0: none is needed
void launch_paged_decode(const PagedDecodeArgs& a, hipStream_t st);
size_t paged_decode8_workspace(int B, int Hq, int Hkv, int max_pages, int page_size, int D);
void launch_paged_decode8(const PagedDecodeArgs& a, hipStream_t st);

struct PagedPrefixArgs {
  PagedDecodeArgs d;
  const int32_t* group_of;    // [B]
  const int32_t* group_lens;  // [n_groups]
  int n_groups;
};
size_t paged_prefix_workspace(int bits, int B, int Hq, int Hkv, int n_groups, int max_pages, int page_size, int D);
void launch_paged_prefix(const PagedPrefixArgs& a, int bits, hipStream_t st);

}  // namespace thrift
