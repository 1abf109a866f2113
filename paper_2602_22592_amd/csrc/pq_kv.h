// The paged key-value cache on the device: where a token's keys, values and steps lie, and which rows belong to which sequence.
#pragma once
#include "pq_internal.h"

// Blocks of 16 tokens: a page's values are stored [token / 16][Dp][token % 16].  With the tokens innermost the values are the transposed
// operand that the matrix instructions of P V want (their contraction runs over tokens), in pieces of 16 bytes for INT8; the keys, whose
// contraction runs over the head, are stored row by row.
constexpr int KV_BLOCK = 16;

struct kv_view {
  uint8_t* cache;
  const int32_t* table;        // [n_seqs][max_pages]
  const int32_t* lens;         // [n_seqs]
  const int32_t* row_start;    // [n_seqs + 1] or NULL: row b is the one row of sequence b
  size_t head_bytes;           // of one head of one page
  int n_pages, n_seqs, max_pages, page_shift, n_kv_heads, d, dp, T;
  int part_bytes;              // keys (or values) of one head of one page; the steps of both follow the values
};

// Host side (pq_kv.hip): the checks of a descriptor, and the device's view of it (dp: d_head up to a multiple of 32).
int pq_kv_check(const pq_kv_desc* d);
kv_view pq_kv_make_view(const pq_kv_desc& d, const void* cache, const int32_t* row_start, const int32_t* lens, const int32_t* table, int T);

__device__ __forceinline__ int kv_page_id(const kv_view& v, int b, int pos) {   // -1: no such page
  const int i = pos >> v.page_shift;
  if (pos < 0 || i >= v.max_pages) return -1;
  const int id = v.table[(size_t)b * v.max_pages + i];
  return (unsigned)id < (unsigned)v.n_pages ? id : -1;
}
__device__ __forceinline__ uint8_t* kv_head(const kv_view& v, int page, int h) {
  return v.cache + ((size_t)page * v.n_kv_heads + h) * v.head_bytes;
}

struct kv_rows { int r0, n, len, first; };   // rows r0 .. r0 + n - 1 of sequence b sit at positions first .. (first may be negative)
__device__ __forceinline__ kv_rows kv_seq_rows(const kv_view& v, int b) {
  kv_rows r;
  if (v.row_start) {
    r.r0 = min(max(v.row_start[b], 0), v.T);
    r.n = min(max(v.row_start[b + 1], r.r0), v.T) - r.r0;
  } else {
    r.r0 = b;
    r.n = b < v.T ? 1 : 0;
  }
  r.len = min(max(v.lens[b], 0), (1 << 30) + r.n);   // (beyond 2^30 no table has a page; T <= 2^29: no position overflows)
  r.first = r.len - r.n;
  return r;
}
// The last sequence b with start(b) <= x, start non-decreasing with start(0) <= x (-1 if there is none): the wavefront looks at 64
// entries a step, so that 4096 sequences take two dependent reads.
template <typename F>
__device__ __forceinline__ int kv_find_seq(int n_seqs, int x, F start) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = n_seqs;
  while (n > 0) {
    const int step = (n + 63) >> 6;
    const int i = lane * step;
    const uint64_t hit = __ballot(i < n && start(lo + i) <= x);
    if (hit == 0) return lo - 1;
    const int last = 63 - __builtin_clzll(hit);      // start is non-decreasing: the hits are a prefix (for any other input: in range)
    lo += last * step;
    if (step == 1) return lo;
    n = min(step, n - last * step);
  }
  return -1;
}

// The same with the sequence's rows; start(first row of a sequence, its number).  Up to 64 sequences: each lane has one, and what belongs to the
// one that is found comes from its lane instead of a second read behind the first.
template <typename F>
__device__ __forceinline__ int kv_find_rows(const kv_view& v, int x, kv_rows& r, F start) {
  if (v.n_seqs > 64) {
    const int b = kv_find_seq(v.n_seqs, x, [&](int i) { return start(v.row_start ? min(max(v.row_start[i], 0), v.T) : min(i, v.T), i); });
    if (b >= 0) r = kv_seq_rows(v, b);
    return b;
  }
  const int lane = threadIdx.x & 63;
  const kv_rows mine = kv_seq_rows(v, min(lane, v.n_seqs - 1));
  const uint64_t hit = __ballot(lane < v.n_seqs && start(min(mine.r0, v.T), lane) <= x);
  if (hit == 0) return -1;
  const int b = 63 - __builtin_clzll(hit);
  r.r0 = __builtin_amdgcn_readlane(mine.r0, b);
  r.n = __builtin_amdgcn_readlane(mine.n, b);
  r.len = __builtin_amdgcn_readlane(mine.len, b);
  r.first = __builtin_amdgcn_readlane(mine.first, b);
  return b;
}

// AbsMax INT8 of one row of a head: the code of pq_quant_act, rint(fl32(x gamma)) between -128 and 127, in the low byte of the result's bits (1.5 2^23
// + x is rounded to a whole number, ties to even; |x gamma| < 128.5 by gamma's definition, so that only 128 has to be held back).
__device__ __forceinline__ float kv_code(float x, float gamma) { return fminf(x * gamma, 127.0f) + 12582912.0f; }
// gamma and step from the largest |x| as fp32 bits (the bits of infinities and NaN are above every finite value's): a row that holds
// one of them has the step NaN and reads back as NaN.
__device__ __forceinline__ void kv_scales(uint32_t amax_bits, float& gamma, float& step) {
  const float amax = fmaxf(__uint_as_float(amax_bits), 1e-5f);
  gamma = 128.0f / amax;
  step = amax_bits >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : amax * 0.0078125f;
}
