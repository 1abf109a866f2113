// Attention over the paged key-value cache: one new token of every sequence (pq_attn_decode) and the rows of prompts (pq_attn_prefill).
#include <math.h>
#include "pq_kv.h"

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

// One wavefront per row and head: 64 tokens at a time, a lane's token scored from the row in LDS, the values summed with a lane per
// element of the head.
template <int KIND>
__global__ __launch_bounds__(64) void attn_row_kernel(kv_view v, const uint16_t* __restrict__ Q, int64_t qs, int heads, int causal, int window,
                                                      float scale, uint16_t* __restrict__ O, float* __restrict__ lse) {
  __shared__ float q[256];
  const int lane = threadIdx.x;
  const int h = blockIdx.x % heads, t = blockIdx.x / heads;
  const int b = v.row_start ? kv_find_seq(v.n_seqs, t, [&](int i) { return v.row_start[i]; }) : t;
  if (b < 0 || b >= v.n_seqs) return;
  const kv_rows r = kv_seq_rows(v, b);
  if (t < r.r0 || t >= r.r0 + r.n) return;
  const int pos = r.first + t - r.r0, kvh = h / (heads / v.n_kv_heads);
  const int cap = v.max_pages << v.page_shift;
  const int hi = min(pos < 0 ? 0 : causal ? pos + 1 : r.len, cap), lo = window > 0 ? max(0, pos + 1 - window) : 0;
  for (int d = lane; d < v.d; d += 64) q[d] = bf16_to_f32(Q[t * qs + (size_t)h * v.d + d]);
  __syncthreads();
  bool any = false;
  float m = -INFINITY, l = 0.0f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int t0 = lo & ~63; t0 < hi; t0 += 64) {
    const int p = t0 + lane, page = p < hi ? kv_page_id(v, b, p) : -1, slot = p & ((1 << v.page_shift) - 1);
    float s = -INFINITY;
    const uint8_t* base = nullptr;
    float vstep = 1.0f;
    if (p >= lo && page >= 0) {
      base = kv_head(v, page, kvh);
      float a = 0.0f;
      if constexpr (KIND == PQ_KV_INT8) {
        const int8_t* k = reinterpret_cast<const int8_t*>(base) + (size_t)slot * v.dp;
        for (int d = 0; d < v.d; ++d) a = fmaf(q[d], (float)k[d], a);
        const float* steps = reinterpret_cast<const float*>(base + 2 * (size_t)v.part_bytes);
        a *= steps[slot];
        vstep = steps[(1 << v.page_shift) + slot];
      } else {
        const uint16_t* k = reinterpret_cast<const uint16_t*>(base) + (size_t)slot * v.dp;
        for (int d = 0; d < v.d; ++d) a = fmaf(q[d], bf16_to_f32(k[d]), a);
      }
      s = a * scale;
    }
    const uint64_t seen = __ballot(base != nullptr);
    if (!seen) continue;
    any = true;
    const float mt = fmaxf(m, wave_max(s)), mx = mt == -INFINITY ? 0.0f : mt;
    const float keep = expf(m - mx), pr = base ? expf(s - mx) : 0.0f;
    l = l * keep + wave_sum(pr);
    m = mt;
    for (int i = 0; i < 4; ++i) acc[i] *= keep;
    for (int j = 0; j < 64; ++j) {
      if (!((seen >> j) & 1)) continue;
      const float pj = __shfl(pr, j, 64) * __shfl(vstep, j, 64);
      const int sj = (t0 + j) & ((1 << v.page_shift) - 1);
      const uint8_t* bj = reinterpret_cast<const uint8_t*>((uintptr_t)__shfl((unsigned long long)(uintptr_t)base, j, 64)) + v.part_bytes;
      for (int i = 0; i < 4; ++i) {
        const int d = lane + 64 * i;
        if (d >= v.d) break;
        const size_t at = ((size_t)(sj / KV_BLOCK) * v.dp + d) * KV_BLOCK + sj % KV_BLOCK;
        const float x = KIND == PQ_KV_INT8 ? (float)reinterpret_cast<const int8_t*>(bj)[at] : bf16_to_f32(reinterpret_cast<const uint16_t*>(bj)[at]);
        acc[i] = fmaf(pj, x, acc[i]);
      }
    }
  }
  for (int i = 0; i < 4; ++i) {
    const int d = lane + 64 * i;
    if (d < v.d) O[((size_t)t * heads + h) * v.d + d] = f32_to_bf16(any ? acc[i] / l : 0.0f);
  }
  if (lse && lane == 0) lse[(size_t)t * heads + h] = any ? m + logf(l) : -INFINITY;
}

int check_attn(const pq_attn_desc* d) {
  PQ_REQUIRE(d != nullptr, PQ_ERR_BAD_ARG, "desc is NULL");
  if (int e = pq_kv_check(&d->kv)) return e;
  PQ_REQUIRE(d->n_heads > 0 && d->n_heads % d->kv.n_kv_heads == 0, PQ_ERR_BAD_ARG, "n_heads=%d must be a multiple of n_kv_heads=%d",
             d->n_heads, d->kv.n_kv_heads);
  PQ_REQUIRE(d->window >= 0 && d->max_len >= 0, PQ_ERR_BAD_ARG, "negative window=%d or max_len=%d", d->window, d->max_len);
  PQ_REQUIRE(d->window == 0 || d->causal, PQ_ERR_BAD_ARG, "a window needs causal rows");
  PQ_REQUIRE(isfinite(d->scale), PQ_ERR_BAD_ARG, "scale is not finite");
  return PQ_OK;
}

int check_attn_call(const pq_attn_desc* d, const void* Q, int64_t qs, int T, const void* cache, size_t cache_bytes, const int32_t* lens,
                    const int32_t* table, const void* O) {
  PQ_REQUIRE(Q && O && cache && lens && table, PQ_ERR_BAD_ARG, "NULL buffer");
  PQ_REQUIRE(qs >= (int64_t)d->n_heads * d->kv.d_head && qs % 2 == 0, PQ_ERR_SHAPE, "row stride %lld must be even and at least n_heads * d_head = %lld",
             (long long)qs, (long long)d->n_heads * d->kv.d_head);
  PQ_REQUIRE((((uintptr_t)Q | (uintptr_t)O | (uintptr_t)cache) & 15) == 0, PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  PQ_REQUIRE(cache_bytes >= pq_kv_cache_bytes(&d->kv), PQ_ERR_WORKSPACE, "cache %zu < %zu bytes", cache_bytes, pq_kv_cache_bytes(&d->kv));
  PQ_REQUIRE((int64_t)T * d->n_heads <= 0x7fffffff, PQ_ERR_SHAPE, "%d rows of %d heads are too many for one call", T, d->n_heads);
  return PQ_OK;
}

int launch_rows(const pq_attn_desc* d, const kv_view& v, const void* Q, int64_t qs, int causal, void* O, float* lse, int label, hipStream_t s) {
  pq_prof_scope prof(label, s);
  const unsigned grid = (unsigned)v.T * (unsigned)d->n_heads;
  if (d->kv.kv_kind == PQ_KV_INT8)
    attn_row_kernel<PQ_KV_INT8><<<grid, 64, 0, s>>>(v, (const uint16_t*)Q, qs, d->n_heads, causal, d->window, d->scale, (uint16_t*)O, lse);
  else
    attn_row_kernel<PQ_KV_BF16><<<grid, 64, 0, s>>>(v, (const uint16_t*)Q, qs, d->n_heads, causal, d->window, d->scale, (uint16_t*)O, lse);
  PQ_CHECK_LAUNCH("attn_row_kernel");
  return PQ_OK;
}

}  // namespace

extern "C" size_t pq_attn_decode_workspace_bytes(const pq_attn_desc* d) {
  if (check_attn(d)) return 0;
  return 256;
}

extern "C" int pq_attn_decode(const pq_attn_desc* d, const void* Q, int64_t q_stride, const void* cache, size_t cache_bytes,
                              const int32_t* lens, const int32_t* page_table, void* O, float* lse, void* workspace, size_t workspace_bytes,
                              void* stream) {
  if (int e = check_attn(d)) return e;
  const int T = d->kv.n_seqs;
  if (T == 0) return PQ_OK;
  if (int e = check_attn_call(d, Q, q_stride, T, cache, cache_bytes, lens, page_table, O)) return e;
  PQ_REQUIRE(workspace, PQ_ERR_BAD_ARG, "NULL workspace");
  PQ_REQUIRE(((uintptr_t)workspace & 15) == 0, PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  PQ_REQUIRE(workspace_bytes >= pq_attn_decode_workspace_bytes(d), PQ_ERR_WORKSPACE, "workspace %zu < %zu", workspace_bytes,
             pq_attn_decode_workspace_bytes(d));
  const kv_view v = pq_kv_make_view(d->kv, cache, nullptr, lens, page_table, T);
  return launch_rows(d, v, Q, q_stride, 1, O, lse, PQP_ATTN_DECODE, (hipStream_t)stream);
}

extern "C" int pq_attn_prefill(const pq_attn_desc* d, const void* Q, int64_t q_stride, int32_t T, const int32_t* row_start, const void* cache,
                               size_t cache_bytes, const int32_t* lens, const int32_t* page_table, void* O, float* lse, void* stream) {
  if (int e = check_attn(d)) return e;
  PQ_REQUIRE(T >= 0, PQ_ERR_BAD_ARG, "T=%d is negative", T);
  if (T == 0 || d->kv.n_seqs == 0) return PQ_OK;
  if (int e = check_attn_call(d, Q, q_stride, T, cache, cache_bytes, lens, page_table, O)) return e;
  const kv_view v = pq_kv_make_view(d->kv, cache, row_start, lens, page_table, T);
  return launch_rows(d, v, Q, q_stride, d->causal, O, lse, PQP_ATTN_PREFILL, (hipStream_t)stream);
}
