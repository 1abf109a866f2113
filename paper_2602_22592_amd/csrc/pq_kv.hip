// The paged key-value cache: rows quantised (or rounded to 16 bits) as they are written, and read back.
#include "pq_kv.h"

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

template <typename T, int KIND>
__global__ __launch_bounds__(256) void kv_write_kernel(kv_view v, const T* __restrict__ K, const T* __restrict__ V, int64_t ks, int64_t vs) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int which = (int)(unit & 1), h = (int)((unit >> 1) % v.n_kv_heads);
  const int64_t t = (unit >> 1) / v.n_kv_heads;
  if (t >= v.T) return;
  const int b = v.row_start ? kv_find_seq(v.n_seqs, (int)t, [&](int i) { return v.row_start[i]; }) : (int)t;
  if (b < 0 || b >= v.n_seqs) return;
  const kv_rows r = kv_seq_rows(v, b);
  if (t < r.r0 || t >= r.r0 + r.n) return;
  const int pos = r.first + (int)t - r.r0;
  const int page = kv_page_id(v, b, pos);
  if (page < 0) return;
  const int slot = pos & ((1 << v.page_shift) - 1);
  const T* src = which ? V + t * vs + (size_t)h * v.d : K + t * ks + (size_t)h * v.d;
  float x[4];
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = lane + 64 * i;
    x[i] = d < v.d ? io_traits<T>::load(src, d) : 0.0f;
    amax = max(amax, __float_as_uint(x[i]) & 0x7fffffffu);
  }
  for (int o = 32; o > 0; o >>= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));
  uint8_t* base = kv_head(v, page, h);
  float gamma = 0.0f, step = 0.0f;
  if constexpr (KIND == PQ_KV_INT8) {
    kv_scales(amax, gamma, step);
    if (lane == 0) reinterpret_cast<float*>(base + 2 * (size_t)v.part_bytes)[(which << v.page_shift) + slot] = step;
  }
  uint8_t* part = base + (which ? v.part_bytes : 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = lane + 64 * i;
    if (d >= v.dp) continue;
    const size_t at = which ? ((size_t)(slot / KV_BLOCK) * v.dp + d) * KV_BLOCK + slot % KV_BLOCK : (size_t)slot * v.dp + d;
    if constexpr (KIND == PQ_KV_INT8) reinterpret_cast<int8_t*>(part)[at] = (int8_t)kv_code(x[i], gamma);
    else reinterpret_cast<uint16_t*>(part)[at] = f32_to_bf16(x[i]);
  }
}

template <typename T, int KIND>
__global__ __launch_bounds__(256) void kv_read_kernel(kv_view v, T* __restrict__ K, T* __restrict__ V, int64_t ks, int64_t vs) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int which = (int)(unit & 1), h = (int)((unit >> 1) % v.n_kv_heads);
  const int64_t t = (unit >> 1) / v.n_kv_heads;
  if (t >= v.T) return;
  T* dst = which ? V : K;
  if (!dst) return;
  const int b = v.row_start ? kv_find_seq(v.n_seqs, (int)t, [&](int i) { return v.row_start[i]; }) : (int)t;
  if (b < 0 || b >= v.n_seqs) return;
  const kv_rows r = kv_seq_rows(v, b);
  if (t < r.r0 || t >= r.r0 + r.n) return;
  const int pos = r.first + (int)t - r.r0;
  const int page = kv_page_id(v, b, pos);
  const int slot = pos & ((1 << v.page_shift) - 1);
  dst += t * (which ? vs : ks) + (size_t)h * v.d;
  const uint8_t* base = page < 0 ? nullptr : kv_head(v, page, h);
  const uint8_t* part = base + (which ? v.part_bytes : 0);
  for (int d = lane; d < v.d; d += 64) {
    float x = 0.0f;
    if (page >= 0) {
      const size_t at = which ? ((size_t)(slot / KV_BLOCK) * v.dp + d) * KV_BLOCK + slot % KV_BLOCK : (size_t)slot * v.dp + d;
      if constexpr (KIND == PQ_KV_INT8)
        x = (float)reinterpret_cast<const int8_t*>(part)[at] *
            reinterpret_cast<const float*>(base + 2 * (size_t)v.part_bytes)[(which << v.page_shift) + slot];
      else x = bf16_to_f32(reinterpret_cast<const uint16_t*>(part)[at]);
    }
    io_traits<T>::store(dst, d, x);
  }
}

}  // namespace

// ---------------------------------------------------------------------------------------------
int pq_kv_check(const pq_kv_desc* d) {
  PQ_REQUIRE(d != nullptr, PQ_ERR_BAD_ARG, "desc is NULL");
  PQ_REQUIRE(d->kv_kind == PQ_KV_BF16 || d->kv_kind == PQ_KV_INT8, PQ_ERR_BAD_ARG, "unknown kv_kind %d", d->kv_kind);
  PQ_REQUIRE(d->n_kv_heads > 0 && d->n_pages > 0 && d->max_pages > 0 && d->n_seqs >= 0 && d->d_head > 0, PQ_ERR_BAD_ARG,
             "negative or zero size (n_kv_heads=%d d_head=%d n_pages=%d n_seqs=%d max_pages=%d)", d->n_kv_heads, d->d_head, d->n_pages,
             d->n_seqs, d->max_pages);
  PQ_REQUIRE(d->d_head % 2 == 0 && d->d_head <= 256, PQ_ERR_SHAPE, "d_head=%d must be even and at most 256", d->d_head);
  PQ_REQUIRE(d->page_tokens >= 16 && d->page_tokens <= 1024 && (d->page_tokens & (d->page_tokens - 1)) == 0, PQ_ERR_SHAPE,
             "page_tokens=%d must be a power of two in 16..1024", d->page_tokens);
  PQ_REQUIRE(d->n_kv_heads <= 65535, PQ_ERR_SHAPE, "n_kv_heads=%d exceeds 65535", d->n_kv_heads);
  PQ_REQUIRE((int64_t)d->max_pages * d->page_tokens <= (1 << 30), PQ_ERR_SHAPE, "max_pages=%d of %d tokens exceed 2^30 tokens a sequence",
             d->max_pages, d->page_tokens);
  return PQ_OK;
}

kv_view pq_kv_make_view(const pq_kv_desc& d, const void* cache, const int32_t* row_start, const int32_t* lens, const int32_t* table, int T) {
  kv_view v;
  v.cache = (uint8_t*)cache; v.table = table; v.lens = lens; v.row_start = row_start;
  v.n_pages = d.n_pages; v.n_seqs = d.n_seqs; v.max_pages = d.max_pages; v.n_kv_heads = d.n_kv_heads;
  v.page_shift = __builtin_ctz((unsigned)d.page_tokens);
  v.d = d.d_head; v.dp = (d.d_head + 31) / 32 * 32; v.T = T;
  v.part_bytes = d.page_tokens * v.dp * (d.kv_kind == PQ_KV_INT8 ? 1 : 2);
  v.head_bytes = 2 * (size_t)v.part_bytes + (d.kv_kind == PQ_KV_INT8 ? 8 * (size_t)d.page_tokens : 0);
  return v;
}

extern "C" size_t pq_kv_cache_bytes(const pq_kv_desc* d) {
  if (pq_kv_check(d)) return 0;
  return pq_kv_make_view(*d, nullptr, nullptr, nullptr, nullptr, 0).head_bytes * d->n_kv_heads * (size_t)d->n_pages;
}

// What pq_kv_write and pq_kv_read check alike.
static int kv_check_call(const pq_kv_desc* d, const void* K, const void* V, int dtype, int T, int64_t ks, int64_t vs, const int32_t* lens,
                         const int32_t* table, const void* cache, size_t cache_bytes) {
  if (int e = pq_kv_check(d)) return e;
  PQ_REQUIRE(dtype == PQ_F32 || dtype == PQ_BF16, PQ_ERR_DTYPE, "dtype %d is not PQ_F32 or PQ_BF16", dtype);
  PQ_REQUIRE(T >= 0, PQ_ERR_BAD_ARG, "T=%d is negative", T);
  if (T == 0 || d->n_seqs == 0) return PQ_OK;
  PQ_REQUIRE(lens && table && cache, PQ_ERR_BAD_ARG, "NULL buffer");
  const int64_t row = (int64_t)d->n_kv_heads * d->d_head;
  PQ_REQUIRE((!K || (ks >= row && ks % 2 == 0)) && (!V || (vs >= row && vs % 2 == 0)), PQ_ERR_SHAPE,
             "row strides %lld and %lld must be even and at least n_kv_heads * d_head = %lld", (long long)ks, (long long)vs, (long long)row);
  PQ_REQUIRE((((uintptr_t)K | (uintptr_t)V | (uintptr_t)cache) & 15) == 0, PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  PQ_REQUIRE(cache_bytes >= pq_kv_cache_bytes(d), PQ_ERR_WORKSPACE, "cache %zu < %zu bytes", cache_bytes, pq_kv_cache_bytes(d));
  PQ_REQUIRE(((int64_t)T * d->n_kv_heads * 2 + 3) / 4 <= 0x7fffffff, PQ_ERR_SHAPE, "T=%d rows of %d heads are too many for one call", T,
             d->n_kv_heads);
  return PQ_OK;
}

extern "C" int pq_kv_write(const pq_kv_desc* d, const void* K, const void* V, int32_t dtype, int32_t T, int64_t k_stride, int64_t v_stride,
                           const int32_t* row_start, const int32_t* lens, const int32_t* page_table, void* cache, size_t cache_bytes,
                           void* stream) {
  if (int e = kv_check_call(d, K, V, dtype, T, k_stride, v_stride, lens, page_table, cache, cache_bytes)) return e;
  if (T == 0 || d->n_seqs == 0) return PQ_OK;
  PQ_REQUIRE(K && V, PQ_ERR_BAD_ARG, "NULL buffer");
  const kv_view v = pq_kv_make_view(*d, cache, row_start, lens, page_table, T);
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_KV, s);
  const unsigned grid = (unsigned)(((int64_t)T * d->n_kv_heads * 2 + 3) / 4);
  const bool i8 = d->kv_kind == PQ_KV_INT8;
  if (dtype == PQ_F32) {
    if (i8) kv_write_kernel<float, PQ_KV_INT8><<<grid, 256, 0, s>>>(v, (const float*)K, (const float*)V, k_stride, v_stride);
    else kv_write_kernel<float, PQ_KV_BF16><<<grid, 256, 0, s>>>(v, (const float*)K, (const float*)V, k_stride, v_stride);
  } else {
    if (i8) kv_write_kernel<uint16_t, PQ_KV_INT8><<<grid, 256, 0, s>>>(v, (const uint16_t*)K, (const uint16_t*)V, k_stride, v_stride);
    else kv_write_kernel<uint16_t, PQ_KV_BF16><<<grid, 256, 0, s>>>(v, (const uint16_t*)K, (const uint16_t*)V, k_stride, v_stride);
  }
  PQ_CHECK_LAUNCH("kv_write_kernel");
  return PQ_OK;
}

extern "C" int pq_kv_read(const pq_kv_desc* d, const void* cache, size_t cache_bytes, const int32_t* row_start, const int32_t* lens,
                          const int32_t* page_table, int32_t T, void* K, void* V, int32_t dtype, int64_t k_stride, int64_t v_stride,
                          void* stream) {
  if (int e = kv_check_call(d, K, V, dtype, T, k_stride, v_stride, lens, page_table, cache, cache_bytes)) return e;
  if (T == 0 || d->n_seqs == 0) return PQ_OK;
  PQ_REQUIRE(K || V, PQ_ERR_BAD_ARG, "neither keys nor values are asked for");
  const kv_view v = pq_kv_make_view(*d, cache, row_start, lens, page_table, T);
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_KV, s);
  const unsigned grid = (unsigned)(((int64_t)T * d->n_kv_heads * 2 + 3) / 4);
  const bool i8 = d->kv_kind == PQ_KV_INT8;
  if (dtype == PQ_F32) {
    if (i8) kv_read_kernel<float, PQ_KV_INT8><<<grid, 256, 0, s>>>(v, (float*)K, (float*)V, k_stride, v_stride);
    else kv_read_kernel<float, PQ_KV_BF16><<<grid, 256, 0, s>>>(v, (float*)K, (float*)V, k_stride, v_stride);
  } else {
    if (i8) kv_read_kernel<uint16_t, PQ_KV_INT8><<<grid, 256, 0, s>>>(v, (uint16_t*)K, (uint16_t*)V, k_stride, v_stride);
    else kv_read_kernel<uint16_t, PQ_KV_BF16><<<grid, 256, 0, s>>>(v, (uint16_t*)K, (uint16_t*)V, k_stride, v_stride);
  }
  PQ_CHECK_LAUNCH("kv_read_kernel");
  return PQ_OK;
}
