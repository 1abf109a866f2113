// The paged key-value cache: rows quantised (or rounded to 16 bits) as they are written, and read back.
#include <type_traits>
#include "pq_kv.h"

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

// Sixteen values a lane, each the maximum over the wavefront's rows of 16 lanes: every exchange halves what a lane carries, lane l ends
// with value l % 16 in v[0].
template <int N, int OFF>
__device__ __forceinline__ void max_transposed(uint32_t* v, int lane) {
  const bool up = (lane & OFF) != 0;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const uint32_t send = up ? v[i] : v[i + N / 2], keep = up ? v[i + N / 2] : v[i];
    v[i] = max(keep, (uint32_t)__shfl_xor((int)send, OFF, 64));
  }
  if constexpr (N > 2) max_transposed<N / 2, OFF / 2>(v, lane);
}

// What a wavefront of both kernels works on: the keys or the values of one block of 16 tokens of a sequence and of 1, 2 or 4 heads (LPH lanes
// a head, E pairs of elements a lane).  Tokens s0 .. s1 - 1 of the block are rows of the call, from row t0 on.
struct kv_unit { int which, head, page, slot, s0, s1; int64_t t0; };
template <int LPH>
__device__ __forceinline__ bool kv_find_unit(const kv_view& v, kv_unit& u) {
  constexpr int HPU = 64 / LPH;
  const int lane = threadIdx.x & 63, groups = (v.n_kv_heads + HPU - 1) / HPU;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  u.which = (int)(unit & 1);
  u.head = (int)((unit >> 1) % groups) * HPU + lane / LPH;
  const int64_t vb = (unit >> 1) / groups;
  // Virtual blocks: sequence b owns those from floor(first row / 16) + 2 b, which are at least as many as its rows touch.
  int b = (int)vb, j = 0;
  kv_rows r;
  if (v.row_start) {
    auto start = [&](int r0, int i) { return (r0 >> 4) + 2 * i; };
    if (vb > 0x7fffffff) return false;
    b = kv_find_rows(v, (int)vb, r, start);
    if (b < 0) return false;
    j = (int)vb - start(r.r0, b);
  } else {
    if (vb >= v.n_seqs) return false;
    r = kv_seq_rows(v, b);
  }
  if (r.n == 0) return false;
  const int from = max(r.first, 0), block = (from >> 4) + j, p0 = block << 4;
  // rows at negative positions belong to no block: the sequence's first virtual block has them too (they read back as zeros)
  u.s0 = j == 0 ? min(r.first, 0) + (from - p0) : 0;
  u.s1 = (int)min((int64_t)16, (int64_t)r.len - p0);
  if (u.s1 <= u.s0) return false;
  u.t0 = (int64_t)r.r0 + (p0 + u.s0 - r.first);
  u.page = kv_page_id(v, b, p0);
  u.slot = p0 & ((1 << v.page_shift) - 1);
  return true;
}

template <typename T> using raw_pair_t = std::conditional_t<std::is_same_v<T, float>, float2, uint32_t>;    // two neighbours as they lie in memory
__device__ __forceinline__ float2 pair_of(float2 w) { return w; }
__device__ __forceinline__ float2 pair_of(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
// Past the L2: a wavefront writes whole lines that nobody of this kernel reads, and lines left dirty are written back behind the kernel's end,
// on time of their own (16 ragged histories of up to 8192 tokens, 8 heads of 128: 52.5 us with ordinary stores, 34.6 with these; not for the
// cache's own pieces of 2 to 32 bytes a lane: four prompts of 2048 tokens written and read 45.8 us with ordinary stores there, 53.2 with these).
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void store_pair(float* p, float x, float y) { __builtin_nontemporal_store(f32x2_t{x, y}, reinterpret_cast<f32x2_t*>(p)); }
__device__ __forceinline__ void store_pair(uint16_t* p, float x, float y) { __builtin_nontemporal_store(pack_bf16x2(x, y), reinterpret_cast<uint32_t*>(p)); }

// Bound by memory: every element is read once and written once.  (Four prompts of 2048 tokens, 32 heads of 64, bf16 to INT8: 102 MB in 26 us, 3.9
// TB/s; nine ragged ones in fp32 to bf16, 32 heads of 90: 26 us.  16 tokens of an element at a time because they are one piece of the values'
// layout: written and read back token by token, with stores of 1 and 2 bytes, the same prompts took 358 us, so 46.)
// A lane holds two neighbouring elements (four beyond 128: E = 2) of all 16 tokens: rows are read a pair of elements a lane, a token's maximum
// is taken over the lanes for all 16 tokens together, keys leave token by token and values, 16 tokens of an element side by side, as
// 16-byte pieces.  A block that the call does not fill is written token by token, so that its other tokens stay as they are.
template <typename T, int KIND, int LPH, int E>
__global__ __launch_bounds__(256) void kv_write_kernel(kv_view v, const T* __restrict__ K, const T* __restrict__ V, int64_t ks, int64_t vs) {
  constexpr bool I8 = KIND == PQ_KV_INT8;
  const int lane = threadIdx.x & 63;
  kv_unit u;
  if (!kv_find_unit<LPH>(v, u)) return;
  u.t0 -= u.s0;                                     // (row of the block's first token)
  const int s0 = max(u.s0, 0), s1 = u.s1;
  const int d0 = 2 * (lane % LPH);
  const bool head_ok = u.head < v.n_kv_heads;
  const int64_t stride = u.which ? vs : ks;
  const T* src = (u.which ? V : K) + (size_t)(head_ok ? u.head : 0) * v.d;
  // Every load is made, of a row and an element that are there (a load in a branch of its own would be waited for at the branch's end, one
  // after the other: four prompts of 2048 tokens 36 us, so 26).
  raw_pair_t<T> raw[16][E];
#pragma unroll
  for (int s = 0; s < 16; ++s)
#pragma unroll
    for (int e = 0; e < E; ++e)
      raw[s][e] = *reinterpret_cast<const raw_pair_t<T>*>(src + (u.t0 + min(max(s, s0), s1 - 1)) * stride + min(d0 + 128 * e, v.d - 2));
  float2 x[16][E];
  uint32_t top[16];
#pragma unroll
  for (int s = 0; s < 16; ++s)
#pragma unroll
    for (int e = 0; e < E; ++e) x[s][e] = d0 + 128 * e < v.d ? pair_of(raw[s][e]) : make_float2(0.f, 0.f);
  if (u.page < 0) return;                           // (looked at with the rows under way)
  uint8_t* base = kv_head(v, u.page, head_ok ? u.head : 0);
  if constexpr (I8) {
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      top[s] = 0;
#pragma unroll
      for (int e = 0; e < E; ++e)
        top[s] = max(top[s], max(__float_as_uint(x[s][e].x) & 0x7fffffffu, __float_as_uint(x[s][e].y) & 0x7fffffffu));
    }
    max_transposed<16, 8>(top, lane);
    uint32_t most = top[0];
    if constexpr (LPH >= 32) most = max(most, (uint32_t)__shfl_xor((int)most, 16, 64));
    if constexpr (LPH >= 64) most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
    float gamma, step;
    kv_scales(most, gamma, step);
    const int s = lane & 15;
    if (head_ok && lane % LPH < 16 && s >= s0 && s < s1)
      reinterpret_cast<float*>(base + 2 * (size_t)v.part_bytes)[(u.which << v.page_shift) + u.slot + s] = step;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float g = __shfl(gamma, (lane & ~(LPH - 1)) | i, 64);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[i][e].x = kv_code(x[i][e].x, g);
        x[i][e].y = kv_code(x[i][e].y, g);
      }
    }
  }
  if (!head_ok) return;
  // the two stored numbers of a token, in the low and the high half of a word
  auto two = [&](int s, int e) {
    if constexpr (I8) return __builtin_amdgcn_perm(__float_as_uint(x[s][e].y), __float_as_uint(x[s][e].x), 0x0c040c00u);
    else return pack_bf16x2(x[s][e].x, x[s][e].y);
  };
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int d = d0 + 128 * e;
    if (d >= v.dp) continue;
    if (u.which == 0) {
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        if (s < s0 || s >= s1) continue;
        const uint32_t w = two(s, e);
        const size_t at = (size_t)(u.slot + s) * v.dp + d;
        if constexpr (I8) *reinterpret_cast<uint16_t*>(base + at) = (uint16_t)(w | w >> 8);
        else *reinterpret_cast<uint32_t*>(base + 2 * at) = w;
      }
    } else if (s1 - s0 == 16) {
      constexpr int WORDS = I8 ? 4 : 8;                               // of an element's 16 tokens
      uint32_t lo[WORDS], hi[WORDS];
#pragma unroll
      for (int j = 0; j < WORDS; ++j) {
        if constexpr (I8) {
          auto four = [&](float a, float b, float c, float d) {       // the low bytes
            return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0c0c0400u) |
                   __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x04000c0cu);
          };
          lo[j] = four(x[4 * j][e].x, x[4 * j + 1][e].x, x[4 * j + 2][e].x, x[4 * j + 3][e].x);
          hi[j] = four(x[4 * j][e].y, x[4 * j + 1][e].y, x[4 * j + 2][e].y, x[4 * j + 3][e].y);
        } else {
          lo[j] = pack_bf16x2(x[2 * j][e].x, x[2 * j + 1][e].x);
          hi[j] = pack_bf16x2(x[2 * j][e].y, x[2 * j + 1][e].y);
        }
      }
      uint4* out = reinterpret_cast<uint4*>(base + v.part_bytes + ((size_t)(u.slot / KV_BLOCK) * v.dp + d) * KV_BLOCK * (I8 ? 1 : 2));
#pragma unroll
      for (int j = 0; j < WORDS / 4; ++j) {
        out[j] = make_uint4(lo[4 * j], lo[4 * j + 1], lo[4 * j + 2], lo[4 * j + 3]);
        out[WORDS / 4 + j] = make_uint4(hi[4 * j], hi[4 * j + 1], hi[4 * j + 2], hi[4 * j + 3]);
      }
    } else {
      const size_t at = ((size_t)(u.slot / KV_BLOCK) * v.dp + d) * KV_BLOCK;
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        if (s < s0 || s >= s1) continue;
        const uint32_t w = two(s, e);
        if constexpr (I8) {
          base[v.part_bytes + at + s] = (uint8_t)w;
          base[v.part_bytes + at + KV_BLOCK + s] = (uint8_t)(w >> 16);
        } else {
          uint16_t* out = reinterpret_cast<uint16_t*>(base + v.part_bytes) + at + s;
          out[0] = (uint16_t)w;
          out[KV_BLOCK] = (uint16_t)(w >> 16);
        }
      }
    }
  }
}

// The way back, block by block as it was written: 16 ragged histories up to 8192 tokens, 8 heads of 128, INT8 to bf16: 211 MB in 34 us.
template <typename T, int KIND, int LPH, int E>
__global__ __launch_bounds__(256) void kv_read_kernel(kv_view v, T* __restrict__ K, T* __restrict__ V, int64_t ks, int64_t vs) {
  constexpr bool I8 = KIND == PQ_KV_INT8;
  const int lane = threadIdx.x & 63;
  kv_unit u;
  if (!kv_find_unit<LPH>(v, u)) return;
  T* dst = u.which ? V : K;
  if (!dst || u.head >= v.n_kv_heads) return;
  const int64_t stride = u.which ? vs : ks;
  const int d0 = 2 * (lane % LPH);
  dst += (size_t)u.head * v.d;
  // rows at negative positions and those without a page
  for (int s = u.s0; s < (u.page < 0 ? u.s1 : min(u.s1, 0)); ++s)
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (d0 + 128 * e < v.d) store_pair(dst + (u.t0 + s - u.s0) * stride + d0 + 128 * e, 0.0f, 0.0f);
  if (u.page < 0) return;
  u.t0 -= u.s0;
  const int s0 = max(u.s0, 0), s1 = u.s1;
  const uint8_t* base = kv_head(v, u.page, u.head);
  float step[16];
  if constexpr (I8) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base + 2 * (size_t)v.part_bytes) + (u.which << v.page_shift) + u.slot);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 x = p[j];
      step[4 * j] = x.x; step[4 * j + 1] = x.y; step[4 * j + 2] = x.z; step[4 * j + 3] = x.w;
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int d = d0 + 128 * e;
    if (d >= v.d) continue;
    float2 x[16];
    if (u.which == 0) {
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        const size_t at = (size_t)(u.slot + s) * v.dp + d;
        if constexpr (I8) {
          const uint16_t w = *reinterpret_cast<const uint16_t*>(base + at);
          x[s] = make_float2((float)(int8_t)w, (float)(int8_t)(w >> 8));
        } else {
          x[s] = pair_of(*reinterpret_cast<const uint32_t*>(base + 2 * at));
        }
      }
    } else {
      constexpr int PER = I8 ? 4 : 2, WORDS = 16 / PER;
      const uint4* p = reinterpret_cast<const uint4*>(base + v.part_bytes + ((size_t)(u.slot / KV_BLOCK) * v.dp + d) * KV_BLOCK * (I8 ? 1 : 2));
      uint32_t w[2 * WORDS];
#pragma unroll
      for (int j = 0; j < WORDS / 2; ++j) {
        const uint4 y = p[j];
        w[4 * j] = y.x; w[4 * j + 1] = y.y; w[4 * j + 2] = y.z; w[4 * j + 3] = y.w;
      }
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        const uint32_t a = w[s / PER] >> (32 / PER * (s % PER)), b = w[WORDS + s / PER] >> (32 / PER * (s % PER));
        x[s] = I8 ? make_float2((float)(int8_t)a, (float)(int8_t)b) : make_float2(__uint_as_float(a << 16), __uint_as_float(b << 16));
      }
    }
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      if (s < s0 || s >= s1) continue;
      if constexpr (I8) { x[s].x *= step[s]; x[s].y *= step[s]; }
      store_pair(dst + (u.t0 + s) * stride + d, x[s].x, x[s].y);
    }
  }
}

template <typename F>
void by_width(int dp, F f) {      // lanes a head, pairs of elements a lane
  if (dp <= 32) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  else if (dp <= 64) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
  else if (dp <= 128) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
}
// Wavefronts of a call: blocks of 16 tokens (see kv_find_unit), groups of heads, keys and values.
int64_t kv_units(const kv_view& v) {
  const int hpu = v.dp <= 32 ? 4 : v.dp <= 64 ? 2 : 1;
  const int64_t blocks = v.row_start ? (int64_t)v.T / 16 + 2 * (int64_t)v.n_seqs : (v.T < v.n_seqs ? v.T : v.n_seqs);
  return blocks * ((v.n_kv_heads + hpu - 1) / hpu) * 2;
}
template <int KIND, typename T>
void launch_write(const kv_view& v, const void* K, const void* V, int64_t ks, int64_t vs, hipStream_t s) {
  const unsigned grid = (unsigned)((kv_units(v) + 3) / 4);
  by_width(v.dp, [&](auto lph, auto e) {
    kv_write_kernel<T, KIND, decltype(lph)::value, decltype(e)::value><<<grid, 256, 0, s>>>(v, (const T*)K, (const T*)V, ks, vs);
  });
}
template <int KIND, typename T>
void launch_read(const kv_view& v, void* K, void* V, int64_t ks, int64_t vs, hipStream_t s) {
  const unsigned grid = (unsigned)((kv_units(v) + 3) / 4);
  by_width(v.dp, [&](auto lph, auto e) {
    kv_read_kernel<T, KIND, decltype(lph)::value, decltype(e)::value><<<grid, 256, 0, s>>>(v, (T*)K, (T*)V, ks, vs);
  });
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
  const size_t page = pq_kv_make_view(*d, nullptr, nullptr, nullptr, nullptr, 0).head_bytes * d->n_kv_heads;      // (at most 2^36)
  PQ_REQUIRE((size_t)d->n_pages <= ((size_t)1 << 62) / page, PQ_ERR_SHAPE, "n_pages=%d of %zu bytes exceed 2^62 bytes", d->n_pages, page);
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
  kv_view v = pq_kv_make_view(*d, cache, lens, lens, table, T);      // (with a row_start: the larger count)
  PQ_REQUIRE(T <= (1 << 29) && d->n_seqs < (1 << 28) && (kv_units(v) + 3) / 4 <= 0x7fffffff, PQ_ERR_SHAPE,
             "T=%d rows of %d heads in %d sequences are too many for one call", T, d->n_kv_heads, d->n_seqs);
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
  const bool i8 = d->kv_kind == PQ_KV_INT8;
  if (dtype == PQ_F32) i8 ? launch_write<PQ_KV_INT8, float>(v, K, V, k_stride, v_stride, s) : launch_write<PQ_KV_BF16, float>(v, K, V, k_stride, v_stride, s);
  else i8 ? launch_write<PQ_KV_INT8, uint16_t>(v, K, V, k_stride, v_stride, s) : launch_write<PQ_KV_BF16, uint16_t>(v, K, V, k_stride, v_stride, s);
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
  const bool i8 = d->kv_kind == PQ_KV_INT8;
  if (dtype == PQ_F32) i8 ? launch_read<PQ_KV_INT8, float>(v, K, V, k_stride, v_stride, s) : launch_read<PQ_KV_BF16, float>(v, K, V, k_stride, v_stride, s);
  else i8 ? launch_read<PQ_KV_INT8, uint16_t>(v, K, V, k_stride, v_stride, s) : launch_read<PQ_KV_BF16, uint16_t>(v, K, V, k_stride, v_stride, s);
  PQ_CHECK_LAUNCH("kv_read_kernel");
  return PQ_OK;
}
