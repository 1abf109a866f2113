// One AdamW step over many tensors in one launch, with states in fp32 or in 8 bits.
#include "pq_internal.h"

#include <cmath>
#include <type_traits>
#include <cstring>

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

constexpr int AW_BLOCK = 256;      // elements that share the steps of their 8-bit states
// Elements of a workgroup, and where that leaves CUs without work.  With 8-bit states, 20M elements: 30 us in pieces of 4096, 28 of 2048, 26 of 1024; two
// layers of the 1.3B shape, read back as well: 476, 468 and 493 (441 to 457 with maxima and codes as they are now).  1.5M elements: 16.7 us in
// pieces of 4096, 12.4 of 1024.
constexpr int AW_PIECE = 2048;
constexpr int AW_SMALL = 1024;

// What a workgroup works on: `n` elements that begin at a multiple of AW_BLOCK of their tensor.
struct adamw_piece {
  void* param;
  const void* grad;
  float* master;
  void* m;
  void* v;
  float* steps;
  float* m_values;
  float* v_values;
  int64_t n;
};

struct adamw_consts { float b1, c1, b2, c2, eps; };

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const uint16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, const float* x) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store4(uint16_t* p, const float* x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = f32_to_bf16(x); }

// The nearest code c to y = |x| / step under the law c^2: the one with (c - 1/2)^2 <= y <= (c + 1/2)^2, of a tie the even one.  Borders below 2^16 are
// fp32 numbers, so a root that is off in its last place is put right exactly; as bits, so that an odd c counts its upper border as passed and its lower
// one as not reached (below 0 it is negative).
__device__ __forceinline__ int square_code(float y, int top) {
  const float c = __builtin_rintf(__builtin_amdgcn_sqrtf(y)), up = c + 0.5f, down = c - 0.5f;
  const int code = (int)c, odd = code & 1, bits = __float_as_int(y);
  return min(code + (bits + odd > __float_as_int(up * up) ? 1 : 0) - (bits < __float_as_int(down * fabsf(down)) + odd ? 1 : 0), top);
}
// The largest x of a wavefront, by lanes' neighbours without LDS: in fours, eights, rows of sixteen, rows 1 and 3, row 3's last lane.
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t x) {
  auto from = [](uint32_t v, auto control, auto rows) {                     // (0 where a row is left out)
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(control)::value, decltype(rows)::value, 0xf, false);
  };
  typedef std::integral_constant<int, 0xf> all;
  x = max(x, from(x, std::integral_constant<int, 0xb1>{}, all{}));          // quad_perm 1 0 3 2
  x = max(x, from(x, std::integral_constant<int, 0x4e>{}, all{}));          // quad_perm 2 3 0 1
  x = max(x, from(x, std::integral_constant<int, 0x141>{}, all{}));         // row_half_mirror
  x = max(x, from(x, std::integral_constant<int, 0x140>{}, all{}));         // row_mirror
  x = max(x, from(x, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{}));   // row_bcast 15
  x = max(x, from(x, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{}));   // row_bcast 31
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// Step of a block from the largest |x| as bits (those of infinities and NaN are above every finite value's), and its inverse; NaN and zero where it
// is not finite.
__device__ __forceinline__ void block_step(uint32_t top_bits, float inv_square, float& step, float& inv) {
  step = fmaxf(__uint_as_float(top_bits) * inv_square, 1.17549435e-38f);
  inv = 1.0f / step;
  if (top_bits >= 0x7f800000u) {
    step = __uint_as_float(0x7fc00000u);
    inv = 0.0f;
  }
}

// A lane has four neighbouring elements, so a wavefront has a block and takes its maxima by exchanges.  Bound by memory: 28 bytes an element with fp32
// masters and states, bf16 weights and gradients (10M elements: 61 us, 4.6 TB/s, of inputs that are not in the last-level cache), 12 with 8-bit states, bf16
// weights and fp32 gradients, where the arithmetic of an element (roots and the nearest codes, exactly) is nearly as long as its bytes.
template <typename P, typename G, bool EIGHT, bool MASTER>
__global__ __launch_bounds__(256) void adamw_kernel(const adamw_piece* __restrict__ pieces, adamw_consts k, const float* __restrict__ scalars) {
  const adamw_piece t = pieces[blockIdx.x];
  const float keep = scalars[0], size = scalars[1], root = scalars[2], gscale = scalars[3];
  P* param = (P*)t.param;
  const G* grad = (const G*)t.grad;
  const int n = (int)t.n;
  for (int at = threadIdx.x * 4; (at & ~255) < n; at += 1024) {
    const int left = n - at;
    float w[4] = {}, g[4] = {}, m[4] = {}, v[4] = {}, r[4];
    auto fill = [&](float* x, float4 y) { x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w; };
    uint32_t qm = 0, qr = 0;
    float2 step = make_float2(0.0f, 0.0f);
    if (left >= 4) {
      if constexpr (MASTER) fill(w, load4(t.master + at));
      else fill(w, load4(param + at));
      fill(g, load4(grad + at));
      if constexpr (EIGHT) {
        qm = *reinterpret_cast<const uint32_t*>((const int8_t*)t.m + at);
        qr = *reinterpret_cast<const uint32_t*>((const uint8_t*)t.v + at);
      } else {
        fill(m, load4((const float*)t.m + at));
        fill(v, load4((const float*)t.v + at));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < left) {
          if constexpr (MASTER) w[j] = t.master[at + j];
          else w[j] = load1(param + at + j);
          g[j] = load1(grad + at + j);
          if constexpr (EIGHT) {
            qm |= (uint32_t)((const uint8_t*)t.m)[at + j] << (8 * j);
            qr |= (uint32_t)((const uint8_t*)t.v)[at + j] << (8 * j);
          } else {
            m[j] = ((const float*)t.m)[at + j];
            v[j] = ((const float*)t.v)[at + j];
          }
        }
    }
    if constexpr (EIGHT) {
      step = *reinterpret_cast<const float2*>(t.steps + 2 * (at >> 8));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float q = (float)(int8_t)(qm >> (8 * j)), u = (float)((qr >> (8 * j)) & 0xff);
        m[j] = q * fabsf(q) * step.x;
        r[j] = u * u * step.y;
        v[j] = r[j] * r[j];
      }
    }
    uint32_t top_m = 0, top_r = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = g[j] * gscale;
      m[j] = m[j] * k.b1 + x * k.c1;
      v[j] = v[j] * k.b2 + x * k.c2 * x;
      r[j] = __builtin_sqrtf(v[j]);
      w[j] = w[j] * keep - m[j] * size / (r[j] * root + k.eps);
      top_m = max(top_m, __float_as_uint(m[j]) & 0x7fffffffu);
      top_r = max(top_r, __float_as_uint(r[j]) & 0x7fffffffu);
    }
    if constexpr (EIGHT) {
      float sm, im, sr, ir;
      block_step(wave_max_bits(top_m), 1.0f / 16129.0f, sm, im);
      block_step(wave_max_bits(top_r), 1.0f / 65025.0f, sr, ir);
      qm = qr = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = square_code(fabsf(m[j]) * im, 127), u = square_code(r[j] * ir, 255);
        qm |= ((uint32_t)(m[j] < 0.0f ? -c : c) & 0xffu) << (8 * j);
        qr |= (uint32_t)max(u, r[j] > 0.0f ? 1 : 0) << (8 * j);
      }
      if ((threadIdx.x & 63) == 0) *reinterpret_cast<float2*>(t.steps + 2 * (at >> 8)) = make_float2(sm, sr);
    }
    if (left >= 4) {
      if constexpr (MASTER) store4(t.master + at, w);
      store4(param + at, w);
      if constexpr (EIGHT) {
        *reinterpret_cast<uint32_t*>((int8_t*)t.m + at) = qm;
        *reinterpret_cast<uint32_t*>((uint8_t*)t.v + at) = qr;
      } else {
        store4((float*)t.m + at, m);
        store4((float*)t.v + at, v);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < left) {
          if constexpr (MASTER) t.master[at + j] = w[j];
          store1(param + at + j, w[j]);
          if constexpr (EIGHT) {
            ((uint8_t*)t.m)[at + j] = (uint8_t)(qm >> (8 * j));
            ((uint8_t*)t.v)[at + j] = (uint8_t)(qr >> (8 * j));
          } else {
            ((float*)t.m)[at + j] = m[j];
            ((float*)t.v)[at + j] = v[j];
          }
        }
    }
  }
}

__global__ __launch_bounds__(256) void adamw_read_kernel(const adamw_piece* __restrict__ pieces) {
  const adamw_piece t = pieces[blockIdx.x];
  const int n = (int)t.n;
  for (int at = threadIdx.x * 4; at < n; at += 1024) {
    const float2 step = *reinterpret_cast<const float2*>(t.steps + 2 * (at >> 8));
    const int left = n - at;
    uint32_t qm = 0, qr = 0;
    if (left >= 4) {
      qm = *reinterpret_cast<const uint32_t*>((const int8_t*)t.m + at);
      qr = *reinterpret_cast<const uint32_t*>((const uint8_t*)t.v + at);
    } else {
      for (int j = 0; j < left; ++j) {
        qm |= (uint32_t)((const uint8_t*)t.m)[at + j] << (8 * j);
        qr |= (uint32_t)((const uint8_t*)t.v)[at + j] << (8 * j);
      }
    }
    float m[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float q = (float)(int8_t)(qm >> (8 * j)), u = (float)((qr >> (8 * j)) & 0xff), r = u * u * step.y;
      m[j] = q * fabsf(q) * step.x;
      v[j] = r * r;
    }
    if (left >= 4) {
      store4(t.m_values + at, m);
      store4(t.v_values + at, v);
    } else {
      for (int j = 0; j < left; ++j) {
        t.m_values[at + j] = m[j];
        t.v_values[at + j] = v[j];
      }
    }
  }
}

int check_adamw(const pq_adamw_desc* d) {
  PQ_REQUIRE(d, PQ_ERR_BAD_ARG, "NULL descriptor");
  PQ_REQUIRE(d->n_tensors >= 0, PQ_ERR_BAD_ARG, "n_tensors=%d is negative", d->n_tensors);
  PQ_REQUIRE((d->param_dtype == PQ_F32 || d->param_dtype == PQ_BF16) && (d->grad_dtype == PQ_F32 || d->grad_dtype == PQ_BF16), PQ_ERR_DTYPE,
             "parameters and gradients are PQ_F32 or PQ_BF16");
  PQ_REQUIRE(d->state_kind == PQ_STATE_F32 || d->state_kind == PQ_STATE_8BIT, PQ_ERR_BAD_ARG, "unknown state_kind %d", d->state_kind);
  PQ_REQUIRE((d->has_masters == 0 || d->has_masters == 1) && (d->has_values == 0 || d->has_values == 1), PQ_ERR_BAD_ARG,
             "has_masters and has_values must be 0 or 1");
  PQ_REQUIRE(!d->has_masters || d->param_dtype == PQ_BF16, PQ_ERR_DTYPE, "masters belong to PQ_BF16 parameters");
  PQ_REQUIRE(!d->has_values || d->state_kind == PQ_STATE_8BIT, PQ_ERR_BAD_ARG, "m_values and v_values belong to 8-bit states");
  PQ_REQUIRE(d->beta1 >= 0.0 && d->beta1 < 1.0 && d->beta2 >= 0.0 && d->beta2 < 1.0, PQ_ERR_BAD_ARG, "beta1 and beta2 must be in [0, 1)");
  PQ_REQUIRE(d->eps >= 1.17549435082228751e-38 && d->eps < 3.0e38, PQ_ERR_BAD_ARG, "eps must be positive (2^-126 at least) and finite");
  return PQ_OK;
}

int check_tensors(const pq_adamw_desc* d, const pq_adamw_tensor* t, int64_t* pieces, int* size) {
  PQ_REQUIRE(t || d->n_tensors == 0, PQ_ERR_BAD_ARG, "NULL tensors");
  const bool eight = d->state_kind == PQ_STATE_8BIT;
  int64_t small = 0, large = 0;
  for (int i = 0; i < d->n_tensors; ++i) {
    PQ_REQUIRE(t[i].n >= 0 && t[i].n <= ((int64_t)1 << 40), PQ_ERR_BAD_ARG, "tensor %d has %lld elements", i, (long long)t[i].n);
    if (t[i].n == 0) continue;
    PQ_REQUIRE(t[i].param && t[i].grad && t[i].m && t[i].v && (!eight || t[i].steps), PQ_ERR_BAD_ARG, "tensor %d: NULL buffer", i);
    PQ_REQUIRE(!t[i].master == !d->has_masters, PQ_ERR_BAD_ARG, "tensor %d: a master with has_masters=%d, or none", i, d->has_masters);
    PQ_REQUIRE(!t[i].m_values == !d->has_values && !t[i].v_values == !d->has_values, PQ_ERR_BAD_ARG,
               "tensor %d: m_values and v_values with has_values=%d, or not both", i, d->has_values);
    PQ_REQUIRE((((uintptr_t)t[i].param | (uintptr_t)t[i].grad | (uintptr_t)t[i].master | (uintptr_t)t[i].m | (uintptr_t)t[i].v |
                 (uintptr_t)t[i].m_values | (uintptr_t)t[i].v_values) & 15) == 0 && (!eight || ((uintptr_t)t[i].steps & 7) == 0),
               PQ_ERR_SHAPE, "tensor %d: buffers must be 16-byte aligned (steps: 8)", i);
    small += (t[i].n + AW_SMALL - 1) / AW_SMALL;
    large += (t[i].n + AW_PIECE - 1) / AW_PIECE;
  }
  PQ_REQUIRE(large <= PQ_MOST_WORKGROUPS, PQ_ERR_SHAPE, "too many elements for one call");
  *size = large < 1024 ? AW_SMALL : AW_PIECE;
  *pieces = large < 1024 ? small : large;
  if (*pieces == 0) *pieces = 1;       // (one without elements)
  return PQ_OK;
}

template <typename P, typename G, bool EIGHT>
void launch_adamw(const adamw_piece* plan, unsigned pieces, const adamw_consts& k, const float* scalars, bool masters, hipStream_t s) {
  if constexpr (sizeof(P) == 2)
    if (masters) {
      adamw_kernel<P, G, EIGHT, true><<<pieces, 256, 0, s>>>(plan, k, scalars);
      return;
    }
  adamw_kernel<P, G, EIGHT, false><<<pieces, 256, 0, s>>>(plan, k, scalars);
}
template <typename P, typename G>
void launch_adamw_states(const adamw_piece* plan, unsigned pieces, const adamw_consts& k, const float* scalars, bool masters, bool eight, hipStream_t s) {
  if (eight) launch_adamw<P, G, true>(plan, pieces, k, scalars, masters, s);
  else launch_adamw<P, G, false>(plan, pieces, k, scalars, masters, s);
}

int check_plan(const pq_adamw_desc* d, const void* plan, size_t plan_bytes) {
  if (int e = check_adamw(d)) return e;
  PQ_REQUIRE(plan, PQ_ERR_BAD_ARG, "NULL plan");
  PQ_REQUIRE(((uintptr_t)plan & 15) == 0, PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  PQ_REQUIRE(plan_bytes > 0 && plan_bytes % sizeof(adamw_piece) == 0 && plan_bytes / sizeof(adamw_piece) <= PQ_MOST_WORKGROUPS, PQ_ERR_WORKSPACE,
             "a plan has pq_adamw_plan_bytes() bytes, not %zu", plan_bytes);
  return PQ_OK;
}

}  // namespace

extern "C" size_t pq_adamw_plan_bytes(const pq_adamw_desc* d, const pq_adamw_tensor* tensors) {
  int64_t pieces;
  int size;
  if (check_adamw(d) || check_tensors(d, tensors, &pieces, &size)) return 0;
  return (size_t)pieces * sizeof(adamw_piece);
}

extern "C" int pq_adamw_plan(const pq_adamw_desc* d, const pq_adamw_tensor* tensors, void* plan, size_t plan_bytes) {
  int64_t pieces;
  int size;
  if (int e = check_adamw(d)) return e;
  if (int e = check_tensors(d, tensors, &pieces, &size)) return e;
  PQ_REQUIRE(plan, PQ_ERR_BAD_ARG, "NULL plan");
  PQ_REQUIRE(((uintptr_t)plan & 7) == 0, PQ_ERR_SHAPE, "a plan on the host is 8-byte aligned");
  PQ_REQUIRE(plan_bytes >= (size_t)pieces * sizeof(adamw_piece), PQ_ERR_WORKSPACE, "plan %zu < %zu bytes", plan_bytes, (size_t)pieces * sizeof(adamw_piece));
  adamw_piece* out = (adamw_piece*)plan;
  memset(out, 0, sizeof(adamw_piece));
  const int ps = d->param_dtype == PQ_F32 ? 4 : 2, gs = d->grad_dtype == PQ_F32 ? 4 : 2, ss = d->state_kind == PQ_STATE_F32 ? 4 : 1;
  for (int i = 0; i < d->n_tensors; ++i) {
    const pq_adamw_tensor& t = tensors[i];
    for (int64_t at = 0; at < t.n; at += size) {
      adamw_piece p;
      p.param = (char*)t.param + at * ps;
      p.grad = (const char*)t.grad + at * gs;
      p.master = t.master ? t.master + at : nullptr;
      p.m = (char*)t.m + at * ss;
      p.v = (char*)t.v + at * ss;
      p.steps = ss == 1 ? t.steps + at / AW_BLOCK * 2 : nullptr;
      p.m_values = t.m_values ? t.m_values + at : nullptr;
      p.v_values = t.v_values ? t.v_values + at : nullptr;
      p.n = t.n - at < size ? t.n - at : size;
      *out++ = p;
    }
  }
  return PQ_OK;
}

extern "C" int pq_adamw_step(const pq_adamw_desc* d, const void* plan, size_t plan_bytes, const float* scalars, void* stream) {
  if (int e = check_plan(d, plan, plan_bytes)) return e;
  PQ_REQUIRE(scalars, PQ_ERR_BAD_ARG, "NULL scalars");
  PQ_REQUIRE(((uintptr_t)scalars & 15) == 0, PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  const adamw_piece* pieces = (const adamw_piece*)plan;
  const unsigned n = (unsigned)(plan_bytes / sizeof(adamw_piece));
  const adamw_consts k = {(float)d->beta1, (float)(1.0 - d->beta1), (float)d->beta2, (float)(1.0 - d->beta2), (float)d->eps};
  const bool eight = d->state_kind == PQ_STATE_8BIT, masters = d->has_masters != 0;
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_ADAMW, s);
  if (d->param_dtype == PQ_F32) {
    if (d->grad_dtype == PQ_F32) launch_adamw_states<float, float>(pieces, n, k, scalars, masters, eight, s);
    else launch_adamw_states<float, uint16_t>(pieces, n, k, scalars, masters, eight, s);
  } else {
    if (d->grad_dtype == PQ_F32) launch_adamw_states<uint16_t, float>(pieces, n, k, scalars, masters, eight, s);
    else launch_adamw_states<uint16_t, uint16_t>(pieces, n, k, scalars, masters, eight, s);
  }
  PQ_CHECK_LAUNCH("adamw_kernel");
  return PQ_OK;
}

extern "C" int pq_adamw_read(const pq_adamw_desc* d, const void* plan, size_t plan_bytes, void* stream) {
  if (int e = check_plan(d, plan, plan_bytes)) return e;
  PQ_REQUIRE(d->state_kind == PQ_STATE_8BIT && d->has_values, PQ_ERR_BAD_ARG, "only 8-bit states whose plan has m_values and v_values are read back");
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_ADAMW, s);
  adamw_read_kernel<<<(unsigned)(plan_bytes / sizeof(adamw_piece)), 256, 0, s>>>((const adamw_piece*)plan);
  PQ_CHECK_LAUNCH("adamw_read_kernel");
  return PQ_OK;
}
