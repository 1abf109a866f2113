// Rotary positions of queries and keys.
#include <cmath>
#include <type_traits>

#include "pq_kv.h"

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

constexpr int ROPE_TABLE = 2048;       // sines and cosines in LDS, of all rows of a workgroup

// i / by for i * by < 2^32, by a product (a division costs more than an element's bytes).
struct divisor {
  uint32_t by, inverse;
  __host__ void set(int x) { by = (uint32_t)x; inverse = (uint32_t)((0xffffffffull + x) / x); }
  __device__ __forceinline__ int into(int i) const { return by == 1 ? i : (int)__umulhi((uint32_t)i, inverse); }
};

struct rope_args {
  kv_view v;                     // row_start, lens, n_seqs, T
  const void *q, *k;
  void *qr, *kr;
  int64_t qs, ks, qrs, krs;      // elements between rows
  const double* freqs;
  int heads, total_heads, d, half, pieces, rows;   // pieces: of a head's pairs, VEC each;  rows: of a workgroup
  divisor by_half, by_row, by_piece;               // by_row: pieces of a row
  int inverse, whole;            // whole: sequences are the call's rows
  float scale;
};

// Sine and cosine of `turns` turns: reduced to an eighth of a turn in 64 bits, there the Taylor series in 32 (x^11 / 11! is 2e-9 at pi / 4).
__device__ __forceinline__ void sine_cosine(double turns, float& s, float& c) {
  const double q = __builtin_rint(4.0 * turns);
  const float x = (float)((turns - 0.25 * q) * 6.283185307179586476925286766559);
  const float z = x * x;
  float p = __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  p = __builtin_fmaf(z, p, 8.3333333e-3f);
  p = __builtin_fmaf(z, p, -0.16666667f);
  const float sn = __builtin_fmaf(x * z, p, x);
  float r = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  r = __builtin_fmaf(z, r, -1.3888889e-3f);
  r = __builtin_fmaf(z, r, 4.1666667e-2f);
  r = __builtin_fmaf(z, r, -0.5f);
  const float cs = __builtin_fmaf(z, r, 1.0f);
  const int k = (int)(q - 4.0 * __builtin_floor(0.25 * q));       // 0 .. 3
  s = k & 1 ? cs : sn;
  c = k & 1 ? sn : cs;
  if (k & 2) s = -s;
  if (k == 1 || k == 2) c = -c;
}

// VEC pairs of a head, as two runs of VEC elements: of PQ_ROPE_HALF x_i .. and y_i .., of PQ_ROPE_PAIRS (and of what is copied) neighbours.
template <typename T, int VEC> using run = T __attribute__((ext_vector_type(VEC)));

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return bf16_to_f32(x); }
template <typename T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t rounded<uint16_t>(float x) { return f32_to_bf16(x); }

// Bound by memory: a workgroup forms the sines and cosines of its rows once, for all heads, then turns them piece by piece, 16 bytes of x and of y a lane
// where everything is aligned to that (32768 rows, 32+8 heads of 128, bf16: 131 us, 5.1 TB/s; a pair a lane 251), else a pair a lane, since heads
// of 90 begin at multiples of four bytes and a piece of 16 would hold pairs of two of them (8192 rows, 32+32 heads of 90, bf16: pairs of neighbours, four bytes a
// lane and load, 52 us, 3.6 TB/s; halves, two bytes, 56; fp32 80 and 86).  The turns are fp64: near position 2^23
// fp32 would be off by 2^-4 of a turn, fp64 is by 2^-32.
template <typename T, int LAYOUT, int VEC>
__global__ __launch_bounds__(256) void rope_kernel(rope_args a) {
  __shared__ float2 table[ROPE_TABLE];
  __shared__ int places[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * a.rows;
  for (int r = wave; r < a.rows; r += 4) {
    const int64_t row = row0 + r;
    int pos = INT32_MIN;                       // (no row of a sequence)
    if (row < a.v.T) {
      kv_rows s;
      const int b = kv_find_rows(a.v, (int)row, s, [&](int r0, int) { return r0; });
      if (b >= 0 && row < (int64_t)s.r0 + s.n) pos = (a.whole ? 0 : s.first) + (int)(row - s.r0);
    }
    if (lane == 0) places[r] = pos;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.rows * a.half; i += 256) {
    const int r = a.by_half.into(i), f = i - r * a.half, pos = places[r];
    float s = 0.0f, c = 1.0f;
    if (pos != INT32_MIN) sine_cosine((double)pos * a.freqs[f], s, c);
    table[i] = make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
  }
  __syncthreads();
  typedef run<T, VEC> R;
  const int per_row = a.total_heads * a.pieces, all = a.rows * per_row;
  for (int i = threadIdx.x; i < all; i += 256) {
    const int r = a.rows > 1 ? a.by_row.into(i) : 0, x = i - r * per_row, head = a.by_piece.into(x), at = (x - head * a.pieces) * VEC;   // pairs at .. at + VEC - 1
    if (places[r] == INT32_MIN) continue;
    const bool is_k = head >= a.heads;
    const int64_t row = row0 + r;
    const T* from = (is_k ? (const T*)a.k + row * a.ks + (int64_t)(head - a.heads) * a.d : (const T*)a.q + row * a.qs + (int64_t)head * a.d);
    T* to = (is_k ? (T*)a.kr + row * a.krs + (int64_t)(head - a.heads) * a.d : (T*)a.qr + row * a.qrs + (int64_t)head * a.d);
    if (LAYOUT == PQ_ROPE_HALF && at < a.half) {
      const R u = *reinterpret_cast<const R*>(from + at), w = *reinterpret_cast<const R*>(from + at + a.half);
      R p, q;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float2 t = table[r * a.half + at + j];
        const float m = value(u[j]), n = value(w[j]);
        p[j] = rounded<T>(m * t.x - n * t.y);
        q[j] = rounded<T>(n * t.x + m * t.y);
      }
      *reinterpret_cast<R*>(to + at) = p;
      *reinterpret_cast<R*>(to + at + a.half) = q;
    } else {
      R u = *reinterpret_cast<const R*>(from + 2 * at), w = *reinterpret_cast<const R*>(from + 2 * at + VEC);
      if (LAYOUT == PQ_ROPE_PAIRS && at < a.half) {
        T e[2 * VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) { e[j] = u[j]; e[VEC + j] = w[j]; }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float2 t = table[r * a.half + at + j];
          const float m = value(e[2 * j]), n = value(e[2 * j + 1]);
          e[2 * j] = rounded<T>(m * t.x - n * t.y);
          e[2 * j + 1] = rounded<T>(n * t.x + m * t.y);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) { u[j] = e[j]; w[j] = e[VEC + j]; }
      }
      *reinterpret_cast<R*>(to + 2 * at) = u;
      *reinterpret_cast<R*>(to + 2 * at + VEC) = w;
    }
  }
}

int check_rope(const pq_rope_desc* d) {
  PQ_REQUIRE(d, PQ_ERR_BAD_ARG, "NULL descriptor");
  PQ_REQUIRE(d->n_seqs >= 0, PQ_ERR_BAD_ARG, "n_seqs=%d is negative", d->n_seqs);
  PQ_REQUIRE(d->n_heads > 0 && d->n_kv_heads >= 0 && (int64_t)d->n_heads + d->n_kv_heads <= 65536, PQ_ERR_BAD_ARG,
             "n_heads=%d and n_kv_heads=%d must be positive (n_kv_heads: or 0) and at most 65536 together", d->n_heads, d->n_kv_heads);
  PQ_REQUIRE(d->d_head >= 2 && d->d_head <= 256 && d->d_head % 2 == 0, PQ_ERR_SHAPE, "d_head=%d must be even and in 2..256", d->d_head);
  PQ_REQUIRE(d->rot_dim >= 2 && d->rot_dim <= d->d_head && d->rot_dim % 2 == 0, PQ_ERR_SHAPE, "rot_dim=%d must be even and in 2..d_head=%d", d->rot_dim,
             d->d_head);
  PQ_REQUIRE(d->layout == PQ_ROPE_HALF || d->layout == PQ_ROPE_PAIRS, PQ_ERR_BAD_ARG, "unknown layout %d", d->layout);
  PQ_REQUIRE(d->inverse == 0 || d->inverse == 1, PQ_ERR_BAD_ARG, "inverse=%d must be 0 or 1", d->inverse);
  PQ_REQUIRE(std::isfinite(d->scale), PQ_ERR_BAD_ARG, "scale must be finite");
  return PQ_OK;
}

template <typename T, int VEC> void launch_rope(const rope_args& a, int layout, unsigned grid, hipStream_t s) {
  if (layout == PQ_ROPE_HALF) rope_kernel<T, PQ_ROPE_HALF, VEC><<<grid, 256, 0, s>>>(a);
  else rope_kernel<T, PQ_ROPE_PAIRS, VEC><<<grid, 256, 0, s>>>(a);
}

}  // namespace

extern "C" int pq_rope(const pq_rope_desc* d, const void* Q, int64_t q_stride, const void* K, int64_t k_stride, int32_t dtype, int32_t T,
                       const double* freqs, const int32_t* row_start, const int32_t* lens, void* Qr, int64_t qr_stride, void* Kr, int64_t kr_stride,
                       void* stream) {
  if (int e = check_rope(d)) return e;
  PQ_REQUIRE(dtype == PQ_F32 || dtype == PQ_BF16, PQ_ERR_DTYPE, "dtype %d is not PQ_F32 or PQ_BF16", dtype);
  PQ_REQUIRE(T >= 0 && T <= (1 << 29), PQ_ERR_BAD_ARG, "T=%d must be in 0..2^29", T);
  if (T == 0 || d->n_seqs == 0) return PQ_OK;
  const bool has_k = d->n_kv_heads > 0;
  PQ_REQUIRE(Q && Qr && freqs && (!has_k || (K && Kr)), PQ_ERR_BAD_ARG, "NULL buffer");
  PQ_REQUIRE(row_start || lens, PQ_ERR_BAD_ARG, "row_start and lens are both NULL");
  const int64_t qn = (int64_t)d->n_heads * d->d_head, kn = (int64_t)d->n_kv_heads * d->d_head;
  PQ_REQUIRE(q_stride >= qn && qr_stride >= qn && (!has_k || (k_stride >= kn && kr_stride >= kn)), PQ_ERR_SHAPE,
             "row strides must be at least the heads' elements (%lld of Q, %lld of K)", (long long)qn, (long long)kn);
  PQ_REQUIRE(((q_stride | qr_stride | (has_k ? k_stride | kr_stride : 0)) & 1) == 0, PQ_ERR_SHAPE, "row strides must be even");
  PQ_REQUIRE(((((uintptr_t)Q | (uintptr_t)Qr | (uintptr_t)(has_k ? K : nullptr) | (uintptr_t)(has_k ? Kr : nullptr)) & 15) == 0) &&
                 ((uintptr_t)freqs & 7) == 0, PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  PQ_REQUIRE((Q != Qr || q_stride == qr_stride) && (!has_k || K != Kr || k_stride == kr_stride), PQ_ERR_SHAPE, "in place, both strides are the same");
  const int size = dtype == PQ_F32 ? 4 : 2;
  const pq_region written[] = {{"Qr", (uintptr_t)Qr, T, qr_stride * size, qn * size, 1}, {"Kr", (uintptr_t)Kr, has_k ? T : 0, kr_stride * size, kn * size, 2}};
  const pq_region read[] = {{"Q", (uintptr_t)Q, T, q_stride * size, qn * size, 1}, {"K", (uintptr_t)K, has_k ? T : 0, k_stride * size, kn * size, 2},
                            pq_flat_region("freqs", freqs, (int64_t)d->rot_dim / 2 * 8),
                            pq_flat_region("row_start", row_start, row_start ? ((int64_t)d->n_seqs + 1) * 4 : 0),
                            pq_flat_region("lens", lens, lens ? (int64_t)d->n_seqs * 4 : 0)};
  if (int e = pq_refuse_overlap(written, 2, read, 5)) return e;
  rope_args a = {};
  a.v.lens = lens; a.v.row_start = row_start; a.v.n_seqs = d->n_seqs; a.v.T = T;
  a.whole = lens == nullptr;
  if (a.whole) a.v.lens = row_start;       // (read, not used)
  a.q = Q; a.k = has_k ? K : nullptr; a.qr = Qr; a.kr = has_k ? Kr : nullptr;
  a.qs = q_stride; a.ks = k_stride; a.qrs = qr_stride; a.krs = kr_stride;
  a.freqs = freqs;
  a.heads = d->n_heads; a.total_heads = d->n_heads + d->n_kv_heads; a.d = d->d_head; a.half = d->rot_dim / 2;
  a.inverse = d->inverse; a.scale = d->scale;
  // pairs of a piece: 16 bytes of either kind of run, or one pair where rows, heads or the part that turns are not multiples of that
  const int wide = dtype == PQ_BF16 ? 8 : 4;
  const int64_t strides = q_stride | qr_stride | (has_k ? k_stride | kr_stride : 0);
  const bool aligned = (d->d_head / 2) % wide == 0 && a.half % wide == 0 && strides % wide == 0;
  a.pieces = d->d_head / 2 / (aligned ? wide : 1);
  // rows of a workgroup: about 1024 pieces, at most what the table holds, and enough workgroups for the CUs (4096 rows of 32+8 heads of 128: 16.8 us whatever
  // the last is, from one row to all that the others allow; fewer rows a workgroup spread short calls)
  const int per_row = a.total_heads * a.pieces;
  int rows = 1024 / per_row;
  if (rows > ROPE_TABLE / a.half) rows = ROPE_TABLE / a.half;
  if (rows > T / 1024) rows = T / 1024;
  if (rows > 64) rows = 64;
  if (rows < 1) rows = 1;
  a.rows = rows;
  a.by_half.set(a.half);         // (at most ROPE_TABLE, ..
  a.by_row.set(per_row);         // .. 1024 where there are several rows ..
  a.by_piece.set(a.pieces);      // .. and 2^16 heads of 2^7 pieces are divided)
  const unsigned grid = (unsigned)((T + rows - 1) / rows);
  PQ_REQUIRE(grid <= PQ_MOST_WORKGROUPS, PQ_ERR_SHAPE, "T=%d rows of %d heads of %d are too many for one call", T, a.total_heads, a.d);
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_ROPE, s);
  if (dtype == PQ_BF16) {
    if (aligned) launch_rope<uint16_t, 8>(a, d->layout, grid, s);
    else launch_rope<uint16_t, 1>(a, d->layout, grid, s);
  } else {
    if (aligned) launch_rope<float, 4>(a, d->layout, grid, s);
    else launch_rope<float, 1>(a, d->layout, grid, s);
  }
  PQ_CHECK_LAUNCH("rope_kernel");
  return PQ_OK;
}
