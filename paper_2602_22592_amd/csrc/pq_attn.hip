// Attention over the paged key-value cache: one new token of every sequence (pq_attn_decode) and the rows of prompts (pq_attn_prefill).
//
//     s_t = scale q . k_t,   m = max s_t,   l = sum exp(s_t - m),   o = sum exp(s_t - m) v_t / l,   lse = m + log l
//
// in one pass over the tokens: a tile's scores move m, and what has been summed is scaled by exp(old m - new m).  Parts of a sequence that
// were summed apart join in the same way.  Exponentials are powers of two, with log2 e in the scale.  m, l and the sums of o are fp32.
#include <math.h>
#include <atomic>
#include "pq_kv.h"

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

// ---------------------------------------------------------------------------------------------
// One new token of every sequence
//
// Bound by reading the cache once: a workgroup has one key-value head of one sequence (or a piece of it) with all query heads that share it,
// and its wavefronts take tiles of 64 tokens in turn, from the cache into the matrix instructions' registers with no LDS between.  The scores
// are formed transposed (token by head) with the key rows in such an order that a lane ends with the probabilities of the tokens that the
// product with the values wants from it.  An INT8 cache multiplies as it lies: the query and p times the value's step are 24-bit integers
// relative to their largest, in three digits of base 256 that occupy three of the four columns of a head (error 2^-22 of the largest, far
// below the quantiser's 2^-8; the fourth column is empty).  For 16 bits p is the sum of two bf16 numbers (2^-16).
// Measured: four sequences of 131072 tokens, 32/8 heads of 128, INT8: 1.11 GB in 192 us, 5.8 TB/s; 64 ragged ones up to 8192, bf16: 585 MB in
// 134 us, 4.4 TB/s; one of 517 tokens 9.1 us, of which a launch is 3.6 and the rest five reads that wait for each other.
// ---------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(2))) long i64x2_t;
// x of the neighbours in a quad of lanes (xor 1, xor 2), without the LDS.
template <int CTRL>
__device__ __forceinline__ float quad_swap(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += quad_swap<0xB1>(x);
  return x + quad_swap<0x4E>(x);
}
// Over the four groups of 16 lanes.  A swap of x with itself leaves every lane its own value and that of the lane 16 (32) from it.
template <typename F>
__device__ __forceinline__ uint32_t groups_fold(uint32_t x, F f) {
  auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f(y[0], y[1]);
  auto z = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f(z[0], z[1]);
}
__device__ __forceinline__ float groups_max(float x) {
  return __uint_as_float(groups_fold(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float groups_sum(float x) {
  return __uint_as_float(groups_fold(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ uint32_t groups_max_u(uint32_t x) {
  return groups_fold(x, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// Infinities and NaN among the values that rows see, in a 16-bit cache (a row of an INT8 cache that holds one is NaN as a whole).  A product with
// a weight of zero, of a token that a row does not see or that fp32 holds no more, would make them NaN, so the products need not get them
// right: a sum that one of them has entered is never finite again, and a wavefront that ends with such a sum, or that has left some of them out,
// looks at its tokens a second time, without weights.  What it finds decides those elements.
// Over tiles of 32 tokens from `from` (a multiple of 32) to before `to`, `step` apart: found(t0, up, down) where there are any, of element lane +
// 64 w in word w: which of the tile's tokens are +infinity or NaN, and which -infinity or NaN.
template <int NK, typename F>
__device__ __forceinline__ void find_nonfinite(const kv_view& v, int b, int kvh, int from, int to, int step, F found) {
  constexpr int NW = (NK + 1) / 2;
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int t0 = from; t0 < to; t0 += step) {
    uint32_t up[NW], down[NW], any = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) up[w] = down[w] = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = t0 + 16 * i, page = t < to ? kv_page_id(v, b, t) : -1;
      if (page < 0) continue;
      const uint8_t* at = kv_head(v, page, kvh) + v.part_bytes + (size_t)(t & ((1 << v.page_shift) - 1)) * (NK * 64);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int d = lane + 64 * w;
        if (d >= NK * 32) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const i32x4_t x = reinterpret_cast<const i32x4_t*>(at + d * 32)[j];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float y = __uint_as_float(k & 1 ? (uint32_t)x[k >> 1] & 0xffff0000u : (uint32_t)x[k >> 1] << 16);
            up[w] |= (uint32_t)!(y < INFINITY) << (16 * i + 8 * j + k);
            down[w] |= (uint32_t)!(y > -INFINITY) << (16 * i + 8 * j + k);
          }
        }
        any |= up[w] | down[w];
      }
    }
    if (__any(any != 0)) found(t0, up, down);
  }
}
// Tokens t0 .. t0 + 31 as a mask, those from lo to before hi.
__device__ __forceinline__ uint32_t tokens_within(int t0, int lo, int hi) {
  const int a = min(max(lo - t0, 0), 32), z = min(max(hi - t0, 0), 32);
  return (uint32_t)(((uint64_t)1 << z) - 1) & ~(uint32_t)(((uint64_t)1 << a) - 1);
}

// Sums of pieces join by weight; one that an infinity or a NaN decides keeps it whatever its piece weighs.
__device__ __forceinline__ float join_sum(float o, float x, float weight) { return o + (__builtin_isfinite(x) ? x * weight : x); }
// (a row all of whose scores are -infinity, sum 0, is NaN)
__device__ __forceinline__ float quotient(float o, float sum) { return sum == 0.0f ? __uint_as_float(0x7fc00000u) : o / sum; }

struct decode_args {
  kv_view v;
  const uint16_t* Q;
  int64_t qs;
  int heads, group, head_blocks, block_heads, window, chunk, n_chunks;
  float scale;                   // times log2 e
  uint16_t* O;
  float* lse;
  float *part_o, *part_ml;       // [b][head][chunk][dp], [b][head][chunk][2]: pieces of sequences that are cut
};

// The tokens of sequence b that its row sees, and where its pieces begin: pieces of `chunk` tokens from lo rounded down to a tile.
struct decode_range { int lo, hi, t0, pieces; };
__device__ __forceinline__ decode_range decode_seq(const decode_args& a, int b) {
  const int len = max(a.v.lens[b], 0);
  decode_range r;
  r.hi = min(len, a.v.max_pages << a.v.page_shift);
  r.lo = a.window > 0 ? max(0, len - a.window) : 0;
  if (r.lo >= r.hi) r.lo = r.hi = 0;   // (sees nothing: a window behind what the table holds may lie at the end of 32 bits)
  r.t0 = r.lo & ~63;
  r.pieces = r.hi <= r.lo ? 1 : min((r.hi - r.t0 + a.chunk - 1) / a.chunk, a.n_chunks);
  return r;
}

template <int KIND, int NK, int W>
__global__ __launch_bounds__(W * 64, NK <= 4 ? 2 : 1) void attn_decode_kernel(decode_args a) {
  constexpr bool I8 = KIND == PQ_KV_INT8;
  constexpr int DP = NK * 32, ND = DP / 16;
  constexpr int TT = 64;                                      // tokens of a tile
  constexpr int KS = I8 ? DP / 64 : NK, TAIL = I8 ? NK % 2 : 0;   // steps of the scores' contraction, and a half one
  const kv_view& v = a.v;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  // element of a lane's j-th word of a row
  constexpr int QW = NK * 4;
  auto q_at = [&](int j) { return I8 ? (j < 8 * KS ? (j >> 3) * 64 + g * 16 + 2 * (j & 7) : KS * 64 + g * 8 + 2 * (j - 8 * KS)) : (j >> 2) * 32 + g * 8 + 2 * (j & 3); };
  // (piece, b, key-value head), with the head blocks of one of them 8 workgroups apart: on the same XCD, whose L2 holds the tiles.  The
  // last pieces, which only the longest sequences have, come first.
  const int blk = blockIdx.x, r = (blk / (8 * a.head_blocks)) * 8 + (blk & 7), hb = (blk >> 3) % a.head_blocks;
  const int pairs = v.n_seqs * v.n_kv_heads;
  if (r >= pairs * a.n_chunks) return;
  const int z = a.n_chunks - 1 - r / pairs, bh = r % pairs, kvh = bh % v.n_kv_heads, b = bh / v.n_kv_heads;
  const int cap = v.max_pages << v.page_shift;
  const int32_t* table = v.table + (size_t)b * v.max_pages;
  // group g of lanes looks up the page of tokens t0 + 16 g ..
  auto pages_at = [&](int t0) {
    const int tg = t0 + 16 * g;
    return tg < cap ? table[tg >> v.page_shift] : -1;
  };
  int page_next = a.window == 0 ? pages_at(z * a.chunk + wave * TT) : -1;     // (before the length is there)
  // the rows of this workgroup's heads, as they lie in memory: all that does not wait for the length is under way before it is there
  const int n_heads = min(a.block_heads, a.group - hb * a.block_heads);
  const int first_head = kvh * a.group + hb * a.block_heads;
  const int hl = I8 ? col >> 2 : col;                          // this column's head
  const bool mine = hl < n_heads;
  const uint16_t* q = a.Q + b * a.qs + (size_t)(first_head + (mine ? hl : 0)) * v.d;
  uint32_t qraw[QW];
#pragma unroll
  for (int j = 0; j < QW; ++j) {
    const int d = q_at(j);
    qraw[j] = *reinterpret_cast<const uint32_t*>(q + (d < v.d ? d : 0));
  }
  const decode_range R = decode_seq(a, b);
  if (z >= R.pieces) return;
  const int begin = R.t0 + z * a.chunk, end = z + 1 == R.pieces ? R.hi : begin + a.chunk;
  if (a.window != 0) page_next = pages_at(begin + wave * TT);
  const int slot_mask = (1 << v.page_shift) - 1;
  const size_t page_bytes = v.head_bytes * v.n_kv_heads;
  const uint8_t* pool = v.cache + (size_t)kvh * v.head_bytes;

  // ---- a tile in registers: the keys of the next one are under way while this one's probabilities and values are worked on, its values
  // while the next scores are
  constexpr int NF = I8 ? 4 * (KS > 0 ? KS : 1) : 4 * NK;
  i32x4_t kf[NF], vf[ND * (I8 ? 1 : 2)];
  long kt[4];
  float ks_[16], vs_[16];
  auto load_keys = [&](int t0, int page) {
    if constexpr (I8) {
      const uint8_t* kp = pool + (size_t)__shfl(page, 16 * (col >> 2), 64) * page_bytes + (size_t)((t0 + 16 * (col >> 2) + (col & 3)) & slot_mask) * DP;
      const float* sp = reinterpret_cast<const float*>(pool + (size_t)page * page_bytes + 2 * (size_t)v.part_bytes) + ((t0 + 16 * g) & slot_mask);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[c * KS + ks] = *reinterpret_cast<const i32x4_t*>(kp + c * 4 * DP + ks * 64 + g * 16);
        if constexpr (TAIL) kt[c] = *reinterpret_cast<const long*>(kp + c * 4 * DP + KS * 64 + g * 8);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4_t x = reinterpret_cast<const f32x4_t*>(sp)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) ks_[4 * i + j] = x[j];
      }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* kp = pool + (size_t)__shfl(page, 16 * (2 * u + (col >> 3)), 64) * page_bytes +
                            (size_t)((t0 + 32 * u + 8 * (col >> 2) + (col & 3)) & slot_mask) * (2 * DP) + g * 16;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int ks = 0; ks < NK; ++ks) kf[(2 * u + w) * NK + ks] = *reinterpret_cast<const i32x4_t*>(kp + w * 4 * 2 * DP + ks * 64);
      }
    }
  };
  auto load_values = [&](int t0, int page) {
    if constexpr (I8) {
      const uint8_t* base = pool + (size_t)page * page_bytes;
      const uint8_t* vp = base + v.part_bytes + (size_t)((t0 + 16 * g) & slot_mask) * DP + col * 16;
      const float* sp = reinterpret_cast<const float*>(base + 2 * (size_t)v.part_bytes) + slot_mask + 1 + ((t0 + 16 * g) & slot_mask);
#pragma unroll
      for (int i = 0; i < ND; ++i) vf[i] = *reinterpret_cast<const i32x4_t*>(vp + i * 256);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4_t x = reinterpret_cast<const f32x4_t*>(sp)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) vs_[4 * i + j] = x[j];
      }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* vp = pool + (size_t)__shfl(page, 16 * (2 * u + (g >> 1)), 64) * page_bytes + v.part_bytes +
                            (size_t)((t0 + 32 * u + 16 * (g >> 1)) & slot_mask) * (2 * DP) + col * 32 + (g & 1) * 16;
#pragma unroll
        for (int i = 0; i < ND; ++i) vf[u * ND + i] = *reinterpret_cast<const i32x4_t*>(vp + i * 512);
      }
    }
  };
  auto there_of = [&](int t0, int page) { return t0 + 16 * g < R.hi && (unsigned)page < (unsigned)v.n_pages; };
  int t0 = begin + wave * TT;
  bool there = there_of(t0, page_next);
  if (t0 < end) {
    const int page = there ? page_next : 0;
    load_keys(t0, page);
    load_values(t0, page);
    page_next = pages_at(t0 + W * TT);
  }

  // ---- the queries as the matrix instructions' second operand: column = head (bf16) or head and digit (INT8)
  i32x4_t qf[KS > 0 ? KS : 1];
  long qt;
  float qw;                                               // what one unit of a score's integer stands for, for this column's digit
  const int digit = lane & 3;
  const float digit_w = digit == 0 ? 1.0f : digit == 1 ? 256.0f : digit == 2 ? 65536.0f : 0.0f;
  if constexpr (I8) {
    // q in 23 bits relative to the power of two above its largest element, in three digits of base 256
    float x[NK * 8];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < QW; ++j) {
      const uint32_t w = mine && q_at(j) < v.d ? qraw[j] : 0;
      x[2 * j] = __uint_as_float(w << 16);
      x[2 * j + 1] = __uint_as_float(w & 0xffff0000u);
    }
#pragma unroll
    for (int j = 0; j < NK * 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    top = groups_max_u(top);
    const bool bad = top >= 0x7f800000u;
    const int eb = max((int)(top >> 23), 27);                // |x| < 2^(eb - 126)
    const float fac = bad ? 0.0f : __uint_as_float((uint32_t)(275 - eb) << 23);
    qw = bad ? __uint_as_float(0x7fc00000u) : digit_w * a.scale * __uint_as_float((uint32_t)(eb - 21) << 23);
    auto digits4 = [&](int at) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n = bad ? 0 : (int)rintf(x[at + j] * fac);
        w |= ((((uint32_t)(n + 0x808080) >> (8 * digit)) & 0xff) ^ 0x80) << (8 * j);
      }
      return digit == 3 ? 0u : w;
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int j = 0; j < 4; ++j) qf[ks][j] = (int)digits4(ks * 16 + 4 * j);
    if constexpr (TAIL) qt = (long)(((uint64_t)digits4(KS * 16 + 4) << 32) | digits4(KS * 16));
  } else {
    qw = a.scale;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int j = 0; j < 4; ++j) qf[ks][j] = mine && q_at(4 * ks + j) < v.d ? (int)qraw[4 * ks + j] : 0;
  }

  f32x4_t acc[ND];
  float m = -INFINITY, l = 0.0f;
  uint32_t seen = 0;
#pragma unroll
  for (int i = 0; i < ND; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  while (t0 < end) {
    const bool full = t0 >= R.lo && t0 + TT <= end && __all(there);
    const int t_next = t0 + W * TT;
    const bool more = t_next < end, there_next = more && there_of(t_next, page_next);
    const int page = there_next ? page_next : 0;
    // Scores: register 4 c + i of group g is the token whose value the group's lanes hold, 16 g + 4 c + i (INT8) or, by 32 tokens,
    // 8 g + k % 8: the keys' rows are read in the order that makes it so.
    float s[16];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if constexpr (I8) {
          i32x4_t S = {0, 0, 0, 0};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            // (A sum takes one kind of instruction: one that goes on in the other, 16x16x32 behind 16x16x64 or the reverse, loses two of its four
            // registers, for want of wait states between them.  With a half step all of them are 16x16x32, on the halves of a piece.)
            if constexpr (!TAIL) {
              S = __builtin_amdgcn_mfma_i32_16x16x64_i8(kf[c * KS + ks], qf[ks], S, 0, 0, 0);
            } else {
              const i64x2_t x = __builtin_bit_cast(i64x2_t, kf[c * KS + ks]), y = __builtin_bit_cast(i64x2_t, qf[ks]);
              S = __builtin_amdgcn_mfma_i32_16x16x32_i8(x[0], y[0], S, 0, 0, 0);
              S = __builtin_amdgcn_mfma_i32_16x16x32_i8(x[1], y[1], S, 0, 0, 0);
            }
          }
          if constexpr (TAIL) S = __builtin_amdgcn_mfma_i32_16x16x32_i8(kt[c], qt, S, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[4 * c + i] = quad_sum((float)S[i] * qw) * ks_[4 * c + i];
        } else {
          f32x4_t S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < NK; ++ks)
            S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[c * NK + ks]), __builtin_bit_cast(bf16x8_t, qf[ks]), S, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[4 * c + i] = S[i] * qw;
        }
      }
    if (more) load_keys(t_next, page);
    // which of the lane's 16 tokens the row sees (all of them in most tiles); token of register k
    auto token = [&](int k) { return I8 ? 16 * g + k : 32 * (k >> 3) + 8 * g + (k & 7); };
    uint32_t mask = 0xffff;
    if (!full) {
      const uint64_t ok = __ballot(there);
      mask = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int t = token(k);
        if (t0 + t >= R.lo && t0 + t < end && ((ok >> (t & 48)) & 1)) mask |= 1u << k;
      }
      if constexpr (!I8) {   // values that nobody sees may be anything: a probability of zero does not silence an infinity
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t two = (mask >> (8 * u + 2 * j)) & 3, keep = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
#pragma unroll
            for (int i = 0; i < ND; ++i) vf[u * ND + i][j] &= (int)keep;
          }
      }
    }
    seen |= mask;
    if (!full)
#pragma unroll
      for (int k = 0; k < 16; ++k) s[k] = (mask >> k) & 1 ? s[k] : -INFINITY;
    float top = s[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = fmaxf(top, s[k]);
    const float mt = fmaxf(m, groups_max(top)), mx = mt == -INFINITY ? 0.0f : mt;
    const float keep = __builtin_amdgcn_exp2f(m - mx);
    m = mt;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      s[k] = __builtin_amdgcn_exp2f(s[k] - mx);
      sum += s[k];
    }
    l = l * keep + sum;
    if (!__all(keep == 1.0f))
#pragma unroll
      for (int i = 0; i < ND; ++i) acc[i] *= keep;
    if constexpr (I8) {
      // p times the value's step, in 23 bits relative to the power of two above the tile's largest
      uint32_t big = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        s[k] = full || ((mask >> k) & 1) ? s[k] * vs_[k] : 0.0f;
        big = max(big, __float_as_uint(s[k]));
      }
      big = groups_max_u(big);
      const int eb = min(max((int)(big >> 23), 27), 254);
      const float fac = __uint_as_float((uint32_t)(275 - eb) << 23);
      const float w = big >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : digit_w * __uint_as_float((uint32_t)(eb - 21) << 23);
      const uint32_t lo_sel = 0x0c0c0400u + 0x0101u * digit, hi_sel = 0x04000c0cu + 0x01010000u * digit;
      i32x4_t pf;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t u[4];   // the integer in the low bits of 1.5 * 2^23 + x, plus 128 in every digit
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(__builtin_fmaf(s[4 * j + i], fac, 12582912.0f)) + (0x808080u - 0x4B400000u);
        pf[j] = (int)((__builtin_amdgcn_perm(u[1], u[0], lo_sel) | __builtin_amdgcn_perm(u[3], u[2], hi_sel)) ^ 0x80808080u);
      }
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const i32x4_t o = __builtin_amdgcn_mfma_i32_16x16x64_i8(vf[i], pf, i32x4_t{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_fmaf((float)o[j], w, acc[i][j]);
      }
    } else {
      // p as the sum of two bf16 numbers
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8_t hi, lo;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          hi[k] = (__bf16)s[8 * u + k];
          lo[k] = (__bf16)(s[8 * u + k] - (float)hi[k]);
        }
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const bf16x8_t x = __builtin_bit_cast(bf16x8_t, vf[u * ND + i]);
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, lo, acc[i], 0, 0, 0);
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, hi, acc[i], 0, 0, 0);
        }
      }
    }
    if (more) {
      load_values(t_next, page);
      page_next = pages_at(t_next + W * TT);
    }
    there = there_next;
    t0 = t_next;
  }

  // ---- the wavefronts' pieces are joined through the LDS: [wave][head][dp] sums, then maximum, sum and "saw a token"
  extern __shared__ float lds[];
  float* ml = lds + (size_t)W * n_heads * DP;
  __shared__ uint32_t marks[I8 ? 1 : DP], odd[W];    // (16 bits) elements that +infinity (1), -infinity (2) or NaN (both) reaches; a wavefront has some
  const bool any = __any(seen != 0);
  const float sum = groups_sum(l);
  float zero = 0.0f;             // NaN if one of the sums is not finite
#pragma unroll
  for (int i = 0; i < ND; ++i) {
    f32x4_t x = acc[i];
    if constexpr (!I8)
#pragma unroll
      for (int j = 0; j < 4; ++j) zero = __builtin_fmaf(x[j], 0.0f, zero);
    if constexpr (I8)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = quad_sum(x[j]);
    if (hl < n_heads && (!I8 || digit == 0)) *reinterpret_cast<f32x4_t*>(lds + ((size_t)wave * n_heads + hl) * DP + i * 16 + g * 4) = x;
  }
  if (hl < n_heads && g == 0 && (!I8 || digit == 0)) {
    ml[(wave * n_heads + hl) * 2] = m;
    ml[(wave * n_heads + hl) * 2 + 1] = any ? sum : -1.0f;   // (a sum is never negative)
  }
  if constexpr (!I8) {
    const bool mine_odd = __any(zero != 0.0f);
    if (lane == 0) odd[wave] = mine_odd;
  }
  __syncthreads();
  bool marked = false;
  if constexpr (!I8) {           // (the same for all heads: they see the same tokens)
#pragma unroll
    for (int w = 0; w < W; ++w) marked |= odd[w] != 0;
    if (marked) {
      for (int d = threadIdx.x; d < DP; d += W * 64) marks[d] = 0;
      __syncthreads();
      const int from = max(R.lo, begin);
      find_nonfinite<NK>(v, b, kvh, (from & ~31) + 32 * wave, end, 32 * W, [&](int t0, const uint32_t* up, const uint32_t* down) {
        const uint32_t mask = tokens_within(t0, from, end);
#pragma unroll
        for (int w = 0; w < (NK + 1) / 2; ++w) {
          const uint32_t bits = (up[w] & mask ? 1u : 0u) | (down[w] & mask ? 2u : 0u);
          if (bits) atomicOr(&marks[lane + 64 * w], bits);
        }
      });
      __syncthreads();
    }
  }
  const bool whole = R.pieces == 1;
  for (int e = threadIdx.x; e < n_heads * DP; e += blockDim.x) {
    const int hl = e / DP, d = e % DP;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, ml[(w * n_heads + hl) * 2]);
    const float mx = M == -INFINITY ? 0.0f : M;
    float sum = 0.0f, o = 0.0f;
    bool some = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {                              // (a wavefront that saw nothing left zeros)
      const float lw = ml[(w * n_heads + hl) * 2 + 1], f = lw < 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ml[(w * n_heads + hl) * 2] - mx);
      some |= !(lw < 0.0f);
      sum += lw * f;
      o += lds[((size_t)w * n_heads + hl) * DP + d] * f;
    }
    if constexpr (!I8)
      if (marked && marks[d]) o = (marks[d] & 1 ? INFINITY : 0.0f) - (marks[d] & 2 ? INFINITY : 0.0f);
    const int h = first_head + hl;
    if (whole) {
      if (d < v.d) a.O[((size_t)b * a.heads + h) * v.d + d] = f32_to_bf16(some ? quotient(o, sum) : 0.0f);
      if (d == 0 && a.lse) a.lse[(size_t)b * a.heads + h] = some ? (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : -INFINITY;
    } else {
      const size_t at = ((size_t)b * a.heads + h) * a.n_chunks + z;
      a.part_o[at * DP + d] = o;
      if (d == 0) { a.part_ml[at * 2] = M; a.part_ml[at * 2 + 1] = some ? sum : -1.0f; }
    }
  }
}

// Joins the pieces of one row and head.  The weights of up to 1024 pieces are formed side by side; then 256 / `width` groups of threads take the
// pieces g, g + groups, .. of their elements, and the groups are added in their order.  What bounds it is the latency of reads behind each other,
// so the first pieces are under way before the length says how many there are (32 pieces of 128 rows of 128: 9.2 us with one thread an
// element that walks through the pieces, 4.8 so).
constexpr int MAX_PIECES = 1024, EARLY = 16;
__global__ __launch_bounds__(256) void attn_join_kernel(decode_args a, int width) {
  const int b = blockIdx.x / a.heads, h = blockIdx.x % a.heads, t = threadIdx.x, lane = t & 63;
  __shared__ float weight[MAX_PIECES], part_l[MAX_PIECES], part[2][256], most[4];
  const size_t at = ((size_t)b * a.heads + h) * a.n_chunks;
  const float *ml = a.part_ml + at * 2, *po = a.part_o + at * a.v.dp;
  const int d = t % width, groups = 256 / width, g0 = t / width;
  const float m0 = ml[2 * min(t, a.n_chunks - 1)], l0 = ml[2 * min(t, a.n_chunks - 1) + 1];
  float early[EARLY];
#pragma unroll
  for (int i = 0; i < EARLY; ++i) early[i] = po[(size_t)min(g0 + i * groups, a.n_chunks - 1) * a.v.dp + min(d, a.v.dp - 1)];
  const decode_range R = decode_seq(a, b);
  if (R.pieces == 1) return;                                   // written by the kernel before
  float M = -INFINITY;
  for (int z = t; z < R.pieces; z += 256) {
    weight[z] = z == t ? m0 : ml[2 * z];
    part_l[z] = z == t ? l0 : ml[2 * z + 1];
    M = fmaxf(M, weight[z]);
  }
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) M = fmaxf(M, __shfl_xor(M, i, 64));
  if (lane == 0) most[t >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
  const float mx = M == -INFINITY ? 0.0f : M;
  int saw = 0;
  for (int z = t; z < R.pieces; z += 256) {                    // (a piece that saw nothing holds zeros)
    const bool none = part_l[z] < 0.0f;
    saw |= !none;
    weight[z] = none ? 0.0f : __builtin_amdgcn_exp2f(weight[z] - mx);
    part_l[z] *= weight[z];
  }
  const bool some = __syncthreads_or(saw);
  float sum = 0.0f, o = 0.0f;
#pragma unroll
  for (int i = 0; i < EARLY; ++i) {
    const int z = g0 + i * groups;
    if (z < R.pieces) {
      sum += part_l[z];
      o = join_sum(o, early[i], weight[z]);
    }
  }
#pragma unroll 8
  for (int z = g0 + EARLY * groups; z < R.pieces; z += groups) {
    sum += part_l[z];
    o = join_sum(o, po[(size_t)z * a.v.dp + min(d, a.v.dp - 1)], weight[z]);
  }
  part[0][t] = o;
  part[1][t] = sum;
  __syncthreads();
  if (t >= width) return;
  for (int g = 1; g < groups; ++g) {
    o += part[0][g * width + d];
    sum += part[1][g * width + d];
  }
  if (d < a.v.d) a.O[((size_t)b * a.heads + h) * a.v.d + d] = f32_to_bf16(some ? quotient(o, sum) : 0.0f);
  if (d == 0 && a.lse) a.lse[(size_t)b * a.heads + h] = some ? (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : -INFINITY;
}

// How a decode call is cut: query heads a workgroup, pieces of a sequence.
struct decode_plan { int waves, head_blocks, block_heads, chunk, n_chunks; size_t part_o, part_ml, total; };
decode_plan plan_decode(const pq_attn_desc& d) {
  decode_plan p;
  const int group = d.n_heads / d.kv.n_kv_heads, dp = (d.kv.d_head + 31) / 32 * 32;
  const int64_t cap = (int64_t)d.kv.max_pages * d.kv.page_tokens;
  int64_t most = d.max_len > 0 && d.max_len < cap ? d.max_len : cap;
  if (d.window > 0 && d.window + (int64_t)63 < most) most = d.window + (int64_t)63;
  // Eight wavefronts where two of them on a SIMD hold a tile each in registers, four beyond (heads of 256, INT8: 150 / 510 us for four sequences
  // of 32768 tokens, 64/8 heads; heads of 128: 200 / 192 us for four of 131072).
  p.waves = dp <= 128 ? 8 : 4;
  // a column of the matrix instructions for a head (bf16) or a quad of columns (INT8), and 64 KiB of LDS for the wavefronts' sums and the marks
  // (at most 1040 bytes)
  const int fit = (65536 - 2048) / (p.waves * (dp + 2) * 4), hb = d.kv.kv_kind == PQ_KV_INT8 ? 4 : fit < 16 ? fit : 16;
  p.head_blocks = (group + hb - 1) / hb;
  p.block_heads = (group + p.head_blocks - 1) / p.head_blocks;
  // Pieces (at most MAX_PIECES): for 256 workgroups, one a CU, where few sequences have whole sequences' worth of work for less; for 1024, which
  // spread ragged lengths, from 65 rows of key-value heads on.  A piece is worth its start and the second launch from 1024 tokens on, or from
  // 2048 where whole sequences already occupy every CU.  (256 / 1024 workgroups, us: INT8, 8 heads of 128, one and four sequences of 131072 56 / 70
  // and 193 / 199, ragged ones in bf16, 4 up to 65536 111 / 125, 8 up to 16384 59 / 67, 16 up to 16384 107 / 95, 64 up to 8192 152 / 133; eight
  // of 2048, 32 heads of 64 in INT8: 14.8 whole, 21.4 in halves; one of 517: 9.1 whole, 11.7 in thirds.)
  const int64_t rows = (int64_t)d.kv.n_seqs * d.kv.n_kv_heads * p.head_blocks, all = rows <= 64 ? 256 : 1024;
  const int64_t want = rows > 0 ? (all + rows - 1) / rows : 1, least = rows >= 256 ? 2048 : 1024;
  int64_t chunk = (most + want - 1) / want;
  if (chunk < least) chunk = least;
  chunk = (chunk + 511) / 512 * 512;
  p.chunk = (int)chunk;
  p.n_chunks = (int)((most + chunk - 1) / chunk);
  // And four, two workgroups a CU, where there are more workgroups than CUs with less than 4096 tokens each: one starts while the other ends.  (8 / 4
  // wavefronts, us.  INT8, 32 heads of 64: 8 sequences of 2048 tokens 14.7 / 16.1, 16 of 300 and 2048 12.0 / 8.7 and 28.8 / 25.3; ragged, 8 heads of
  // 128: 16 up to 4096 25.7 / 22.6, 24 up to 8192 38.9 / 32.3, 64 up to 8192, in pieces of 4096, 85.6 / 90.3; in bf16 16 up to 16384 95 / 78 and
  // 65536 233 / 239, 64 up to 8192 133 / 144.)
  if (p.waves == 8 && rows > 64 && rows * p.n_chunks > 256 && (chunk < most ? chunk : most) < 4096) p.waves = 4;
  const size_t pieces = p.n_chunks > 1 ? (size_t)d.kv.n_seqs * d.n_heads * p.n_chunks : 0;
  p.part_o = 0;
  p.part_ml = pq_align_up(pieces * (size_t)dp * 4, 256);
  p.total = p.part_ml + pq_align_up(pieces * 8, 256);
  if (p.total < 256) p.total = 256;
  return p;
}

template <int KIND, int NK>
void launch_decode_nk(const decode_args& a, const decode_plan& p, unsigned grid, hipStream_t s) {
  const size_t lds = p.waves * (size_t)p.block_heads * (NK * 32 + 2) * 4;
  if constexpr (NK <= 4)
    if (p.waves == 8) {
      attn_decode_kernel<KIND, NK, 8><<<grid, 512, lds, s>>>(a);
      return;
    }
  attn_decode_kernel<KIND, NK, 4><<<grid, 256, lds, s>>>(a);
}
template <int KIND>
void launch_decode(const decode_args& a, const decode_plan& p, unsigned grid, hipStream_t s) {
  switch (a.v.dp / 32) {
    case 1: launch_decode_nk<KIND, 1>(a, p, grid, s); break;
    case 2: launch_decode_nk<KIND, 2>(a, p, grid, s); break;
    case 3: launch_decode_nk<KIND, 3>(a, p, grid, s); break;
    case 4: launch_decode_nk<KIND, 4>(a, p, grid, s); break;
    case 5: launch_decode_nk<KIND, 5>(a, p, grid, s); break;
    case 6: launch_decode_nk<KIND, 6>(a, p, grid, s); break;
    case 7: launch_decode_nk<KIND, 7>(a, p, grid, s); break;
    default: launch_decode_nk<KIND, 8>(a, p, grid, s); break;
  }
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
  PQ_REQUIRE(T <= (1 << 29) && (int64_t)T * d->n_heads <= 0x7fffffff, PQ_ERR_SHAPE, "%d rows of %d heads are too many for one call", T, d->n_heads);
  return PQ_OK;
}

// ---------------------------------------------------------------------------------------------
// The rows of prompts
//
// A workgroup has 128 rows (token by query head of one key-value head: the heads that share keys are rows of the same tile), 32 a wavefront, and
// takes the tokens in stages that all four wavefronts share through two buffers of LDS; codes become bf16 on their way there (exact), so both
// products run on the bf16 instructions.  Scores are formed transposed, a column a row of Q, so that a row's maximum and sum need one
// exchange between two lanes and the probabilities are the second product's operand as they stand.  Probabilities (times the value's step)
// are rounded to bf16, 2^-9 of each: what a 16-bit product takes (error of the outputs 2.1e-3, 1.6e-3 of it from their own rounding).
// Bound by the sum of what a stage costs one after the other with two wavefronts a SIMD.  8192 tokens, 32/8 heads of 128, INT8: 623 to 653 us on
// different cards (842 to 882 TFLOP/s of the causal products); where it took 630, its matrix instructions alone 253, with the LDS reads 354, with
// the staging 477.
// ---------------------------------------------------------------------------------------------
struct prefill_args {
  kv_view v;
  const uint16_t* Q;
  int64_t qs;
  int heads, group, causal, window, tiles;
  float scale;                   // times log2 e
  uint16_t* O;
  float* lse;
};

// Tokens of a stage.  16-bit heads beyond 64 take half: their stage on its way through the registers beside 64 scores a row spills (8192 tokens,
// 32/8 heads of 128: 1.72 ms with 64, 0.73 with 32; heads of 64: 139 us for four prompts of 2048 with 64, 153 with 32).
template <int KIND, int NK> constexpr int prefill_tokens() { return KIND == PQ_KV_BF16 && NK > 2 ? 32 : 64; }
// Bytes of a key row and a value row of a stage in the LDS (16 more than they hold: sixteen rows' pieces of 16 bytes lie in different
// banks), and of the stage with both steps and a flag a wavefront.
template <int NK> constexpr int prefill_krow() { return NK * 64 + 16; }
template <int KIND, int NK> constexpr int prefill_vrow() { return 2 * prefill_tokens<KIND, NK>() + 16; }
template <int KIND, int NK> constexpr int prefill_stage() {
  return prefill_tokens<KIND, NK>() * (prefill_krow<NK>() + 8) + NK * 32 * prefill_vrow<KIND, NK>() + 16;
}

// Order of a run of N LDS reads and as many products on them: four reads ahead.
template <int N>
__device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
  for (int i = 0; i < N - 4; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
}

// Four codes as bf16 (every code has at most eight significant bits: exact).
__device__ __forceinline__ uint2 codes_bf16(int w) {
  const uint32_t a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8)), c = __float_as_uint((float)(int8_t)(w >> 16)),
                 d = __float_as_uint((float)(w >> 24));
  return make_uint2(__builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u));
}
__device__ __forceinline__ bool has_nonfinite(uint32_t two) { return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u; }

// The first token that a row at `pos` sees; a window is up to 2^31 - 1 and a position may be negative.
__device__ __forceinline__ int first_seen(const prefill_args& a, int pos) { return a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0; }

// Elements of the 32x32 products' columns (register 4 q + j of half h of block i is element 32 i + 8 q + 4 h + j) that infinities and NaN which
// the column's row sees reach: bit 4 q + j of reach[i] for +infinity, of its high half for -infinity, both for NaN.  The row sees tokens `low` .. `lim`.
template <int NK>
__device__ __forceinline__ void find_reach(const kv_view& v, int b, int kvh, int from, int to, int step, int low, int lim, uint32_t* reach) {
  const int h = (threadIdx.x & 63) >> 5;
  find_nonfinite<NK>(v, b, kvh, from, to, step, [&](int t0, const uint32_t* up, const uint32_t* down) {
    const uint32_t mask = tokens_within(t0, low, lim + 1);
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll 1
      for (int k = 0; k < 16; ++k) {
        const int from_lane = 32 * (i & 1) + 8 * (k >> 2) + 4 * h + (k & 3);
        const uint32_t u = (uint32_t)__shfl((int)up[i >> 1], from_lane, 64) & mask, d = (uint32_t)__shfl((int)down[i >> 1], from_lane, 64) & mask;
        reach[i] |= ((u ? 1u : 0u) | (d ? 0x10000u : 0u)) << k;
      }
  });
}
// Whether one of the lane's sums is infinite or NaN.
template <int NK>
__device__ __forceinline__ bool any_nonfinite(const f32x16_t* acc) {
  float z = 0.0f;
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) z = __builtin_fmaf(acc[i][j], 0.0f, z);
  return z != 0.0f;              // (NaN: not equal)
}
// An element from its sum and the inverse of the row's: what reaches it decides, in a row that is not NaN by its scores (inv: NaN, or infinite where
// all of them are -infinity).
__device__ __forceinline__ float settle(float sum, float inv, bool up, bool down) {
  float x = up || down ? inv * 0.0f : sum * inv;
  if (up) x += INFINITY;
  if (down) x -= INFINITY;
  return x;
}

// Which sequence and which of its tiles of ROWS rows workgroup `vt` of the call has (b < 0: none).  Up to 8 sequences are taken in the order of the
// tokens that their last tiles see, most first, and a sequence's last tiles first, so that long tiles do not start when the others end.  Beyond
// that: virtual tiles, of which sequence b owns those from floor(first row / ROWS) + b on, at least as many as it has, the last ones first.
// (INT8, heads of 90, 32 of them, sorted / not: seven ragged prompts up to 1500 rows 81 / 84 us with a window, 86 / 91 without; eight of 512
// 48.8 / 46.5, of 128 12.8 / 14.2; 16 and 32 of 128, 19.7 / 18.1 and 42 / 31: each sequence costs every wavefront a step of the loop.)
struct tile_place { int b, tile; kv_rows r; };
template <int ROWS>
__device__ __forceinline__ tile_place find_tile(const prefill_args& a, int vt) {
  const kv_view& v = a.v;
  const int lane = threadIdx.x & 63;
  tile_place w;
  w.b = -1;
  if (v.n_seqs <= 8) {
    const kv_rows mine = kv_seq_rows(v, min(lane, v.n_seqs - 1));
    const int tiles = lane < v.n_seqs ? (int)(((int64_t)mine.n * a.group + ROWS - 1) / ROWS) : 0;
    const int sees = a.window > 0 && a.window < mine.len ? min(mine.len, a.window + ROWS) : mine.len;
    int before = 0;                    // tiles of the sequences that come first
    for (int i = 0; i < v.n_seqs; ++i) {
      const int s = __builtin_amdgcn_readlane(sees, i), n = __builtin_amdgcn_readlane(tiles, i);
      before += s > sees || (s == sees && i < lane) ? n : 0;
    }
    const uint64_t hit = __ballot(vt >= before && vt < before + tiles);
    if (hit == 0) return w;
    w.b = __builtin_ctzll(hit);
    w.r.r0 = __builtin_amdgcn_readlane(mine.r0, w.b);
    w.r.n = __builtin_amdgcn_readlane(mine.n, w.b);
    w.r.len = __builtin_amdgcn_readlane(mine.len, w.b);
    w.r.first = __builtin_amdgcn_readlane(mine.first, w.b);
    w.tile = __builtin_amdgcn_readlane(before + tiles, w.b) - 1 - vt;
  } else {
    vt = a.tiles - 1 - vt;
    auto start = [&](int r0, int i) { return r0 * a.group / ROWS + i; };
    const int b = kv_find_rows(v, vt, w.r, start);
    if (b < 0) return w;
    w.tile = vt - start(w.r.r0, b);
    if (w.r.n > 0 && w.tile <= (w.r.n * a.group - 1) / ROWS) w.b = b;
  }
  return w;
}

// Eight elements of a row of d from element `at` on, zeros behind its end (rows of 8 and more: one load of 16 bytes that ends with the row).
typedef int i32x4_a4_t __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ i32x4_t row_piece(const uint16_t* q, int d, int at) {
  i32x4_t x;
  if (d >= 8) {
    const int from = min(at, d - 8), shift = (at - from) >> 1;
    x = *reinterpret_cast<const i32x4_a4_t*>(q + from);
    if (shift & 1) x = i32x4_t{x[1], x[2], x[3], 0};
    if (shift & 2) x = i32x4_t{x[2], x[3], 0, 0};
    if (shift >= 4) x = i32x4_t{0, 0, 0, 0};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int w = *reinterpret_cast<const int*>(q + (at + 2 * j < d ? at + 2 * j : 0));
      x[j] = at + 2 * j < d ? w : 0;
    }
  }
  return x;
}
// Four outputs from element `at` of a row of d on, as many as it has.
typedef uint32_t u32x2_a4_t __attribute__((ext_vector_type(2), aligned(4)));
__device__ __forceinline__ void store_quad(uint16_t* row, int d, int at, const float* x) {
  const uint32_t lo = pack_bf16x2(x[0], x[1]), hi = pack_bf16x2(x[2], x[3]);
  if (at + 4 <= d) *reinterpret_cast<u32x2_a4_t*>(row + at) = u32x2_a4_t{lo, hi};
  else if (at < d) *reinterpret_cast<uint32_t*>(row + at) = lo;
}

template <int KIND, int NK>
__global__ __launch_bounds__(256, NK <= 4 ? 2 : 1) void attn_prefill_kernel(prefill_args a) {
  constexpr bool I8 = KIND == PQ_KV_INT8;
  constexpr int TOK = prefill_tokens<KIND, NK>(), DP = NK * 32, ES = I8 ? 1 : 2, NS = NK * 2;
  constexpr int KROW = prefill_krow<NK>(), VROW = prefill_vrow<KIND, NK>(), STAGE = prefill_stage<KIND, NK>();
  constexpr int W = 4, THREADS = W * 64, ROWS = W * 32, U = TOK / 32, NB = TOK / 16, ALL = (1 << NB) - 1;
  // Pieces of a stage's keys (or values): 16 bytes, or 8 where that gives every thread as many.
  constexpr int PB = TOK * DP * ES % (16 * THREADS) == 0 ? 16 : 8, CT = TOK * DP * ES / (PB * THREADS);
  constexpr int ROW_PIECES = DP * ES / PB, BLOCK_PIECES = 16 * DP * ES / PB, PT = PB / ES;      // of a key, of 16 tokens' values; tokens of a piece
  static_assert(CT * PB * THREADS == TOK * DP * ES, "whole pieces");
  typedef __attribute__((ext_vector_type(PB / 4))) int piece_t;
  extern __shared__ uint8_t lds8[];
  const kv_view& v = a.v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), h = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.x % v.n_kv_heads;                       // (one key-value head of every eight on an XCD)
  const tile_place w = find_tile<ROWS>(a, blockIdx.x / v.n_kv_heads);
  if (w.b < 0) return;
  const kv_rows r = w.r;
  const int b = w.b, all_rows = r.n * a.group, row0 = w.tile * ROWS;
  const int cap = v.max_pages << v.page_shift, hi = min(r.len, cap);
  auto pos_of = [&](int row) { return r.first + row / a.group; };
  const int rows_here = min(ROWS, all_rows - row0);
  const int pos_first = pos_of(row0), pos_last = pos_of(row0 + rows_here - 1);
  const int t_begin = first_seen(a, pos_first) & ~(TOK - 1);
  const int t_end = pos_last < 0 ? 0 : a.causal ? min(pos_last + 1, hi) : hi;

  // this lane's row, and what the wavefront's rows see between them
  const bool active = wave * 32 < rows_here, mine = wave * 32 + col < rows_here;
  const int row = row0 + (mine ? wave * 32 + col : 0);
  const int pos = mine ? pos_of(row) : -1, head = kvh * a.group + row % a.group;
  const size_t trow = (size_t)r.r0 + row / a.group;
  const int lim = pos < 0 ? -1 : a.causal ? min(pos, hi - 1) : hi - 1, low = first_seen(a, pos);
  const int wfirst = active ? pos_of(row0 + wave * 32) : 0, wlast = active ? pos_of(row0 + min(wave * 32 + 32, rows_here) - 1) : -1;
  const int w_end = wlast < 0 ? 0 : a.causal ? min(wlast + 1, hi) : hi;                 // some row sees up to here
  const int w_all_end = wfirst < 0 ? 0 : a.causal ? min(wfirst + 1, hi) : hi;           // every row sees up to here ..
  const int w_begin = first_seen(a, wfirst), w_all_begin = first_seen(a, wlast);   // .. from here

  // ---- staging: pages of a stage's blocks of 16 tokens in the first lanes of every wavefront, one stage ahead of the loads
  const int slot_mask = (1 << v.page_shift) - 1;
  const int32_t* table = v.table + (size_t)b * v.max_pages;
  const uint8_t* pool = v.cache + (size_t)kvh * v.head_bytes;
  const size_t page_bytes = v.head_bytes * v.n_kv_heads;
  auto pages_at = [&](int t0) {
    const int t = t0 + 16 * (lane & (NB - 1));
    int p = -1;
    if (t < t_end) p = table[t >> v.page_shift];
    return p;                    // (looked at a stage later: a wait for it here would wait for the stage's loads too)
  };
  const int n = t_begin < t_end ? (t_end - t_begin + TOK - 1) / TOK : 0;
  auto t_of = [&](int s) { return t_begin + s * TOK; };
  const int pages0 = pages_at(t_of(0));
  int pages = pages_at(t_of(1));

  bf16x8_t qf[NS];
#pragma unroll
  for (int ks = 0; ks < NS; ++ks) {
    const i32x4_t x = row_piece(a.Q + trow * a.qs + (size_t)head * v.d, v.d, ks * 16 + h * 8);
    qf[ks] = __builtin_bit_cast(bf16x8_t, mine ? x : i32x4_t{0, 0, 0, 0});
  }
  f32x16_t acc[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;
  float m = 0.0f, l = 0.0f;      // reference of the exponentials (log2), their sum over this lane's tokens
  uint32_t seen = 0;             // not zero: the row has seen a token
  bool set = !mine;              // .. and one whose score is not -infinity: m is a score's (a lane without a row asks for nothing)

  piece_t kreg[CT], vreg[CT];
  float steps = 0.0f;
  // Where a stage lies: which of its blocks have a page, and the pages with those that are missing as page 0; where a page holds the
  // whole stage, its address.
  struct place { int safe; uint32_t there; const uint8_t* at; };
  const bool one_page = (1 << v.page_shift) >= TOK;
  auto place_of = [&](int t0, int pages) {
    const bool ok = (unsigned)pages < (unsigned)v.n_pages;
    place w;
    w.there = (uint32_t)__ballot(ok) & ALL;
    w.safe = ok ? pages : 0;
    w.at = pool + (size_t)__builtin_amdgcn_readfirstlane(w.safe) * page_bytes;
    return w;
  };
  auto load_stage = [&](int t0, const place& w) {
    if (one_page) {              // a thread's place in the stage does not change
      const uint8_t* at = w.at + (size_t)((t0 & slot_mask) * (DP * ES));
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const int i = threadIdx.x + THREADS * c;
        kreg[c] = *reinterpret_cast<const piece_t*>(at + i * PB);
        vreg[c] = *reinterpret_cast<const piece_t*>(at + v.part_bytes + i * PB);
      }
      if constexpr (I8)
        if (wave < 2) steps = reinterpret_cast<const float*>(w.at + 2 * (size_t)v.part_bytes)[(wave << v.page_shift) + (t0 & slot_mask) + (lane & (TOK - 1))];
    } else {
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const int i = threadIdx.x + THREADS * c;
        const int t = i / ROW_PIECES, vb = i / BLOCK_PIECES;           // keys token by token, values block by block
        const int bk = __shfl(w.safe, t >> 4, 64), bv = __shfl(w.safe, vb, 64);
        kreg[c] = *reinterpret_cast<const piece_t*>(pool + (size_t)bk * page_bytes + ((t0 + t) & slot_mask) * (DP * ES) + (i % ROW_PIECES) * PB);
        vreg[c] = *reinterpret_cast<const piece_t*>(pool + (size_t)bv * page_bytes + v.part_bytes + ((t0 + 16 * vb) & slot_mask) * (DP * ES) + (i % BLOCK_PIECES) * PB);
      }
      if constexpr (I8) {
        const int bs = __shfl(w.safe, (lane & (TOK - 1)) >> 4, 64);
        if (wave < 2) steps = reinterpret_cast<const float*>(pool + (size_t)bs * page_bytes + 2 * (size_t)v.part_bytes)[(wave << v.page_shift) + ((t0 + (lane & (TOK - 1))) & slot_mask)];
      }
    }
  };
  // `check`: whether some row of the workgroup does not see some of the stage's tokens
  auto store_stage = [&](int t0, uint8_t* buf, bool check, uint32_t there) {
    uint8_t *lk = buf, *lv = buf + TOK * KROW;
    bool bad = false;
    const bool clean = check || there != ALL;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int i = threadIdx.x + THREADS * c;
      const int t = i / ROW_PIECES, vb = i / BLOCK_PIECES, e = i % BLOCK_PIECES / (16 / PT), vt = i % (16 / PT) * PT;   // e, vt: element, first token
      const int rk = (t & 0x33) | ((t & 4) << 1) | ((t & 8) >> 1);     // see the scores' tokens below
      uint8_t *ko = lk + rk * KROW + i % ROW_PIECES * (PB * 2 / ES), *vo = lv + e * VROW + vb * 32 + vt * 2;
      if constexpr (I8) {
#pragma unroll
        for (int j = 0; j < PB / 4; j += 2) {
          const uint2 x0 = codes_bf16(kreg[c][j]), x1 = codes_bf16(kreg[c][j + 1]);
          *reinterpret_cast<uint4*>(ko + 8 * j) = make_uint4(x0.x, x0.y, x1.x, x1.y);
          const uint2 y0 = codes_bf16(vreg[c][j]), y1 = codes_bf16(vreg[c][j + 1]);
          *reinterpret_cast<uint4*>(vo + 8 * j) = make_uint4(y0.x, y0.y, y1.x, y1.y);
        }
      } else {
        *reinterpret_cast<piece_t*>(ko) = kreg[c];
        piece_t x = vreg[c];
        if (clean) {                       // tokens that are not there become zeros: a probability of zero does not silence an infinity
          const int left = (there >> vb) & 1 ? t_end - (t0 + 16 * vb + vt) : 0;
#pragma unroll
          for (int j = 0; j < PB / 4; ++j) {
            x[j] &= (int)((left > 2 * j ? 0xffffu : 0u) | (left > 2 * j + 1 ? 0xffff0000u : 0u));
            bad |= has_nonfinite((uint32_t)x[j]);
          }
        }
        *reinterpret_cast<piece_t*>(vo) = x;
      }
    }
    float* ls = reinterpret_cast<float*>(lv + DP * VROW);
    if constexpr (I8) {
      if (wave < 2 && lane < TOK) ls[wave * TOK + lane] = wave == 0 ? steps * a.scale : steps;
    } else if (clean) {
      const bool any = __any(bad);
      if (lane == 0) reinterpret_cast<int*>(ls + 2 * TOK)[wave] = any;
    }
  };
  auto partly = [&](int t0) {    // some row of the workgroup does not see all of the stage
    return t0 + TOK > (pos_first < 0 ? 0 : a.causal ? min(pos_first + 1, hi) : hi) || t0 < first_seen(a, pos_last);
  };

  // A stage for one wavefront is three steps.  Scores are formed transposed (a column is a row of Q): register k of half h is token
  // 16 (k / 8) + 8 h + k % 8, the eight tokens that the half's lanes hold of the values' second operand; the keys' rows lie in
  // the LDS in the order that makes it so.
  constexpr int P = 16 * U;      // tokens of a lane in a stage
  float p[P];
  bf16x8_t pb[NB];
  bool bad = false;              // values that are not finite in a stage that some row sees a part of: the product leaves them out
  bool left_out = false;
  auto scores = [&](const uint8_t* lk) {
    f32x16_t S[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) S[u][j] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < NS; ++ks)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(lk + (32 * u + col) * KROW + ks * 32 + h * 16);
        S[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], S[u], 0, 0, 0);
      }

    reads_ahead<NS * U>();
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) p[16 * u + j] = S[u][j];
  };
  // Probabilities relative to the row's reference m, which moves only where a score exceeds it by 16 (and where the row sees its first
  // tokens): any reference gives the same quotient, and bf16 and fp32 have the range.
  auto soften = [&](int t0, const uint8_t* lk, uint32_t blocks, bool full) {
    const uint8_t* lv = lk + TOK * KROW;
    const float* ls = reinterpret_cast<const float*>(lv + DP * VROW);
#pragma unroll
    for (int q = 0; q < 4 * U; ++q) {
      f32x4_t x = {a.scale, a.scale, a.scale, a.scale};
      if constexpr (I8) x = *reinterpret_cast<const f32x4_t*>(ls + 16 * (q >> 1) + 8 * h + 4 * (q & 1));
#pragma unroll
      for (int j = 0; j < 4; ++j) p[4 * q + j] = __builtin_fmaf(p[4 * q + j], x[j], -m);
    }
    uint32_t mask = (uint32_t)(((uint64_t)1 << P) - 1);
    if (!full) {                 // the seen tokens of every eight are those from `from` to before `to`
      mask = 0;
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const int to = min(max(lim + 1 - t0 - 8 * h - 16 * q, 0), 8), from = min(max(low - t0 - 8 * h - 16 * q, 0), 8);
        const uint32_t eight = ((1u << to) - 1) & ~((1u << from) - 1);
        mask |= ((blocks >> q) & 1 ? eight : 0u) << (8 * q);
      }
#pragma unroll
      for (int k = 0; k < P; ++k) p[k] = (mask >> k) & 1 ? p[k] : -INFINITY;
      seen |= mask | (uint32_t)__shfl_xor((int)mask, 32, 64);
    } else {
      seen = mask;
    }
    float top = fmaxf(p[0], p[1]);
#pragma unroll
    for (int k = 2; k < P; ++k) top = fmaxf(top, p[k]);
    if (!__all(set && top <= 16.0f)) {
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float delta = (set ? top > 16.0f : top != -INFINITY) ? top : 0.0f;     // (by the row alone, whatever the wavefront's others do)
      const float keep = set ? __builtin_amdgcn_exp2f(-delta) : 1.0f;      // (nothing to keep before the first scores)
      set |= top != -INFINITY;
#pragma unroll
      for (int k = 0; k < P; ++k) p[k] -= delta;
      m += delta;
      l *= keep;
#pragma unroll
      for (int i = 0; i < NK; ++i) acc[i] *= keep;
    }
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < P; ++k) {
      p[k] = __builtin_amdgcn_exp2f(p[k]);
      sum[k & 1] += p[k];
    }
    l += sum[0] + sum[1];
    if constexpr (I8) {
#pragma unroll
      for (int q = 0; q < 4 * U; ++q) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t*>(ls + TOK + 16 * (q >> 1) + 8 * h + 4 * (q & 1));
#pragma unroll
        for (int j = 0; j < 4; ++j) p[4 * q + j] *= x[j];
      }
      if (!full)                 // (a step that nobody sees may be NaN)
#pragma unroll
        for (int k = 0; k < P; ++k) p[k] = (mask >> k) & 1 ? p[k] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < NB; ++q) // rounded to bf16, the operand's type; the sum l is of the unrounded ones
#pragma unroll
      for (int j = 0; j < 8; ++j) pb[q][j] = (__bf16)p[8 * q + j];
    bad = false;
    if constexpr (!I8)
      if (!full) {
        const int* f = reinterpret_cast<const int*>(ls + 2 * TOK);
        int any = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) any |= f[w];
        bad = __builtin_amdgcn_readfirstlane(any) != 0;
        left_out |= bad;
      }
  };
  auto values = [&](const uint8_t* lk) {
    const uint8_t* lv = lk + TOK * KROW;
    if (I8 || !bad) {
#pragma unroll
      for (int q = 0; q < NB; ++q)
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          const bf16x8_t x = *reinterpret_cast<const bf16x8_t*>(lv + (32 * i + col) * VROW + q * 32 + h * 16);
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, pb[q], acc[i], 0, 0, 0);
        }

    reads_ahead<NB * NK>();
    } else {
#pragma unroll
      for (int q = 0; q < NB; ++q)
#pragma unroll
        for (int i = 0; i < NK; ++i) {
          i32x4_t x = *reinterpret_cast<const i32x4_t*>(lv + (32 * i + col) * VROW + q * 32 + h * 16);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if ((x[j] & 0x7f80) == 0x7f80) x[j] &= (int)0xffff0000;
            if ((x[j] & 0x7f800000) == 0x7f800000) x[j] &= 0xffff;
          }
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), pb[q], acc[i], 0, 0, 0);
        }
    }
  };
  auto sees = [&](int t0) { return t0 < w_end && t0 + TOK > w_begin; };
  auto sees_all = [&](int t0, uint32_t there) { return t0 >= w_all_begin && t0 + TOK <= w_all_end && there == ALL; };

  place here{0, 0, nullptr};
  if (n > 0) {
    here = place_of(t_of(0), pages0);
    load_stage(t_of(0), here);
    store_stage(t_of(0), lds8, partly(t_of(0)), here.there);
  }
  uint32_t there = here.there;
  for (int s = 0; s < n; ++s) {
    __syncthreads();
    uint32_t next = 0;
    if (s + 1 < n) {
      here = place_of(t_of(s + 1), pages);
      next = here.there;
      load_stage(t_of(s + 1), here);
      pages = pages_at(t_of(s + 2));
    }
    const uint8_t* lk = lds8 + (s & 1) * STAGE;
    if (sees(t_of(s))) {
      scores(lk);
      soften(t_of(s), lk, there, sees_all(t_of(s), there));
      values(lk);
    }
    if (s + 1 < n) store_stage(t_of(s + 1), lds8 + (~s & 1) * STAGE, partly(t_of(s + 1)), next);
    there = next;
  }
  uint32_t reach[NK];
  if constexpr (!I8) {
#pragma unroll
    for (int i = 0; i < NK; ++i) reach[i] = 0;
    if (__any(left_out || any_nonfinite<NK>(acc))) find_reach<NK>(v, b, kvh, w_begin & ~31, w_end, 32, low, lim, reach);
  }
  if (!mine) return;
  // ---- every column is a row: register 4 q + j of half h is element 8 q + 4 h + j of each 32
  l += __shfl_xor(l, 32, 64);
  const bool any = seen != 0;
  const float inv = any ? 1.0f / l : 0.0f;
  uint16_t* o = a.O + (trow * a.heads + head) * v.d;
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (I8) x[j] = any ? acc[i][4 * q + j] * inv : 0.0f;
        else x[j] = any ? settle(acc[i][4 * q + j], inv, (reach[i] >> (4 * q + j)) & 1, (reach[i] >> (16 + 4 * q + j)) & 1) : 0.0f;
      }
      store_quad(o, v.d, 32 * i + 8 * q + 4 * h, x);
    }
  if (a.lse && h == 0) a.lse[trow * a.heads + head] = any ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : -INFINITY;
}

// ---------------------------------------------------------------------------------------------
// Few rows: 32 a workgroup, the wavefronts share the tokens
// ---------------------------------------------------------------------------------------------
// The same products with the keys and values read straight from the cache into the matrix instructions' registers: wavefront w takes
// the tiles w, w + W, .. of 32 tokens, so that a row's tokens pass W times as fast, and what the wavefronts found is joined through
// the LDS.  For calls too small to fill the chip with tiles of 128 rows, whose time is that of the longest row's chain of tiles.  Bound by the
// chain of reads and products of a wavefront (130 tokens of 16 heads of 128, bf16: 10.5 us, of which a launch is 3.6), in larger calls by
// the conversions and softmax of 32 rows where the other kernel shares the conversions of 128.
template <int NK> constexpr int rows_waves() { return NK <= 4 ? 8 : 4; }
template <int NK> constexpr int rows_pitch() { return NK * 32 + 4; }       // floats: sixteen rows' pieces of 16 bytes lie in different banks
template <int KIND, int NK> constexpr int rows_lds() {                     // sums, maximum and sum of a row, elements that infinities reach
  return rows_waves<NK>() * (32 * rows_pitch<NK>() * 4 + 32 * 8 + (KIND == PQ_KV_BF16 ? NK * 256 : 0));
}

template <int KIND, int NK>
__global__ __launch_bounds__(rows_waves<NK>() * 64, NK <= 4 ? 2 : 1) void attn_rows_kernel(prefill_args a) {
  constexpr bool I8 = KIND == PQ_KV_INT8;
  constexpr int W = rows_waves<NK>(), DP = NK * 32, ES = I8 ? 1 : 2, NS = NK * 2, NF = I8 ? NK : NS, PITCH = rows_pitch<NK>();
  constexpr int ROWS = 32, TT = 32;
  const kv_view& v = a.v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), h = lane >> 5, col = lane & 31;
  const int kvh = blockIdx.x % v.n_kv_heads;
  const tile_place w = find_tile<ROWS>(a, blockIdx.x / v.n_kv_heads);
  if (w.b < 0) return;
  const kv_rows r = w.r;
  const int b = w.b, all_rows = r.n * a.group, row0 = w.tile * ROWS;
  const int cap = v.max_pages << v.page_shift, hi = min(r.len, cap);
  auto pos_of = [&](int row) { return r.first + row / a.group; };
  const int rows_here = min(ROWS, all_rows - row0);
  const int pos_first = pos_of(row0), pos_last = pos_of(row0 + rows_here - 1);
  const int t_end = pos_last < 0 ? 0 : a.causal ? min(pos_last + 1, hi) : hi;                        // some row sees up to here
  const int all_end = pos_first < 0 ? 0 : a.causal ? min(pos_first + 1, hi) : hi;                    // every row sees up to here ..
  const int all_begin = first_seen(a, pos_last);                                                     // .. from here
  const int t_begin = first_seen(a, pos_first) & ~(TT - 1);
  const int tiles = t_begin < t_end ? (t_end - t_begin + TT - 1) / TT : 0;

  const bool mine = col < rows_here;
  const int row = row0 + (mine ? col : 0);
  const int pos = mine ? pos_of(row) : -1, head = kvh * a.group + row % a.group;
  const size_t trow = (size_t)r.r0 + row / a.group;
  const int lim = pos < 0 ? -1 : a.causal ? min(pos, hi - 1) : hi - 1, low = first_seen(a, pos);

  // ---- a tile in registers: keys and values of the lane's row of the operand, and (INT8) the steps of the half's sixteen tokens
  const int slot_mask = (1 << v.page_shift) - 1;
  const int32_t* table = v.table + (size_t)b * v.max_pages;
  const uint8_t* pool = v.cache + (size_t)kvh * v.head_bytes;
  const size_t page_bytes = v.head_bytes * v.n_kv_heads;
  struct pages { int id[2]; };                   // of the tile's two blocks of 16 tokens
  auto pages_at = [&](int t0) {
    pages g;
#pragma unroll
    for (int i = 0; i < 2; ++i) g.id[i] = t0 + 16 * i < t_end ? table[(t0 + 16 * i) >> v.page_shift] : -1;
    return g;
  };
  auto there_of = [&](const pages& g) {
    return ((unsigned)g.id[0] < (unsigned)v.n_pages ? 1u : 0u) | ((unsigned)g.id[1] < (unsigned)v.n_pages ? 2u : 0u);
  };
  auto page_of = [&](const pages& g, uint32_t there, int i) { return pool + (size_t)((there >> i) & 1 ? g.id[i] : 0) * page_bytes; };
  i32x4_t kf[NF], vf[NF];
  float ks[16], vs[16];
  // Key row `col` of the first operand is the token that makes a half's sixteen scores the tokens whose values the half's lanes hold:
  // 16 h + k (INT8) or 16 (k / 8) + 8 h + k % 8.
  const int ktok = I8 ? 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3) : 16 * (col >> 4) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
  auto load_keys = [&](int t0, const pages& g, uint32_t there) {
    const uint8_t* p0 = page_of(g, there, 0) + (t0 & slot_mask) * (DP * ES);
    const uint8_t* p1 = page_of(g, there, 1) + ((t0 + 16) & slot_mask) * (DP * ES);
    const uint8_t* kp = (ktok >> 4 ? p1 : p0) + (ktok & 15) * (DP * ES) + h * 16;
#pragma unroll
    for (int i = 0; i < NF; ++i) kf[i] = *reinterpret_cast<const i32x4_t*>(kp + i * 32);
    if constexpr (I8) {
      const float* s0 = reinterpret_cast<const float*>(page_of(g, there, 0) + 2 * (size_t)v.part_bytes) + (t0 & slot_mask);
      const float* s1 = reinterpret_cast<const float*>(page_of(g, there, 1) + 2 * (size_t)v.part_bytes) + ((t0 + 16) & slot_mask);
      const f32x4_t* sp = reinterpret_cast<const f32x4_t*>(h ? s1 : s0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4_t x = sp[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) ks[4 * i + j] = x[j];
      }
    }
  };
  auto load_values = [&](int t0, const pages& g, uint32_t there) {
    const uint8_t* p0 = page_of(g, there, 0) + v.part_bytes + (t0 & slot_mask) * (DP * ES) + col * (16 * ES);
    const uint8_t* p1 = page_of(g, there, 1) + v.part_bytes + ((t0 + 16) & slot_mask) * (DP * ES) + col * (16 * ES);
    if constexpr (I8) {
      const uint8_t* vp = h ? p1 : p0;
#pragma unroll
      for (int i = 0; i < NK; ++i) vf[i] = *reinterpret_cast<const i32x4_t*>(vp + i * 512);
      const float* s0 = reinterpret_cast<const float*>(page_of(g, there, 0) + 2 * (size_t)v.part_bytes) + slot_mask + 1 + (t0 & slot_mask);
      const float* s1 = reinterpret_cast<const float*>(page_of(g, there, 1) + 2 * (size_t)v.part_bytes) + slot_mask + 1 + ((t0 + 16) & slot_mask);
      const f32x4_t* sp = reinterpret_cast<const f32x4_t*>(h ? s1 : s0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4_t x = sp[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) vs[4 * i + j] = x[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        vf[i] = *reinterpret_cast<const i32x4_t*>(p0 + h * 16 + i * 1024);
        vf[NK + i] = *reinterpret_cast<const i32x4_t*>(p1 + h * 16 + i * 1024);
      }
    }
  };
  int t0 = t_begin + wave * TT;
  pages here = pages_at(t0);

  bf16x8_t qf[NS];               // element of step s: the keys' pieces of 16 bytes are two steps of INT8, one of bf16
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const i32x4_t x = row_piece(a.Q + trow * a.qs + (size_t)head * v.d, v.d, I8 ? (s >> 1) * 32 + h * 16 + (s & 1) * 8 : s * 16 + h * 8);
    qf[s] = __builtin_bit_cast(bf16x8_t, mine ? x : i32x4_t{0, 0, 0, 0});
  }
  f32x16_t acc[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[i][j] = 0.0f;
  float m = -INFINITY, l = 0.0f;
  uint32_t seen = 0;
  bool left_out = false;         // values that are not finite in a tile that some row sees a part of: the product leaves them out

  uint32_t there = there_of(here);
  if (t0 < t_end) {
    load_keys(t0, here, there);
    load_values(t0, here, there);
  }
  pages next = pages_at(t0 + W * TT);
  while (t0 < t_end) {
    const int t_next = t0 + W * TT;
    const bool more = t_next < t_end, full = t0 >= all_begin && t0 + TT <= all_end && there == 3;
    const uint32_t there_next = there_of(next);
    f32x16_t S;
#pragma unroll
    for (int j = 0; j < 16; ++j) S[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      if constexpr (I8) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint2 x = codes_bf16(kf[i][2 * j]), y = codes_bf16(kf[i][2 * j + 1]);
          S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(x.x, x.y, y.x, y.y)), qf[2 * i + j], S, 0, 0, 0);
        }
      } else {
        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), qf[i], S, 0, 0, 0);
      }
    }
    float p[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) p[k] = S[k] * (I8 ? ks[k] * a.scale : a.scale);
    if (more) load_keys(t_next, next, there_next);
    uint32_t mask = 0xffff;
    if (!full) {
      mask = 0;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int c = I8 ? 16 * h + k : 16 * (k >> 3) + 8 * h + (k & 7);
        if (t0 + c <= lim && t0 + c >= low && ((there >> (c >> 4)) & 1)) mask |= 1u << k;
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) p[k] = (mask >> k) & 1 ? p[k] : -INFINITY;
    }
    seen |= mask | (uint32_t)__shfl_xor((int)mask, 32, 64);
    float top = p[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = fmaxf(top, p[k]);
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float mt = fmaxf(m, top), mx = mt == -INFINITY ? 0.0f : mt;
    const float keep = __builtin_amdgcn_exp2f(m - mx);
    m = mt;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      p[k] = __builtin_amdgcn_exp2f(p[k] - mx);
      sum += p[k];
    }
    l = l * keep + sum;
    if (!__all(keep == 1.0f))
#pragma unroll
      for (int i = 0; i < NK; ++i) acc[i] *= keep;
    if constexpr (I8)
#pragma unroll
      for (int k = 0; k < 16; ++k) p[k] = full || ((mask >> k) & 1) ? p[k] * vs[k] : 0.0f;   // (a step that nobody sees may be NaN)
    bf16x8_t pb[2];              // rounded to bf16, the operand's type; the sum l is of the unrounded ones
#pragma unroll
    for (int k = 0; k < 16; ++k) pb[k >> 3][k & 7] = (__bf16)p[k];
    if constexpr (!I8) {
      if (!full) {               // a probability of zero does not silence an infinity
        bool bad = false;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int left = (there >> q) & 1 ? t_end - (t0 + 16 * q + 8 * h) : 0;
#pragma unroll
          for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              vf[q * NK + i][j] &= (int)((left > 2 * j ? 0xffffu : 0u) | (left > 2 * j + 1 ? 0xffff0000u : 0u));
              bad |= has_nonfinite((uint32_t)vf[q * NK + i][j]);
            }
        }
        if (__any(bad)) {
          left_out = true;
#pragma unroll
          for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((vf[i][j] & 0x7f80) == 0x7f80) vf[i][j] &= (int)0xffff0000;
              if ((vf[i][j] & 0x7f800000) == 0x7f800000) vf[i][j] &= 0xffff;
            }
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        if constexpr (I8) {
          const uint2 x = codes_bf16(vf[i][2 * q]), y = codes_bf16(vf[i][2 * q + 1]);
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, make_uint4(x.x, x.y, y.x, y.y)), pb[q], acc[i], 0, 0, 0);
        } else {
          acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf[q * NK + i]), pb[q], acc[i], 0, 0, 0);
        }
      }
    if (more) {
      load_values(t_next, next, there_next);
      here = next;
      next = pages_at(t_next + W * TT);
    }
    there = there_next;
    t0 = t_next;
  }

  // ---- the wavefronts' parts, joined in their order: register 4 q + j of half h is element 8 q + 4 h + j of each 32 of row `col`
  extern __shared__ float lds[];
  float* ml = lds + W * ROWS * PITCH;
  uint32_t* lr = reinterpret_cast<uint32_t*>(ml + W * ROWS * 2);
  if (wave < tiles) {
    l += __shfl_xor(l, 32, 64);
    uint32_t reach[NK];
    if constexpr (!I8) {
#pragma unroll
      for (int i = 0; i < NK; ++i) reach[i] = 0;
      if (__any(left_out || any_nonfinite<NK>(acc))) find_reach<NK>(v, b, kvh, t_begin + wave * TT, t_end, W * TT, low, lim, reach);
    }
#pragma unroll
    for (int i = 0; i < NK; ++i) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4_t x = {acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]};
        *reinterpret_cast<f32x4_t*>(lds + (wave * ROWS + col) * PITCH + 32 * i + 8 * q + 4 * h) = x;
      }
      if constexpr (!I8) lr[(wave * NK + i) * 64 + lane] = reach[i];
    }
    if (h == 0) {
      ml[(wave * ROWS + col) * 2] = m;
      ml[(wave * ROWS + col) * 2 + 1] = seen ? l : -1.0f;      // (a sum is never negative)
    }
  }
  __syncthreads();
  const int parts = min(W, tiles);
  for (int e = threadIdx.x; e < rows_here * (DP / 4); e += W * 64) {
    const int rr = e / (DP / 4), d = e % (DP / 4) * 4;
    float M = -INFINITY;
    for (int w = 0; w < parts; ++w) M = fmaxf(M, ml[(w * ROWS + rr) * 2]);
    const float mx = M == -INFINITY ? 0.0f : M;
    float sum = 0.0f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    uint32_t hit = 0;
    bool some = false;
    for (int w = 0; w < parts; ++w) {                          // (a wavefront that saw nothing of a row holds zeros)
      const float lw = ml[(w * ROWS + rr) * 2 + 1], f = lw < 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ml[(w * ROWS + rr) * 2] - mx);
      some |= !(lw < 0.0f);
      sum += lw * f;
      o += *reinterpret_cast<const f32x4_t*>(lds + (w * ROWS + rr) * PITCH + d) * f;
      if constexpr (!I8) hit |= lr[(w * NK + (d >> 5)) * 64 + (d & 4) * 8 + rr] >> (4 * ((d & 31) >> 3));
    }
    const float inv = some ? 1.0f / sum : 0.0f;
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (I8) x[j] = some ? o[j] * inv : 0.0f;
      else x[j] = some ? settle(o[j], inv, (hit >> j) & 1, (hit >> (16 + j)) & 1) : 0.0f;
    }
    const int row = row0 + rr;
    const size_t at = ((size_t)r.r0 + row / a.group) * a.heads + kvh * a.group + row % a.group;
    store_quad(a.O + at * v.d, v.d, d, x);
    if (d == 0 && a.lse) a.lse[at] = some ? (M + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f : -INFINITY;
  }
}

// Which of the two: tiles of 32 rows up to 16384 rows times heads, half the CUs' worth of tiles of 128.  (32 / 128 rows a tile, INT8, us: 130 rows of
// 16 heads of 128 9.3 / 11.9; five sequences of 24 rows behind 2000 tokens, 20/4 heads of 128, 29 / 68; 256, 512 and 1024 rows of 32/8 heads of 128
// 12.4 / 14.5, 23.7 / 21.7 and 55 / 37; 512 and 1024 rows of 32 heads of 64 15.4 / 17.9 and 35.7 / 29.2; 512 rows behind 7680 tokens, 32/8 heads
// of 128, 157 / 242.)  And for 16-bit heads beyond 128, where one wavefront a SIMD holds the tile and the barriers of the other kernel cost
// more than its shared reads save, or its tile spills, but not for those of 162 to 192, the only ones that are faster shared (8192 and 2048 tokens,
// 16/4 heads of 160 0.84 / 0.89 ms and 105 / 120 us, of 192 1.08 / 0.83 and 116 / 108, of 224 1.07 / 1.28 and 127 / 165, of 256 1.44 / 1.80 and
// 154 / 227).
template <int KIND, int NK> constexpr bool always_few() { return KIND == PQ_KV_BF16 && NK > 4 && NK != 6; }
template <int KIND, int NK>
bool few_rows(const prefill_args& a) { return always_few<KIND, NK>() || (int64_t)a.v.T * a.heads <= 16384; }

// The LDS beyond 64 KiB of a kernel, asked for once on each device.
int allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& asked) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return pq_set_error(PQ_ERR_HIP, "hipGetDevice failed");
  const uint64_t bit = (uint64_t)1 << (dev & 63);
  if (asked.load(std::memory_order_relaxed) & bit) return PQ_OK;
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)
    return pq_set_error(PQ_ERR_HIP, "hipFuncSetAttribute failed for an attention kernel");
  asked.fetch_or(bit, std::memory_order_relaxed);
  return PQ_OK;
}

template <int KIND, int NK>
int launch_prefill_nk(prefill_args a, hipStream_t s) {
  static std::atomic<uint64_t> asked[2];
  const bool few = few_rows<KIND, NK>(a);
  const int64_t tiles = (int64_t)a.v.T * a.group / (few ? 32 : 128) + a.v.n_seqs, grid = tiles * a.v.n_kv_heads;
  if (grid > 0x7fffffff) return pq_set_error(PQ_ERR_SHAPE, "%d rows of %d heads in %d sequences are too many for one call", a.v.T, a.heads, a.v.n_seqs);
  a.tiles = (int)tiles;
  if (few) {
    constexpr int lds = rows_lds<KIND, NK>();
    if (int e = allow_lds((const void*)attn_rows_kernel<KIND, NK>, lds, asked[0])) return e;
    attn_rows_kernel<KIND, NK><<<(unsigned)grid, rows_waves<NK>() * 64, lds, s>>>(a);
  } else if constexpr (!always_few<KIND, NK>()) {
    constexpr int lds = 2 * prefill_stage<KIND, NK>();
    if (int e = allow_lds((const void*)attn_prefill_kernel<KIND, NK>, lds, asked[1])) return e;
    attn_prefill_kernel<KIND, NK><<<(unsigned)grid, 256, lds, s>>>(a);
  }
  return PQ_OK;
}
template <int KIND>
int launch_prefill(const prefill_args& a, hipStream_t s) {
  switch (a.v.dp / 32) {
    case 1: return launch_prefill_nk<KIND, 1>(a, s);
    case 2: return launch_prefill_nk<KIND, 2>(a, s);
    case 3: return launch_prefill_nk<KIND, 3>(a, s);
    case 4: return launch_prefill_nk<KIND, 4>(a, s);
    case 5: return launch_prefill_nk<KIND, 5>(a, s);
    case 6: return launch_prefill_nk<KIND, 6>(a, s);
    case 7: return launch_prefill_nk<KIND, 7>(a, s);
    default: return launch_prefill_nk<KIND, 8>(a, s);
  }
}

}  // namespace

extern "C" size_t pq_attn_decode_workspace_bytes(const pq_attn_desc* d) {
  if (check_attn(d)) return 0;
  return plan_decode(*d).total;
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
  const decode_plan p = plan_decode(*d);
  decode_args a;
  a.v = pq_kv_make_view(d->kv, cache, nullptr, lens, page_table, T);
  a.Q = (const uint16_t*)Q; a.qs = q_stride;
  a.heads = d->n_heads; a.group = d->n_heads / d->kv.n_kv_heads; a.head_blocks = p.head_blocks; a.block_heads = p.block_heads;
  a.window = d->window; a.chunk = p.chunk; a.n_chunks = p.n_chunks;
  a.scale = d->scale * 1.4426950408889634f;
  a.O = (uint16_t*)O; a.lse = lse;
  a.part_o = (float*)((char*)workspace + p.part_o); a.part_ml = (float*)((char*)workspace + p.part_ml);
  const int64_t pieces = (int64_t)T * d->kv.n_kv_heads * p.n_chunks, grid = (pieces + 7) / 8 * 8 * p.head_blocks;
  PQ_REQUIRE(grid <= 0x7fffffff, PQ_ERR_SHAPE, "%d sequences of %d heads are too many for one call", T, d->n_heads);
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_ATTN_DECODE, s);
  if (d->kv.kv_kind == PQ_KV_INT8) launch_decode<PQ_KV_INT8>(a, p, (unsigned)grid, s);
  else launch_decode<PQ_KV_BF16>(a, p, (unsigned)grid, s);
  PQ_CHECK_LAUNCH("attn_decode_kernel");
  if (p.n_chunks > 1) {
    attn_join_kernel<<<(unsigned)(T * d->n_heads), 256, 0, s>>>(a, a.v.dp <= 32 ? 32 : a.v.dp <= 64 ? 64 : a.v.dp <= 128 ? 128 : 256);
    PQ_CHECK_LAUNCH("attn_join_kernel");
  }
  return PQ_OK;
}

extern "C" int pq_attn_prefill(const pq_attn_desc* d, const void* Q, int64_t q_stride, int32_t T, const int32_t* row_start, const void* cache,
                               size_t cache_bytes, const int32_t* lens, const int32_t* page_table, void* O, float* lse, void* stream) {
  if (int e = check_attn(d)) return e;
  PQ_REQUIRE(T >= 0, PQ_ERR_BAD_ARG, "T=%d is negative", T);
  if (T == 0 || d->kv.n_seqs == 0) return PQ_OK;
  if (int e = check_attn_call(d, Q, q_stride, T, cache, cache_bytes, lens, page_table, O)) return e;
  prefill_args a;
  a.v = pq_kv_make_view(d->kv, cache, row_start, lens, page_table, T);
  a.Q = (const uint16_t*)Q; a.qs = q_stride;
  a.heads = d->n_heads; a.group = d->n_heads / d->kv.n_kv_heads;
  a.causal = d->causal; a.window = d->window;
  a.scale = d->scale * 1.4426950408889634f;
  a.O = (uint16_t*)O; a.lse = lse;
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_ATTN_PREFILL, s);
  if (int e = d->kv.kv_kind == PQ_KV_INT8 ? launch_prefill<PQ_KV_INT8>(a, s) : launch_prefill<PQ_KV_BF16>(a, s)) return e;
  PQ_CHECK_LAUNCH("attn_prefill_kernel");
  return PQ_OK;
}
