// Attention over the rows of a call, for training: forward pass and gradients.
//
//     s_ij = scale q_i . k_j (visible j),  lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
//     delta_i = sum_d dO_id O_id,  dP_ij = dO_i . v_j,  dS_ij = p_ij (dP_ij - delta_i)
//     dQ_i = scale sum_j dS_ij k_j,   dK_j = scale sum_i dS_ij q_i,   dV_j = sum_i p_ij dO_i     (j's sums over the heads that share it, too)
//
// No tensor of scores exists: tiles of 32 x 32 scores are formed by v_mfma_f32_32x32x16_bf16, used, and formed again from lse in the backward pass.
// Long sequences are bound by the matrix pipe and by what one wavefront can issue beside it; memory is read once or from the L2.  A score tile's columns
// are the lanes (queries in the forward pass and for dQ, tokens for dK and dV), so that its weights are the next product's operand as they stand in
// registers, in an order of the contraction that the other operand's reads follow, and softmax never leaves a lane but for halves of sums.
#include "pq_kv.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

namespace {

#define PQ_REQUIRE(cond, code, ...) \
  do { if (!(cond)) return pq_set_error(code, __VA_ARGS__); } while (0)

constexpr int SA_ROWS = 128;      // rows of a workgroup's tile, 32 a wavefront
constexpr int SA_STAGE = 64;      // rows of a stage in LDS
constexpr float SA_LOG2E = 1.4426950408889634f;

struct self_args {
  const uint16_t *Q, *K, *V, *O, *dO;
  int64_t qs, ks, vs;            // elements between rows
  uint16_t *out, *dQ, *dK, *dV;
  int64_t dqs, dks, dvs;
  float* lse;                    // [T][heads]
  float2* stats;                 // [heads][T]: lse times log2 e, delta
  float* parts;                  // [pieces][T][kv_heads][2][d]: parts of dK and dV where a tile's work is cut
  const int32_t* row_start;
  int T, n_seqs, heads, kv_heads, group, d, causal, window, tiles, pieces;
  float c;                       // |scale| log2 e; the sign is in the operand that stays in registers
  float scale;
};

// ---------------------------------------------------------------------------------------------
// Tiles in LDS: rows of DP elements as they lie in memory, their pieces of 16 bytes exchanged within a row by a number that the row gives, so that both
// ways of reading go through all 64 banks: the same piece of eight rows (operand rows), and four neighbouring pieces of four rows (the transposing
// reads, whose rows therefore lie in different quarters of the banks).
// ---------------------------------------------------------------------------------------------
template <int DP> __device__ __forceinline__ int piece_at(int row, int c) {
  const int low = (row >> 2) & 3;
  if constexpr (DP % 128 == 0) return c ^ (4 * (row & 3) + low);
  else if constexpr (DP % 64 == 0) return c ^ (4 * ((row >> 1) & 1) + low);
  else return c ^ low;            // (rows an odd number of quarters apart)
}

typedef int i32x4_u_t __attribute__((ext_vector_type(4), aligned(4)));
// Eight elements of a row of d from element `at` on, zeros behind its end.
__device__ __forceinline__ i32x4_t load_piece(const uint16_t* q, int d, int at) {
  i32x4_t x = {0, 0, 0, 0};
  if (at + 8 <= d) {
    x = *reinterpret_cast<const i32x4_u_t*>(q + at);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (at + 2 * j < d) x[j] = *reinterpret_cast<const int*>(q + at + 2 * j);
  }
  return x;
}

// Sixteen bytes a lane from memory to LDS, lane by lane from `lds` on: from base + offset, the base and `lds` the same for all lanes.  (Not through the
// compiler's builtin: it would wait for these loads in front of every later read of LDS, of the other buffer as well.  m0 is a
// register that the compiler keeps for itself and sets where it needs it: naming it as clobbered is taken with a warning and no promise.  It needs it nowhere
// in these kernels, and forms the base by scalar instructions, which need no wait states in front of the load; both are tested on what is built.)
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// A stage of SA_STAGE rows of one tensor on its way to LDS.  DIRECT: rows and heads lie at multiples of 16 bytes, the loads go straight there;
// otherwise through registers, four bytes aligned.  Rows behind the sequence's last are the last once more: whoever uses the stage hides them.
template <int DP, bool DIRECT>
struct stage_t {
  static constexpr int CPR = DP / 8, N = SA_STAGE * CPR / 256, BYTES = SA_STAGE * DP * 2;
  const uint16_t* base;          // the sequence's first row
  int64_t stride;                // elements, at most 2^23: 64 rows are within 2^31 bytes
  int d, n;
  bool is_last;                  // the sequence's last row is the call's
  uint32_t offset[N];            // of the lane's pieces from a stage's first row, in bytes
  i32x4_t hold[DIRECT ? 1 : N];

  __device__ __forceinline__ void begin(const uint16_t* base_, int64_t stride_, int d_, int n_, bool is_last_) {
    base = base_; stride = stride_; d = d_; n = n_; is_last = is_last_;
#pragma unroll
    for (int i = 0; i < N; ++i) offset[i] = (uint32_t)row_of(i) * (uint32_t)stride * 2 + place_in_row(i);
  }
  static __device__ __forceinline__ int place(int i) { return (int)((threadIdx.x >> 6) * N + i) * 64 + (int)(threadIdx.x & 63); }
  static __device__ __forceinline__ int row_of(int i) { return place(i) / CPR; }
  static __device__ __forceinline__ int piece_of(int i) { return piece_at<DP>(row_of(i), place(i) % CPR); }
  // Pieces behind d are not loaded (DIRECT), or are the first once more and cleared afterwards.
  __device__ __forceinline__ uint32_t place_in_row(int i) const { return DIRECT || piece_of(i) * 8 < d ? piece_of(i) * 16 : 0; }

  __device__ __forceinline__ void load(int first, unsigned char* lds) {
    const uint16_t* from = base + (int64_t)first * stride;
    const bool whole = first + SA_STAGE <= n;
    if constexpr (DIRECT) {
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(lds) + (threadIdx.x >> 6) * N * 1024);
      if (whole && d == DP) {
#pragma unroll
        for (int i = 0; i < N; ++i) load_to_lds(from, offset[i], to + i * 1024);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t x = (uint32_t)min(row_of(i), n - 1 - first) * (uint32_t)stride * 2 + place_in_row(i);
          if (piece_of(i) * 8 < d) load_to_lds(from, x, to + i * 1024);
        }
      }
    } else {
      // A row's last piece takes up to six elements of what follows (cleared by `store`): the next head's, or the next row's.  Not from the call's last
      // row, behind which nothing need be, nor where rows are shorter than a piece.
      const char* bytes = reinterpret_cast<const char*>(from);
      uint32_t x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = whole ? offset[i] : (uint32_t)min(row_of(i), n - 1 - first) * (uint32_t)stride * 2 + place_in_row(i);
      if (d >= 8 && !(is_last && first + SA_STAGE >= n)) {
#pragma unroll
        for (int i = 0; i < N; ++i) hold[i] = *reinterpret_cast<const i32x4_u_t*>(bytes + x[i]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) hold[i] = load_piece(reinterpret_cast<const uint16_t*>(bytes + (x[i] - place_in_row(i))), d, piece_of(i) * 8);
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char* lds) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        i32x4_t x = hold[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = piece_of(i) * 8 + 2 * j < d ? x[j] : 0;
        *reinterpret_cast<i32x4_t*>(lds + place(i) * 16) = x;
      }
    }
  }
  // Pieces behind d are never written by direct loads: zeros, once.
  static __device__ __forceinline__ void clear(unsigned char* lds, int d) {
    if constexpr (DIRECT) {
      if (d == DP) return;
      for (int L = threadIdx.x; L < SA_STAGE * CPR; L += 256)
        if (piece_at<DP>(L / CPR, L % CPR) * 8 >= d) *reinterpret_cast<i32x4_t*>(lds + L * 16) = i32x4_t{0, 0, 0, 0};
    }
  }
};

// Operand of 32 rows (row l % 32) and elements 16 step + 8 (l / 32) .. of the contraction.
template <int DP> __device__ __forceinline__ bf16x8_t row_operand(const unsigned char* lds, int row0, int step) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  return *reinterpret_cast<const bf16x8_t*>(lds + (row0 + r) * (DP * 2) + (piece_at<DP>(r, 2 * step + h) << 4));
}
// Operand of 32 columns (column 32 block + l % 32) whose contraction runs over the 16 rows from row0 on, in the order in which the lanes hold a
// tile's rows: 4 h + 0 .. 3, 8 + 4 h + 0 .. 3.
typedef short s16x4_t __attribute__((ext_vector_type(4)));
template <int DP> __device__ __forceinline__ bf16x8_t column_operand(const unsigned char* lds, int row0, int block) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int r = 4 * h + ((lane & 15) >> 2), c = 4 * block + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), in = (lane & 1) * 8;
  auto at = [&](int row) { return lds + (row0 + row) * (DP * 2) + (piece_at<DP>(row, c) << 4) + in; };
  typedef __attribute__((address_space(3))) s16x4_t* p3;
  const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p3)at(r));
  const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p3)at(r + 8));
  const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
  return __builtin_bit_cast(bf16x8_t, make_uint4(a.x, a.y, b.x, b.y));
}
// All of a product's operands for 32 rows: DP / 16 of either kind.
template <int DP> __device__ __forceinline__ void row_operands(bf16x8_t* x, const unsigned char* lds, int row0) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) x[s] = row_operand<DP>(lds, row0, s);
}
// (the j-th of columns: block j % (DP / 32) of rows 16 (j / (DP / 32)) ..)
template <int DP> __device__ __forceinline__ bf16x8_t nth_column_operand(const unsigned char* lds, int row0, int j) {
  return column_operand<DP>(lds, row0 + 16 * (j / (DP / 32)), j % (DP / 32));
}
template <int DP> __device__ __forceinline__ void column_operands(bf16x8_t* x, const unsigned char* lds, int row0) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) x[u * (DP / 32) + i] = column_operand<DP>(lds, row0 + 16 * u, i);
}
// The operand that stays in registers: columns are rows `row` (per lane) of a tensor.  DIRECT rows of DP elements are read without a condition, so
// that all loads are under way at once.
template <int DP, bool DIRECT> __device__ __forceinline__ void load_columns(bf16x8_t* x, const uint16_t* row, int d) {
  const int h = (threadIdx.x & 63) >> 5;
  if (DIRECT && d == DP) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) x[s] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const i32x4_t*>(row + 16 * s + 8 * h));
  } else {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) x[s] = __builtin_bit_cast(bf16x8_t, load_piece(row, d, 16 * s + 8 * h));
  }
}
template <int DP> __device__ __forceinline__ void negate(bf16x8_t* x) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const uint4 w = __builtin_bit_cast(uint4, x[s]);
    x[s] = __builtin_bit_cast(bf16x8_t, make_uint4(w.x ^ 0x80008000u, w.y ^ 0x80008000u, w.z ^ 0x80008000u, w.w ^ 0x80008000u));
  }
}

__device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// Register j of a tile is its row 8 (j / 4) + 4 h + j % 4.
__device__ __forceinline__ constexpr int tile_row(int j) { return 8 * (j >> 2) + (j & 3); }

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
// Two neighbours rounded by one instruction (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t round_two(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x, y}, bf16x2_t)); }

// The order of a run of instructions where there is nothing to do beside the products: READS reads of LDS in front, then PRODUCTS times a product
// and as many more reads.
template <int READS> __device__ __forceinline__ void reads_first() { __builtin_amdgcn_sched_group_barrier(0x100, READS, 0); }
template <int PRODUCTS, int READS, int VALU> __device__ __forceinline__ void steps() {
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    if constexpr (VALU > 0) __builtin_amdgcn_sched_group_barrier(0x2, VALU, 0);
  }
}
// A phase: N steps of a product, the read of an operand that the next phase wants, and a share of the eight pairs of elements of a tile whose
// exponentials or dS are formed meanwhile.  Nothing moves from step to step: an instruction waits for the one before it to be issued, an exponential
// takes four slots, and where the compiler puts them in a row the matrix pipe is idle behind them.
template <int N, typename P, typename R, typename V> __device__ __forceinline__ void phase(P product, R read, V pair) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    product(k);
    read(k);
#pragma unroll
    for (int x = 8 * k / N; x < 8 * (k + 1) / N; ++x) pair(x);
    __builtin_amdgcn_sched_barrier(0);
  }
}
struct nothing { template <typename T> __device__ __forceinline__ void operator()(T) const {} };
// Four pairs as an operand.
__device__ __forceinline__ bf16x8_t four_pairs(const uint32_t* w) { return __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3])); }

// Eight rows of a tile as the second product's operand (registers 8 u .. 8 u + 7).
__device__ __forceinline__ bf16x8_t as_operand(const f32x16_t& x, int u) {
  const uint4 w = make_uint4(round_two(x[8 * u], x[8 * u + 1]), round_two(x[8 * u + 2], x[8 * u + 3]), round_two(x[8 * u + 4], x[8 * u + 5]),
                             round_two(x[8 * u + 6], x[8 * u + 7]));
  return __builtin_bit_cast(bf16x8_t, w);
}

// What that left of them, rounded itself.
__device__ __forceinline__ bf16x8_t as_remainder(const f32x16_t& x, int u, bf16x8_t r) {
  uint32_t w[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) w[y] = round_two(x[8 * u + 2 * y] - (float)r[2 * y], x[8 * u + 2 * y + 1] - (float)r[2 * y + 1]);
  return four_pairs(w);
}

// The sum of an operand's eight elements and x.
__device__ __forceinline__ float sum_of(bf16x8_t a, float x) {
  const uint4 w = __builtin_bit_cast(uint4, a);
  const bf16x2_t ones = {(__bf16)1.0f, (__bf16)1.0f};
  x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.x), ones, x, false);
  x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.y), ones, x, false);
  x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.z), ones, x, false);
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w.w), ones, x, false);
}

// a x b where b holds zeros for what is not seen, which an infinity or a NaN of a must not reach (0 times infinity is NaN): such elements are left
// out, and where they are seen the sum becomes infinite (twice the largest bf16 number is beyond fp32).  Three products for one, for tiles that hold such
// elements: a branch would keep two copies of the sums.
__device__ __forceinline__ f32x16_t mfma_seen(bf16x8_t a, bf16x8_t b, uint32_t seen /* bits of the operand's eight rows */, f32x16_t c) {
  const uint4 w = __builtin_bit_cast(uint4, a);
  uint32_t clean[4] = {w.x, w.y, w.z, w.w}, top[4], ones[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t x = clean[j], lo = (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
    clean[j] = x & ~(lo | hi);
    top[j] = 0x7f7f7f7fu & (lo | hi);
    ones[j] = ((seen >> (2 * j)) & 1 ? 0x3f80u : 0u) | ((seen >> (2 * j + 1)) & 1 ? 0x3f800000u : 0u);
  }
  const bf16x8_t t = __builtin_bit_cast(bf16x8_t, make_uint4(top[0], top[1], top[2], top[3]));
  const bf16x8_t s = __builtin_bit_cast(bf16x8_t, make_uint4(ones[0], ones[1], ones[2], ones[3]));
  c = mfma(__builtin_bit_cast(bf16x8_t, make_uint4(clean[0], clean[1], clean[2], clean[3])), b, c);
  c = mfma(t, s, c);
  return mfma(t, s, c);
}

// Bits low .. high of 32, as far as there are such.
__device__ __forceinline__ uint32_t bits_between(int low, int high) {
  const uint32_t up = high >= 31 ? 0xffffffffu : high < 0 ? 0u : (2u << high) - 1u;
  return low <= 0 ? up : low > 31 ? 0u : up & (0xffffffffu << low);
}
// x where bit k of the mask is set, otherwise 0 (two instructions, no comparison).
__device__ __forceinline__ float where_set(float x, uint32_t mask, int k) {
  return __uint_as_float(__float_as_uint(x) & (uint32_t)__builtin_amdgcn_sbfe((int)mask, k, 1));
}
// The bits of a tile's registers 8 u .. among those of its rows (shifted by 4 h): what mfma_seen wants.
__device__ __forceinline__ uint32_t register_bits(uint32_t rows, int u) {
  const uint32_t x = rows >> (16 * u);
  return (x & 15u) | ((x >> 8) & 15u) << 4;
}

// The value of the other half's lane joined to a lane's own (both halves hold the same columns).
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }

// Which sequence and which of its tiles of SA_ROWS rows workgroup tile vt is.  Up to 8 sequences: the longest first, of each the tiles with most work
// first (`down`: its last ones), so that long tiles do not start when the others end (32 heads of 128 on eight, 8 ragged sequences of up to 1166 rows: 64 us
// and 300 for the gradients, otherwise 68 and 315; 16 of up to 868: 85 and 351 in this order, 81 and 379 without; 60 of up to 292: 107 and 391 to 74 and 318, the
// search for the order takes longer).  Up to 63: from one load of all of row_start.  Any number: virtual
// tiles, of which sequence b owns those from floor(first row / SA_ROWS) + b on, at least as many as it has.
struct self_tile { int r0, n, at; };     // rows r0 .. r0 + n - 1 of the call, the tile's first row among them (n == 0: none)
__device__ __forceinline__ self_tile find_self_tile(const self_args& a, int vt, bool down) {
  auto first = [&](int i) { return min(max(a.row_start[i], 0), a.T); };
  self_tile t = {0, 0, 0};
  if (a.n_seqs <= 63) {
    const int lane = threadIdx.x & 63, at = first(min(lane, a.n_seqs));
    const int next = __shfl_down(at, 1, 64);               // (of all lanes: one that sits out hands nothing over)
    const int mine = lane < a.n_seqs ? max(next - at, 0) : 0;
    int before = at / SA_ROWS + lane;
    if (a.n_seqs <= 8) {
      before = 0;
      for (int i = 0; i < a.n_seqs; ++i) {
        const int n = __builtin_amdgcn_readlane(mine, i);
        before += n > mine || (n == mine && i < lane) ? (n + SA_ROWS - 1) / SA_ROWS : 0;
      }
    } else if (down) {
      vt = a.tiles - 1 - vt;
    }
    const int tiles = (mine + SA_ROWS - 1) / SA_ROWS;
    const uint64_t hit = __ballot(vt >= before && vt < before + tiles);
    if (hit == 0) return t;
    const int b = __builtin_ctzll(hit);
    int tile = vt - __builtin_amdgcn_readlane(before, b);
    if (down && a.n_seqs <= 8) tile = __builtin_amdgcn_readlane(tiles, b) - 1 - tile;
    t.r0 = __builtin_amdgcn_readlane(at, b);
    t.n = __builtin_amdgcn_readlane(mine, b);
    t.at = tile * SA_ROWS;
    return t;
  }
  if (down) vt = a.tiles - 1 - vt;
  const int b = kv_find_seq(a.n_seqs, vt, [&](int i) { return first(i) / SA_ROWS + i; });
  if (b < 0) return t;
  t.r0 = first(b);
  const int n = max(first(b + 1), t.r0) - t.r0;
  t.at = (vt - (t.r0 / SA_ROWS + b)) * SA_ROWS;
  if (t.at < n) t.n = n;
  return t;
}
// Tokens that rows from .. to - 1 of a sequence of n see between them.
__device__ __forceinline__ int first_token(const self_args& a, int row) { return a.window > 0 && row >= a.window ? row - a.window + 1 : 0; }

// The stages that a tile needs, and of them those of which a wavefront's 32 rows (or tokens) see something, from .. to - 1: these are a loop of their own,
// since a branch around accumulators costs a second copy of them all.  Those from `all` to `part` - 1 are seen by all of its rows.
// FINE stages of the gradients: p and dS as sums of two bf16 numbers, off by 2^-16 of themselves instead of 2^-8.  The first 64 rows of causal sequences and
// whole ones of up to 64 rows: they see few tokens, so that few large elements make their parts of the gradients, and these parts are the largest.  What the
// gradients of short sequences are off by is then the outputs' own rounding alone; with one rounding each it came to 1.4 times that, in one of ten short
// calls to more than 1.5 times.  A sequence has one such stage a head: 130 tokens 32 us instead of 31.  (Stages taken with care have one rounding.)
enum { PLAIN, FINE, CAREFUL };
struct stages_of { int first, n, from, all, part, to, begin; };     // begin: the first of those that are taken at all
// Stages of tokens that rows row0 .. row0 + 31 of the tile see.
__device__ __forceinline__ stages_of token_stages(const self_args& a, const self_tile& t, int row0) {
  const int end = a.causal ? min(t.at + SA_ROWS, t.n) : t.n, last = min(row0 + 31, t.n - 1);
  stages_of g;
  g.first = first_token(a, t.at) & ~(SA_STAGE - 1);
  g.n = (end - g.first + SA_STAGE - 1) / SA_STAGE;
  g.to = row0 < t.n ? ((a.causal ? last : t.n - 1) - g.first) / SA_STAGE + 1 : 0;
  g.from = min((first_token(a, row0) - g.first) / SA_STAGE, g.to);
  g.all = (first_token(a, last) - g.first + SA_STAGE - 1) / SA_STAGE;
  g.part = ((a.causal ? row0 + 1 : t.n) - g.first) / SA_STAGE;
  g.begin = 0;
  return g;
}
// Stages of rows that see tokens tok0 .. tok0 + 31 of the tile.
__device__ __forceinline__ int first_blind_row(const self_args& a, int n, int tok) {   // the first that sees `tok` no more
  return a.window > 0 && a.window < n && tok < n - a.window ? tok + a.window : n;
}
__device__ __forceinline__ stages_of row_stages(const self_args& a, const self_tile& t, int tok0) {
  stages_of g;
  g.first = (a.causal ? t.at : 0) & ~(SA_STAGE - 1);
  g.n = (first_blind_row(a, t.n, min(t.at + SA_ROWS, t.n) - 1) - g.first + SA_STAGE - 1) / SA_STAGE;
  g.to = tok0 < t.n ? (first_blind_row(a, t.n, min(tok0 + 31, t.n - 1)) - g.first + SA_STAGE - 1) / SA_STAGE : 0;
  g.from = min(a.causal ? (tok0 - g.first) / SA_STAGE : 0, g.to);
  g.all = a.causal ? (tok0 + 31 - g.first + SA_STAGE - 1) / SA_STAGE : 0;
  g.part = (first_blind_row(a, t.n, tok0) - g.first) / SA_STAGE;
  g.begin = 0;
  return g;
}
// `next` waits for a stage and has the loads of the one behind it started, `store` puts away what came through registers; `use` is told whether the
// stage needs its mask.  (Masked and unmasked stages are loops in turn inside a loop, so that each is there once: heads of 128, 8192 and 130 tokens,
// always masked 2320 and 29.1 us, two masked loops around an unmasked one 2150 and 33.)
struct fine_t { static constexpr bool value = true; };              // (masked, and one by itself)
template <bool ANY_FINE, typename N, typename S, typename U>
__device__ __forceinline__ void in_stages(const stages_of& g, N next, S store, U use, bool fine = false) {
  int i = g.begin;
#pragma unroll 1
  for (; i < min(g.from, g.n); ++i) { next(i); store(i); }
  if constexpr (ANY_FINE) {
#pragma unroll 1
    for (; i < min(fine ? 1 : 0, g.to); ++i) { next(i); use(i, fine_t{}); store(i); }
  }
  int masked = min(g.all, g.to);
  const int part = min(g.part, g.to);
#pragma unroll 1
  while (i < g.to) {
#pragma unroll 1
    for (; i < masked; ++i) { next(i); use(i, std::true_type{}); store(i); }
#pragma unroll 1
    for (; i < part; ++i) { next(i); use(i, std::false_type{}); store(i); }
    masked = g.to;
  }
#pragma unroll 1
  for (; i < g.n; ++i) { next(i); store(i); }
}
// The same where `use` asks by itself.
template <typename N, typename S, typename U>
__device__ __forceinline__ void in_stages_alike(const stages_of& g, N next, S store, U use) {
  int i = g.begin;
#pragma unroll 1
  for (; i < min(g.from, g.n); ++i) { next(i); store(i); }
#pragma unroll 1
  for (; i < g.to; ++i) { next(i); use(i); store(i); }
#pragma unroll 1
  for (; i < g.n; ++i) { next(i); store(i); }
}

typedef uint32_t u32x2_u_t __attribute__((ext_vector_type(2), aligned(4)));
__device__ __forceinline__ void store_four(uint16_t* row, int d, int at, const float* x) {
  const uint32_t lo = round_two(x[0], x[1]), hi = round_two(x[2], x[3]);
  if (at + 4 <= d) *reinterpret_cast<u32x2_u_t*>(row + at) = u32x2_u_t{lo, hi};
  else if (at < d) *reinterpret_cast<uint32_t*>(row + at) = lo;
}
// Accumulators [DP / 32] of a column each lane (elements 32 i + 8 q + 4 h + j) times f into a row.
template <int DP> __device__ __forceinline__ void store_column(const f32x16_t* acc, float f, uint16_t* row, int d) {
  const int h = (threadIdx.x & 63) >> 5;
  uint16_t* mine = row + 4 * h;
  if (d == DP) {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<u32x2_u_t*>(mine + 32 * i + 8 * q) = u32x2_u_t{round_two(acc[i][4 * q] * f, acc[i][4 * q + 1] * f),
                                                                        round_two(acc[i][4 * q + 2] * f, acc[i][4 * q + 3] * f)};
  } else {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float x[4] = {acc[i][4 * q] * f, acc[i][4 * q + 1] * f, acc[i][4 * q + 2] * f, acc[i][4 * q + 3] * f};
        store_four(row, d, 32 * i + 8 * q + 4 * h, x);
      }
  }
}
template <int DP> __device__ __forceinline__ void store_part(const f32x16_t* acc, float f, float* row, int d) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
      const int at = 32 * i + tile_row(j) + 4 * h;
      if (at < d) *reinterpret_cast<f32x2_t*>(row + at) = f32x2_t{acc[i][j] * f, acc[i][j + 1] * f};
    }
}

// Head and tile of a workgroup: the heads first, those of a key-value head a multiple of kv_heads apart (its tokens then stay in one L2).
struct self_place { int head, kv_head, vt; };
__device__ __forceinline__ self_place place_of(const self_args& a) {
  const int t = blockIdx.x / a.heads, x = blockIdx.x - t * a.heads, kv = x % a.kv_heads;
  return {kv * a.group + x / a.kv_heads, kv, t};
}

// ---------------------------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------------------------
// A stage of tokens.  Any reference m gives the same quotient as long as nothing overflows and the row's largest p is not tiny: the maximum of what a row
// sees in its first stage serves for all others (it has p = 1, so nothing that counts is lost below; what overflows above ends as infinity or NaN,
// and the tile is taken once more with care).  So the stages have no maximum to keep and no accumulators to rescale.
// MASKED: stages that some row sees in part, or as its first.
//
// 128 rows a workgroup, 32 a wavefront; stages of 64 tokens, the next one's loads on their way to LDS.  Two workgroups share a CU: one's softmax runs beside
// the other's products (one wavefront a SIMD: 627 us where two take 525).  A phase is a row of products with what the next phase needs read between
// them and the other half's softmax in the gaps, in an order that the compiler is held to.  8192 causal rows, 32 heads of 128 on eight: 525 us,
// 1.05 PFLOP/s, the matrix pipe busy 60 % of the cycles at the 1.7 GHz that the power limit leaves, LDS without bank conflicts; the rest is
// the issue of softmax (exponentials, sums, conversion) in two wavefronts a SIMD.  Four stages in LDS instead of two: 545 us.
template <int DP, bool MASKED>
__device__ __forceinline__ void forward_stage(const self_args& a, const unsigned char* lk, const unsigned char* lv, const bf16x8_t* q, f32x16_t* o,
                                              float& m, float& l, int low, int lim) {
  constexpr int NK = DP / 32, N = DP / 16;
  const int h = (threadIdx.x & 63) >> 5;
  f32x16_t s[2];
  float sum[2] = {0.0f, 0.0f};
  auto scores = [&](int t, const bf16x8_t* x) {
    s[t] = f32x16_t{};
#pragma unroll
    for (int k = 0; k < N; ++k) s[t] = mfma(x[k], q[k], s[t]);
  };
  float ref, c = a.c;
  auto weights = [&](int t) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[t][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][j], c, -ref));
      sum[j & 1] += s[t][j];
    }
  };
  auto products = [&](int t, const bf16x8_t* x) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8_t p = as_operand(s[t], u);
#pragma unroll
      for (int i = 0; i < NK; ++i) o[i] = mfma(x[u * NK + i], p, o[i]);
    }
  };
  bf16x8_t x[2][N];
  if constexpr (MASKED) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      row_operands<DP>(x[0], lk, 32 * t);
      scores(t, x[0]);
    }
    reads_first<4>();
    steps<2 * N, 1, 0>();
    const uint32_t seen[2] = {bits_between(low, lim) >> (4 * h), bits_between(low - 32, lim - 32) >> (4 * h)};
#pragma unroll
    for (int j = 0; j < 32; ++j) s[j >> 4][j & 15] = (seen[j >> 4] >> tile_row(j & 15)) & 1 ? s[j >> 4][j & 15] : -INFINITY;
    if (__ballot(m == -INFINITY)) {
      float top = s[0][0];
#pragma unroll
      for (int j = 1; j < 32; ++j) top = fmaxf(top, s[j >> 4][j & 15]);
      top = fmaxf(top, other_half(top));
      if (m == -INFINITY && top > -INFINITY) m = top * a.c;
    }
    ref = m == -INFINITY ? 0.0f : m;
    if (c == 0.0f) c = 1.17549435e-38f;               // (hidden ones times a scale of 0 would be NaN)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      weights(t);
      column_operands<DP>(x[0], lv, 32 * t);
      products(t, x[0]);
    }
    __builtin_amdgcn_sched_group_barrier(0x2, 28, 0);
    reads_first<2 * NK>();
    steps<3 * NK, 2, 28 / NK>();
    steps<NK, 0, 0>();
  } else {
    ref = m;
    uint32_t w[2][8];
    auto pair = [&](int t, int y) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][2 * y], c, -ref)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][2 * y + 1], c, -ref));
      sum[0] += p0;
      sum[1] += p1;
      w[t][y] = round_two(p0, p1);
    };
    auto product = [&](int t, int j) { o[j % NK] = mfma(x[t][j], four_pairs(w[t] + 4 * (j / NK)), o[j % NK]); };
    row_operands<DP>(x[0], lk, 0);
    s[0] = s[1] = f32x16_t{};
    __builtin_amdgcn_sched_barrier(0);
    phase<N>([&](int k) { s[0] = mfma(x[0][k], q[k], s[0]); }, [&](int k) { x[1][k] = row_operand<DP>(lk, 32, k); }, nothing{});
    phase<N>([&](int k) { s[1] = mfma(x[1][k], q[k], s[1]); }, [&](int k) { x[0][k] = nth_column_operand<DP>(lv, 0, k); }, [&](int y) { pair(0, y); });
    phase<N>([&](int k) { product(0, k); }, [&](int k) { x[1][k] = nth_column_operand<DP>(lv, 32, k); }, [&](int y) { pair(1, y); });
    phase<N>([&](int k) { product(1, k); }, nothing{}, nothing{});
  }
  l += sum[0] + sum[1];
}

// The same with care, 32 tokens at a time: the reference follows the largest score, and an infinity or a NaN among the values reaches those rows
// alone that see it.
template <int DP>
__device__ __forceinline__ void forward_block(const self_args& a, const unsigned char* lk, const unsigned char* lv, int at, const bf16x8_t* q, f32x16_t* o,
                                              float& m, float& l, int low, int lim) {
  constexpr int NK = DP / 32;
  const int h = (threadIdx.x & 63) >> 5;
  f32x16_t s = {};
#pragma unroll
  for (int k = 0; k < DP / 16; ++k) s = mfma(row_operand<DP>(lk, at, k), q[k], s);
  uint32_t seen = 0;
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const bool v = at + tile_row(j) + 4 * h >= low && at + tile_row(j) + 4 * h <= lim;
    seen |= (v ? 1u : 0u) << j;
    s[j] = v ? s[j] * a.c : -INFINITY;
    top = fmaxf(top, s[j]);
  }
  top = fmaxf(top, other_half(top));
  const float next = fmaxf(m, top), f = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - next);
  m = next;
  l *= f;
#pragma unroll
  for (int i = 0; i < NK; ++i) o[i] *= f;
  const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    s[j] = __builtin_amdgcn_exp2f(s[j] - ref);
    l += s[j];
  }
#pragma unroll 1
  for (int u = 0; u < 2; ++u) {
    const bf16x8_t p = u ? as_operand(s, 1) : as_operand(s, 0);
#pragma unroll
    for (int i = 0; i < NK; ++i) o[i] = mfma_seen(column_operand<DP>(lv, at + 16 * u, i), p, seen >> (8 * u), o[i]);
  }
}

// Whether one of the lane's sums is infinite or NaN (in eight chains: one would wait for each of its instructions).
template <int NK> __device__ __forceinline__ bool any_nonfinite(const f32x16_t* acc) {
  float z[8] = {};
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) z[j & 7] = __builtin_fmaf(acc[i][j], 0.0f, z[j & 7]);
  return !(((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7])) == 0.0f);     // (NaN: not equal)
}

template <int DP, bool DIRECT, bool CAREFUL>
__device__ __forceinline__ void forward_tile(const self_args& a, const self_place& w, const self_tile& t, int row0, bf16x8_t* q, f32x16_t* o, float& m,
                                             float& l, unsigned char* lds) {
  typedef stage_t<DP, DIRECT> stage;
  constexpr int BUF = 2 * stage::BYTES;
  const int row = row0 + (threadIdx.x & 31);
  const uint16_t* K = a.K + (int64_t)t.r0 * a.ks + w.kv_head * a.d;
  const uint16_t* V = a.V + (int64_t)t.r0 * a.vs + w.kv_head * a.d;
  const stages_of g = token_stages(a, t, row0);
  stage k, v;
  k.begin(K, a.ks, a.d, t.n, t.r0 + t.n == a.T);
  v.begin(V, a.vs, a.d, t.n, t.r0 + t.n == a.T);
  auto load = [&](int i) {
    unsigned char* to = lds + (i & 1) * BUF;
    k.load(g.first + i * SA_STAGE, to);
    v.load(g.first + i * SA_STAGE, to + stage::BYTES);
  };
  auto put = [&](int i) {
    unsigned char* to = lds + (i & 1) * BUF;
    k.store(to);
    v.store(to + stage::BYTES);
  };
  auto next = [&](int i) {
    wait_loads();
    __syncthreads();                                  // everybody's loads are there, and nobody reads the other buffer any more
    if (i + 1 < g.n) load(i + 1);
  };
  auto store = [&](int i) {
    if (i + 1 < g.n) put(i + 1);
  };
  load(0);
  if constexpr (!CAREFUL) {                             // (behind the first stage's loads, and under way together with them)
    load_columns<DP, DIRECT>(q, a.Q + ((int64_t)t.r0 + min(row, t.n - 1)) * a.qs + w.head * a.d, a.d);
    if (a.scale < 0.0f) negate<DP>(q);
  }
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) o[i] = f32x16_t{};
  m = -INFINITY;
  l = 0.0f;
  put(0);
  auto use = [&](int i, auto masked) {
    unsigned char* here = lds + (i & 1) * BUF;
    const int j0 = g.first + i * SA_STAGE;
    // (lanes behind the sequence's last row are that row once more, its window too: with one of their own they could see nothing of the masked stages, have
    // no reference in the others, and have the tile taken with care)
    const int last = min(row, t.n - 1), lim = (a.causal ? last : t.n - 1) - j0, low = first_token(a, last) - j0;
    if constexpr (CAREFUL) {
#pragma unroll 1
      for (int at = 0; at < SA_STAGE; at += 32) forward_block<DP>(a, here, here + stage::BYTES, at, q, o, m, l, low, lim);
    } else {
      forward_stage<DP, decltype(masked)::value>(a, here, here + stage::BYTES, q, o, m, l, low, lim);
    }
  };
  if constexpr (CAREFUL) {
    in_stages_alike(g, next, store, [&](int i) { use(i, std::true_type{}); });
  } else {
    // (the stage of the last row's first token is masked as well: there its reference is found)
    stages_of f = g;
    f.all = (first_token(a, min(row0 + 31, t.n - 1)) - g.first) / SA_STAGE + 1;
    in_stages<false>(f, next, store, use);
  }
}

template <int DP, bool DIRECT>
__global__ __launch_bounds__(256, 2) void self_forward_kernel(self_args a) {
  constexpr int NK = DP / 32;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  typedef stage_t<DP, DIRECT> stage;
  const self_place w = place_of(a);
  const self_tile t = find_self_tile(a, w.vt, a.causal);
  if (t.n == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row0 = t.at + 32 * wave, row = row0 + (lane & 31);
#pragma unroll
  for (int i = 0; i < 4; ++i) stage::clear(lds + i * stage::BYTES, a.d);
  bf16x8_t q[DP / 16];
  f32x16_t o[NK];
  float m, l;
  forward_tile<DP, DIRECT, false>(a, w, t, row0, q, o, m, l, lds);
  // An infinity or a NaN among values that not all rows of a wavefront see has reached all of them (0 times infinity): once more, with care.
  if (__builtin_expect(__syncthreads_or(any_nonfinite<NK>(o) || !(l < INFINITY)), 0)) forward_tile<DP, DIRECT, true>(a, w, t, row0, q, o, m, l, lds);
  l += other_half(l);
  if (row >= t.n) return;
  const int64_t out = ((int64_t)t.r0 + row) * a.heads + w.head;
  store_column<DP>(o, 1.0f / l, a.out + out * a.d, a.d);
  if (lane < 32) a.lse[out] = (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// ---------------------------------------------------------------------------------------------
// Gradient of the queries.  Leaves lse and delta head by head for the other kernel.
// ---------------------------------------------------------------------------------------------
// Rows that see one token have p = 1 whatever its score: no gradient passes through it.
__device__ __forceinline__ bool see_one(const self_args& a, int n) { return n == 1 || a.window == 1; }

// Wavefronts a SIMD of the backward kernels: their accumulators and both operands that stay take 1.5 DP registers, of 256 or 512 (heads of 96 with two
// wavefronts spill).
template <int DP> constexpr int backward_waves() { return DP > 64 ? 1 : 2; }

// delta is dO . O with O as it was rounded to bf16, which costs dS as much as all else together; what is missing to sum_j p_ij dP_ij is the sum of
// the dS themselves, known at the end.  So the products with p are kept beside those with dS (they share their other operand), and dQ is put right by
// them: dQ = sum (dS - p sum dS) k.  With the sum of the dS as they were rounded for the product, which takes the part of their roundings that the
// mean of the k would carry out as well: the true dS add up to nothing.  (Relative error of dQ: 3.6e-3 to 4.7e-3 with delta from the rounded O, 2.8e-3 to
// 3.1e-3 with the exact sum of the dS, 2.4e-3 so.  The other kernel gets delta with the exact sum; with that of the rounded dS, dK's error
// was 2.6e-3 instead of 2.3e-3.)
//
// Four products a tile (scores, dP, dS k, p k), as many as the kernel below: eight in all where five would do if dQ were added to by the workgroups of
// all tokens, with atomics whose order changes results or parts of it in memory.  8192 causal rows, 32 heads of 128 on eight: 1050 us a kernel, 650
// TFLOP/s of the five products, 1040 of the eight; the matrix pipe is busy 47 % of the cycles (46 % below; heads of 64: 45 % and 43 %).  A lone
// wavefront takes 1.9 us for a stage and still 1.4 us with its products left out, so what bounds both is the issue of one wavefront's vector
// instructions (one in about 5 cycles), not LDS (no bank conflicts) or loads.
template <int DP, bool MASKED, int CARE>
__device__ __forceinline__ void query_blocks(const self_args& a, const unsigned char* lk, const unsigned char* lv, int at, const bf16x8_t* q,
                                             const bf16x8_t* g, f32x16_t* dq, f32x16_t* pk, float lse, float delta, float& rest, float& rest_odd, float& rounded, int low, int lim) {
  constexpr int NK = DP / 32, NB = CARE == PLAIN ? 2 : 1;
  const int h = (threadIdx.x & 63) >> 5;
  f32x16_t s[NB], dp[NB];
  uint32_t seen[NB];
  constexpr int N = DP / 16;
  bf16x8_t x[2][N];              // operands of the present phase and, being read, of the next
  auto scores = [&](int b, const bf16x8_t* o) {
    s[b] = f32x16_t{};
#pragma unroll
    for (int k = 0; k < N; ++k) s[b] = mfma(o[k], q[k], s[b]);
  };
  auto slopes = [&](int b, const bf16x8_t* o) {
#pragma unroll
    for (int j = 0; j < 16; ++j) dp[b][j] = -delta;
#pragma unroll
    for (int k = 0; k < N; ++k) dp[b] = mfma(o[k], g[k], dp[b]);
  };
  auto weights = [&](int b) {
    seen[b] = bits_between(low - at - 32 * b, lim - at - 32 * b) >> (4 * h);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], a.c, -lse));
      if constexpr (MASKED) s[b][j] = where_set(s[b][j], seen[b], tile_row(j));
    }
  };
  auto through = [&](int b) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      // (without care 0 times what is not finite is NaN, and has the tile taken with care)
      dp[b][j] = CARE == CAREFUL ? where_set(s[b][j] * dp[b][j], seen[b], tile_row(j)) : s[b][j] * dp[b][j];
      rest += dp[b][j];
    }
  };
  auto products = [&](int b, const bf16x8_t* o) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8_t x = as_operand(dp[b], u), p = as_operand(s[b], u);
      rounded = sum_of(x, rounded);
      bf16x8_t left;
      if constexpr (CARE == FINE) {
        left = as_remainder(dp[b], u, x);
        rounded = sum_of(left, rounded);
      }
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const bf16x8_t k = o[u * NK + i];
        if constexpr (CARE == CAREFUL) {
          dq[i] = mfma_seen(k, x, register_bits(seen[b], u), dq[i]);
          pk[i] = mfma_seen(k, p, register_bits(seen[b], u), pk[i]);
        } else {
          dq[i] = mfma(k, x, dq[i]);
          pk[i] = mfma(k, p, pk[i]);
          if constexpr (CARE == FINE) dq[i] = mfma(k, left, dq[i]);
        }
      }
    }
  };
  if constexpr (CARE != PLAIN) {
    row_operands<DP>(x[0], lk, at);
    scores(0, x[0]);
    row_operands<DP>(x[1], lv, at);
    slopes(0, x[1]);
    weights(0);
    through(0);
    column_operands<DP>(x[0], lk, at);
    products(0, x[0]);
  } else {
    uint32_t pw[2][8], xw[2][8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = f32x16_t{};
#pragma unroll
      for (int j = 0; j < 16; ++j) dp[b][j] = -delta;
      if constexpr (MASKED) seen[b] = bits_between(low - at - 32 * b, lim - at - 32 * b) >> (4 * h);
    }
    auto weight = [&](int b, int y) {
#pragma unroll
      for (int j = 2 * y; j < 2 * y + 2; ++j) {
        s[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], a.c, -lse));
        if constexpr (MASKED) s[b][j] = where_set(s[b][j], seen[b], tile_row(j));
      }
      pw[b][y] = round_two(s[b][2 * y], s[b][2 * y + 1]);
    };
    auto slope = [&](int b, int y) {
      const float x0 = s[b][2 * y] * dp[b][2 * y], x1 = s[b][2 * y + 1] * dp[b][2 * y + 1];
      rest += x0;
      rest_odd += x1;
      xw[b][y] = round_two(x0, x1);
      rounded = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, xw[b][y]), bf16x2_t{(__bf16)1.0f, (__bf16)1.0f}, rounded, false);
    };
    auto product = [&](int b, int j) {
      dq[j % NK] = mfma(x[b][j], four_pairs(xw[b] + 4 * (j / NK)), dq[j % NK]);
      pk[j % NK] = mfma(x[b][j], four_pairs(pw[b] + 4 * (j / NK)), pk[j % NK]);
    };
    row_operands<DP>(x[0], lk, at);
    __builtin_amdgcn_sched_barrier(0);
    phase<N>([&](int k) { s[0] = mfma(x[0][k], q[k], s[0]); }, [&](int k) { x[1][k] = row_operand<DP>(lv, at, k); }, nothing{});
    phase<N>([&](int k) { dp[0] = mfma(x[1][k], g[k], dp[0]); }, [&](int k) { x[0][k] = row_operand<DP>(lk, at + 32, k); }, [&](int y) { weight(0, y); });
    phase<N>([&](int k) { s[1] = mfma(x[0][k], q[k], s[1]); }, [&](int k) { x[1][k] = row_operand<DP>(lv, at + 32, k); }, [&](int y) { slope(0, y); });
    phase<N>([&](int k) { dp[1] = mfma(x[1][k], g[k], dp[1]); }, [&](int k) { x[0][k] = nth_column_operand<DP>(lk, at, k); }, [&](int y) { weight(1, y); });
    phase<N>([&](int k) { product(0, k); }, [&](int k) { x[1][k] = nth_column_operand<DP>(lk, at + 32, k); }, [&](int y) { slope(1, y); });
    phase<N>([&](int k) { product(1, k); }, nothing{}, nothing{});
  }
}

template <int DP, bool DIRECT, int CARE>
__device__ __forceinline__ void query_tile(const self_args& a, const self_place& w, const self_tile& t, int row0, bf16x8_t* q, bf16x8_t* g,
                                           f32x16_t* dq, f32x16_t* pk, float& lse, float& delta, float& rest, float& rest_odd, float& rounded, unsigned char* lds) {
  typedef stage_t<DP, DIRECT> stage;
  constexpr int BUF = 2 * stage::BYTES;
  const int row = row0 + (threadIdx.x & 31);
  const uint16_t* K = a.K + (int64_t)t.r0 * a.ks + w.kv_head * a.d;
  const uint16_t* V = a.V + (int64_t)t.r0 * a.vs + w.kv_head * a.d;
  const stages_of st = token_stages(a, t, row0);
  const bool fine = a.causal ? row0 < SA_STAGE : t.n <= SA_STAGE;
  stage k, v;
  k.begin(K, a.ks, a.d, t.n, t.r0 + t.n == a.T);
  v.begin(V, a.vs, a.d, t.n, t.r0 + t.n == a.T);
  auto load = [&](int i) {
    unsigned char* to = lds + (i & 1) * BUF;
    k.load(st.first + i * SA_STAGE, to);
    v.load(st.first + i * SA_STAGE, to + stage::BYTES);
  };
  auto put = [&](int i) {
    unsigned char* to = lds + (i & 1) * BUF;
    k.store(to);
    v.store(to + stage::BYTES);
  };
  auto next = [&](int i) {
    wait_loads();
    __syncthreads();
    if (i + 1 < st.n) load(i + 1);
  };
  auto store = [&](int i) {
    if (i + 1 < st.n) put(i + 1);
  };
  load(0);
  if constexpr (CARE != CAREFUL) {
    const int64_t mine = (int64_t)t.r0 + min(row, t.n - 1);
    bf16x8_t o[DP / 16];
    load_columns<DP, DIRECT>(q, a.Q + mine * a.qs + w.head * a.d, a.d);
    load_columns<DP, DIRECT>(g, a.dO + (mine * a.heads + w.head) * a.d, a.d);
    load_columns<DP, DIRECT>(o, a.O + (mine * a.heads + w.head) * a.d, a.d);
    lse = a.lse[mine * a.heads + w.head] * SA_LOG2E;
    if (a.scale < 0.0f) negate<DP>(q);
    float sum[4] = {};
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j & 3] = __builtin_fmaf((float)o[s][j], (float)g[s][j], sum[j & 3]);
    delta = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    delta += other_half(delta);
  }
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) dq[i] = pk[i] = f32x16_t{};
  rest = rest_odd = rounded = 0.0f;
  put(0);
  auto use = [&](int i, auto masked) {
    unsigned char* here = lds + (i & 1) * BUF;
    const int j0 = st.first + i * SA_STAGE;
    const int lim = (a.causal ? min(row, t.n - 1) : t.n - 1) - j0, low = first_token(a, row) - j0;
    constexpr int HERE = std::is_same<decltype(masked), fine_t>::value ? FINE : CARE, NB = HERE == PLAIN ? 2 : 1;
#pragma unroll 1
    for (int at = 0; at < SA_STAGE; at += 32 * NB)
      query_blocks<DP, decltype(masked)::value, HERE>(a, here, here + stage::BYTES, at, q, g, dq, pk, lse, delta, rest, rest_odd, rounded, low, lim);
  };
  if constexpr (CARE == CAREFUL) in_stages_alike(st, next, store, [&](int i) { use(i, std::true_type{}); });
  else in_stages<true>(st, next, store, use, fine);
}

template <int DP, bool DIRECT>
__global__ __launch_bounds__(256, backward_waves<DP>()) void self_query_kernel(self_args a) {
  constexpr int NK = DP / 32;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  typedef stage_t<DP, DIRECT> stage;
  const self_place w = place_of(a);
  const self_tile t = find_self_tile(a, w.vt, a.causal);
  if (t.n == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row0 = t.at + 32 * wave, row = row0 + (lane & 31);
#pragma unroll
  for (int i = 0; i < 4; ++i) stage::clear(lds + i * stage::BYTES, a.d);
  const int64_t mine = (int64_t)t.r0 + min(row, t.n - 1);
  bf16x8_t q[DP / 16], g[DP / 16];
  float lse, delta;
  f32x16_t dq[NK], pk[NK];
  float rest, rest_odd, rounded;
  query_tile<DP, DIRECT, PLAIN>(a, w, t, row0, q, g, dq, pk, lse, delta, rest, rest_odd, rounded, lds);
  if (__builtin_expect(__syncthreads_or(any_nonfinite<NK>(dq) || any_nonfinite<NK>(pk)), 0))
    query_tile<DP, DIRECT, CAREFUL>(a, w, t, row0, q, g, dq, pk, lse, delta, rest, rest_odd, rounded, lds);
  rest += rest_odd;
  rest += other_half(rest);
  rounded += other_half(rounded);
  if (row >= t.n) return;
  if (lane < 32) a.stats[(int64_t)w.head * a.T + mine] = make_float2(lse, delta + rest);
  const bool one = see_one(a, t.n) || (a.causal && row == 0);
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) dq[i][j] = one ? 0.0f : dq[i][j] - rounded * pk[i][j];
  store_column<DP>(dq, a.scale, a.dQ + mine * a.dqs + w.head * a.d, a.d);
}

// ---------------------------------------------------------------------------------------------
// Gradients of the keys and values
// ---------------------------------------------------------------------------------------------
template <int DP, bool MASKED, int CARE>
__device__ __forceinline__ void token_blocks(const self_args& a, const unsigned char* lq, const unsigned char* lg, const float* lst, int at, int low, int lim,
                                             const bf16x8_t* k, const bf16x8_t* v, f32x16_t* dk, f32x16_t* dv) {
  constexpr int NK = DP / 32, NB = CARE == PLAIN ? 2 : 1;
  const int h = (threadIdx.x & 63) >> 5;
  f32x16_t s[NB], dp[NB];
  uint32_t seen[NB];
  constexpr int N = DP / 16;
  const bf16x8_t* k_of = k;      // (`k` counts steps below)
  bf16x8_t o[2][N];              // operands of the present phase and, being read, of the next
  f32x4_t lse[NB][4];            // (-lse log2 e)
  auto sums = [&](int b) {       // and -delta, which dP begins with
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      lse[b][y] = *reinterpret_cast<const f32x4_t*>(lst + at + 32 * b + 8 * y + 4 * h);
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(lst + SA_STAGE + at + 32 * b + 8 * y + 4 * h);
#pragma unroll
      for (int j = 0; j < 4; ++j) dp[b][4 * y + j] = x[j];
    }
  };
  auto scores = [&](int b, const bf16x8_t* o) {
    s[b] = f32x16_t{};
#pragma unroll
    for (int x = 0; x < N; ++x) s[b] = mfma(o[x], k[x], s[b]);
  };
  auto slopes = [&](int b, const bf16x8_t* o) {
#pragma unroll
    for (int x = 0; x < N; ++x) dp[b] = mfma(o[x], v[x], dp[b]);
  };
  auto weights = [&](int b) {
    seen[b] = bits_between(low - at - 32 * b, lim - at - 32 * b) >> (4 * h);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      s[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], a.c, lse[b][j >> 2][j & 3]));
      if constexpr (MASKED) s[b][j] = where_set(s[b][j], seen[b], tile_row(j));
    }
  };
  auto through = [&](int b) {
#pragma unroll
    for (int j = 0; j < 16; ++j) dp[b][j] = CARE == CAREFUL ? where_set(s[b][j] * dp[b][j], seen[b], tile_row(j)) : s[b][j] * dp[b][j];
  };
  auto value_products = [&](int b, const bf16x8_t* o) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8_t x = as_operand(s[b], u);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        if constexpr (CARE == CAREFUL) dv[i] = mfma_seen(o[u * NK + i], x, register_bits(seen[b], u), dv[i]);
        else dv[i] = mfma(o[u * NK + i], x, dv[i]);
        if constexpr (CARE == FINE) dv[i] = mfma(o[u * NK + i], as_remainder(s[b], u, x), dv[i]);
      }
    }
  };
  auto key_products = [&](int b, const bf16x8_t* o) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16x8_t x = as_operand(dp[b], u);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        if constexpr (CARE == CAREFUL) dk[i] = mfma_seen(o[u * NK + i], x, register_bits(seen[b], u), dk[i]);
        else dk[i] = mfma(o[u * NK + i], x, dk[i]);
        if constexpr (CARE == FINE) dk[i] = mfma(o[u * NK + i], as_remainder(dp[b], u, x), dk[i]);
      }
    }
  };
  if constexpr (CARE != PLAIN) {
    row_operands<DP>(o[0], lq, at);
    scores(0, o[0]);
    sums(0);
    row_operands<DP>(o[1], lg, at);
    slopes(0, o[1]);
    weights(0);
    through(0);
    column_operands<DP>(o[0], lg, at);
    value_products(0, o[0]);
    column_operands<DP>(o[1], lq, at);
    key_products(0, o[1]);
  } else {
    uint32_t pw[2][8], xw[2][8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = f32x16_t{};
      if constexpr (MASKED) seen[b] = bits_between(low - at - 32 * b, lim - at - 32 * b) >> (4 * h);
    }
    auto weight = [&](int b, int y) {
#pragma unroll
      for (int j = 2 * y; j < 2 * y + 2; ++j) {
        s[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], a.c, lse[b][j >> 2][j & 3]));
        if constexpr (MASKED) s[b][j] = where_set(s[b][j], seen[b], tile_row(j));
      }
      pw[b][y] = round_two(s[b][2 * y], s[b][2 * y + 1]);
    };
    auto slope = [&](int b, int y) { xw[b][y] = round_two(s[b][2 * y] * dp[b][2 * y], s[b][2 * y + 1] * dp[b][2 * y + 1]); };
    auto value_product = [&](int b, const bf16x8_t* o, int j) { dv[j % NK] = mfma(o[j], four_pairs(pw[b] + 4 * (j / NK)), dv[j % NK]); };
    auto key_product = [&](int b, const bf16x8_t* o, int j) { dk[j % NK] = mfma(o[j], four_pairs(xw[b] + 4 * (j / NK)), dk[j % NK]); };
    row_operands<DP>(o[0], lq, at);
    sums(0);
    __builtin_amdgcn_sched_barrier(0);
    phase<N>([&](int k) { s[0] = mfma(o[0][k], k_of[k], s[0]); }, [&](int k) { o[1][k] = row_operand<DP>(lg, at, k); }, nothing{});
    sums(1);
    phase<N>([&](int k) { dp[0] = mfma(o[1][k], v[k], dp[0]); }, [&](int k) { o[0][k] = row_operand<DP>(lq, at + 32, k); }, [&](int y) { weight(0, y); });
    phase<N>([&](int k) { s[1] = mfma(o[0][k], k_of[k], s[1]); }, [&](int k) { o[1][k] = row_operand<DP>(lg, at + 32, k); }, [&](int y) { slope(0, y); });
    phase<N>([&](int k) { dp[1] = mfma(o[1][k], v[k], dp[1]); }, [&](int k) { o[0][k] = nth_column_operand<DP>(lg, at, k); }, [&](int y) { weight(1, y); });
    phase<N>([&](int k) { value_product(0, o[0], k); }, [&](int k) { o[1][k] = nth_column_operand<DP>(lq, at, k); }, [&](int y) { slope(1, y); });
    phase<N>([&](int k) { key_product(0, o[1], k); }, [&](int k) { o[0][k] = nth_column_operand<DP>(lg, at + 32, k); }, nothing{});
    phase<N>([&](int k) { value_product(1, o[0], k); }, [&](int k) { o[1][k] = nth_column_operand<DP>(lq, at + 32, k); }, nothing{});
    phase<N>([&](int k) { key_product(1, o[1], k); }, nothing{}, nothing{});
  }
}

template <int DP, bool DIRECT, int CARE>
__device__ __forceinline__ void token_tile(const self_args& a, int kv_head, const self_tile& t, int tok0, int piece, bf16x8_t* k, bf16x8_t* v,
                                           f32x16_t* dk, f32x16_t* dv, unsigned char* lds) {
  typedef stage_t<DP, DIRECT> stage;
  constexpr int BUF = 2 * stage::BYTES + SA_STAGE * 8;
  const int tok = tok0 + (threadIdx.x & 31);
  const stages_of all = row_stages(a, t, tok0);
  const bool fine = all.first == 0 && (a.causal || t.n <= SA_STAGE);
  // The stages of the heads that share the tile one behind the other, and of these the piece's.
  const int steps = all.n * a.group, begin = (int)((int64_t)steps * piece / a.pieces), end = (int)((int64_t)steps * (piece + 1) / a.pieces);
  const uint16_t* Q = a.Q + (int64_t)t.r0 * a.qs + (int64_t)kv_head * a.group * a.d;
  const uint16_t* G = a.dO + ((int64_t)t.r0 * a.heads + (int64_t)kv_head * a.group) * a.d;
  const int64_t gs = (int64_t)a.heads * a.d;
  stage q, g;
  q.begin(Q, a.qs, a.d, t.n, t.r0 + t.n == a.T);
  g.begin(G, gs, a.d, t.n, t.r0 + t.n == a.T);
  float2 sums = make_float2(0.0f, 0.0f);
  int at = 0;                                          // the buffer of the present stage
  auto load = [&](int head, int i, int to_at) {
    unsigned char* to = lds + to_at * BUF;
    const int i0 = all.first + i * SA_STAGE;
    q.base = Q + head * a.d;
    g.base = G + head * a.d;
    q.load(i0, to);
    g.load(i0, to + stage::BYTES);
    if (threadIdx.x < SA_STAGE)
      sums = a.stats[(int64_t)(kv_head * a.group + head) * a.T + t.r0 + min(i0 + (int)threadIdx.x, t.n - 1)];
  };
  auto put = [&](int to_at) {
    unsigned char* to = lds + to_at * BUF;
    q.store(to);
    g.store(to + stage::BYTES);
    if (threadIdx.x < SA_STAGE) {
      float* s = reinterpret_cast<float*>(to + 2 * stage::BYTES);
      s[threadIdx.x] = -sums.x;
      s[SA_STAGE + threadIdx.x] = -sums.y;
    }
  };
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) dk[i] = dv[i] = f32x16_t{};
  if (begin == end) return;
  const int head0 = begin / all.n, head1 = (end - 1) / all.n;
  load(head0, begin - head0 * all.n, 0);
  if constexpr (CARE != CAREFUL) {
    const int64_t mine = (int64_t)t.r0 + min(tok, t.n - 1);
    load_columns<DP, DIRECT>(k, a.K + mine * a.ks + kv_head * a.d, a.d);
    load_columns<DP, DIRECT>(v, a.V + mine * a.vs + kv_head * a.d, a.d);
    if (a.scale < 0.0f) negate<DP>(k);
  }
  put(0);
#pragma unroll 1
  for (int head = head0; head <= head1; ++head) {
    stages_of st = all;
    st.begin = max(begin - head * all.n, 0);
    st.n = min(end - head * all.n, all.n);
    st.to = min(all.to, st.n);
    auto more = [&](int i) { return i + 1 < st.n || head < head1; };
    auto next = [&](int i) {
      wait_loads();
      __syncthreads();
      if (more(i)) {
        const bool same = i + 1 < st.n;
        load(same ? head : head + 1, same ? i + 1 : 0, at ^ 1);
      }
    };
    auto store = [&](int i) {
      at ^= 1;
      if (more(i)) put(at);
    };
    auto use = [&](int i, auto masked) {
      unsigned char* here = lds + at * BUF;
      const float* lst = reinterpret_cast<const float*>(here + 2 * stage::BYTES);
      const int i0 = st.first + i * SA_STAGE;
      const int low = (a.causal ? tok : 0) - i0, lim = first_blind_row(a, t.n, tok) - 1 - i0;      // the rows that see the lane's token
      constexpr int HERE = std::is_same<decltype(masked), fine_t>::value ? FINE : CARE, NB = HERE == PLAIN ? 2 : 1;
#pragma unroll 1
      for (int x = 0; x < SA_STAGE; x += 32 * NB)
        token_blocks<DP, decltype(masked)::value, HERE>(a, here, here + stage::BYTES, lst, x, low, lim, k, v, dk, dv);
    };
    if constexpr (CARE == CAREFUL) in_stages_alike(st, next, store, [&](int i) { use(i, std::true_type{}); });
    else in_stages<true>(st, next, store, use, fine);
  }
}

template <int DP, bool DIRECT>
__global__ __launch_bounds__(256, backward_waves<DP>()) void self_token_kernel(self_args a) {
  constexpr int NK = DP / 32;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  typedef stage_t<DP, DIRECT> stage;
  const int per_tile = a.kv_heads * a.pieces, vt = blockIdx.x / per_tile, x = blockIdx.x - vt * per_tile, kv_head = x % a.kv_heads, piece = x / a.kv_heads;
  const self_tile t = find_self_tile(a, vt, false);
  if (t.n == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int tok0 = t.at + 32 * wave, tok = tok0 + (lane & 31);
  constexpr int BUF = 2 * stage::BYTES + SA_STAGE * 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) stage::clear(lds + (i >> 1) * BUF + (i & 1) * stage::BYTES, a.d);
  const int64_t mine = (int64_t)t.r0 + min(tok, t.n - 1);
  bf16x8_t k[DP / 16], v[DP / 16];
  f32x16_t dk[NK], dv[NK];
  token_tile<DP, DIRECT, PLAIN>(a, kv_head, t, tok0, piece, k, v, dk, dv, lds);
  if (__builtin_expect(__syncthreads_or(any_nonfinite<NK>(dk) || any_nonfinite<NK>(dv)), 0))
    token_tile<DP, DIRECT, CAREFUL>(a, kv_head, t, tok0, piece, k, v, dk, dv, lds);
  if (tok >= t.n) return;
  const float f = see_one(a, t.n) ? 0.0f : a.scale;
  if (a.pieces == 1) {
    store_column<DP>(dk, f, a.dK + mine * a.dks + kv_head * a.d, a.d);
    store_column<DP>(dv, 1.0f, a.dV + mine * a.dvs + kv_head * a.d, a.d);
  } else {
    float* to = a.parts + (((int64_t)piece * a.T + mine) * a.kv_heads + kv_head) * 2 * a.d;
    store_part<DP>(dk, f, to, a.d);
    store_part<DP>(dv, 1.0f, to + a.d, a.d);
  }
}

// The pieces' parts of dK and dV added in their order, two neighbouring elements a lane.  Rows of no sequence are left alone.  Bound by memory, most of it
// from the last-level cache.
__global__ __launch_bounds__(256) void self_join_kernel(self_args a) {
  const int half = a.d / 2, per_row = a.kv_heads * 2 * half;
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x, row = x / per_row;
  if (row >= min(max(a.row_start[a.n_seqs], 0), a.T) || row < max(a.row_start[0], 0)) return;
  const int y = (int)(x - row * per_row), kv = y / (2 * half), z = y - kv * 2 * half, which = z / half, e = 2 * (z - which * half);
  const int64_t stride = (int64_t)a.T * a.kv_heads * 2 * a.d;
  const float* from = a.parts + (row * a.kv_heads + kv) * 2 * a.d + which * a.d + e;
  float2 sum = *reinterpret_cast<const float2*>(from);
  for (int i = 1; i < a.pieces; ++i) {
    const float2 p = *reinterpret_cast<const float2*>(from + i * stride);
    sum.x += p.x;
    sum.y += p.y;
  }
  uint16_t* to = which ? a.dV + row * a.dvs : a.dK + row * a.dks;
  *reinterpret_cast<uint32_t*>(to + (int64_t)kv * a.d + e) = round_two(sum.x, sum.y);
}

// ---------------------------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------------------------
int check_self(const pq_self_attn_desc* d) {
  PQ_REQUIRE(d, PQ_ERR_BAD_ARG, "NULL descriptor");
  PQ_REQUIRE(d->n_seqs >= 0, PQ_ERR_BAD_ARG, "n_seqs=%d is negative", d->n_seqs);
  PQ_REQUIRE(d->n_heads > 0 && d->n_kv_heads > 0 && d->n_heads % d->n_kv_heads == 0, PQ_ERR_SHAPE, "n_heads=%d must be a multiple of n_kv_heads=%d",
             d->n_heads, d->n_kv_heads);
  PQ_REQUIRE(d->d_head >= 2 && d->d_head <= 128 && d->d_head % 2 == 0, PQ_ERR_SHAPE, "d_head=%d must be even and in 2..128", d->d_head);
  PQ_REQUIRE((int64_t)d->n_heads * d->d_head <= (1 << 23), PQ_ERR_SHAPE, "n_heads=%d of %d are more than 2^23 elements", d->n_heads, d->d_head);
  PQ_REQUIRE(d->causal == 0 || d->causal == 1, PQ_ERR_BAD_ARG, "causal=%d must be 0 or 1", d->causal);
  PQ_REQUIRE(d->window >= 0 && (d->causal || d->window == 0), PQ_ERR_BAD_ARG, "window=%d must not be negative, and needs causal", d->window);
  PQ_REQUIRE(std::isfinite(d->scale), PQ_ERR_BAD_ARG, "scale must be finite");
  return PQ_OK;
}
int check_rows(const pq_self_attn_desc* d, int T) {
  PQ_REQUIRE(T >= 0, PQ_ERR_BAD_ARG, "T=%d is negative", T);
  PQ_REQUIRE(T <= (1 << 29) && (int64_t)T * d->n_heads <= 0x7fffffff &&
                 ((int64_t)T / SA_ROWS + d->n_seqs) * d->n_heads <= PQ_MOST_WORKGROUPS, PQ_ERR_SHAPE, "%d rows of %d heads in %d sequences are too many for one call",
             T, d->n_heads, d->n_seqs);
  return PQ_OK;
}
int check_stride(const char* name, int64_t stride, int heads, int d) {
  PQ_REQUIRE(stride >= (int64_t)heads * d && stride % 2 == 0 && stride <= (1 << 23), PQ_ERR_SHAPE,
             "%s: row stride %lld must be even, at least %lld and at most 2^23", name, (long long)stride, (long long)heads * d);
  return PQ_OK;
}
bool at16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// T rows of `heads` heads, `stride` elements apart.
pq_region rows_region(const char* name, const void* p, int T, int64_t stride, int heads, int d) {
  return {name, (uintptr_t)p, T, stride * 2, (int64_t)heads * d * 2, 0};
}
pq_region row_start_region(const pq_self_attn_desc* d, const int32_t* row_start) {
  return pq_flat_region("row_start", row_start, ((int64_t)d->n_seqs + 1) * 4);
}

// Pieces of a token tile's work, whose parts are joined in their order.  As many as give 512 workgroups, of 8 stages each at least (16 heads of 64 on one,
// 2000 rows: 91 us, 713 in one piece; 4 heads of 128 on one, 1000 rows: 72, in pieces of 16 stages 83, in one 168).  Tiles of causal rows differ
// in length and come in few rounds, so long ones are cut further: to 2048 workgroups of 64 stages where two share a CU (32 heads of 64 on four, 10000
// rows: 1560 us, uncut 2500; on eight, 8192 rows: 1060 and 1230; cut to 4096 1616 and 1124), to 1024 of 32 where one has it alone (32 heads of 128
// on eight, 5000 rows: 900, uncut 1040, cut to 2048 980; 8192 rows, which stay whole: 2150, cut 2210).  Whole sequences gain as well, from fewer
// tiles (of 2000 rows, 32 heads of 64 on eight: 159 us, uncut 244; 5000 rows of 128: 1700 and 2056; 8192 of 64 lose 2 %).  Stages by the window (5000 rows, a window of 512:
// 311 uncut, 335 and 411 in pieces) and, for the second cut, by the sequences' mean length (16 of 512 rows: 295, cut 387).
int token_pieces(const pq_self_attn_desc* d, int T) {
  const int64_t tiles = ((int64_t)T / SA_ROWS + d->n_seqs) * d->n_kv_heads, group = d->n_heads / d->n_kv_heads;
  if (tiles == 0 || d->n_seqs == 0) return 1;
  auto stages = [&](int64_t rows) {
    if (d->window > 0 && rows > (int64_t)d->window + SA_ROWS) rows = (int64_t)d->window + SA_ROWS;
    return group * (rows / SA_STAGE + 1);
  };
  const bool alone = d->d_head > 64;           // a workgroup on its CU
  const int64_t few = std::min(512 / tiles, stages(T) / 8);
  const int64_t even = std::min((alone ? 1024 : 2048) / tiles, stages(T / d->n_seqs) / (alone ? 32 : 64));
  return (int)std::min<int64_t>(std::max<int64_t>(std::max(few, even), 1), 32);
}
size_t part_bytes(const pq_self_attn_desc* d, int T) { return (size_t)T * d->n_kv_heads * 2 * d->d_head * sizeof(float); }
size_t stats_bytes(const pq_self_attn_desc* d, int T) { return pq_align_up((size_t)T * d->n_heads * sizeof(float2), 256); }

self_args make_args(const pq_self_attn_desc* d, int T, const int32_t* row_start) {
  self_args a = {};
  a.T = T; a.n_seqs = d->n_seqs; a.heads = d->n_heads; a.kv_heads = d->n_kv_heads; a.group = d->n_heads / d->n_kv_heads; a.d = d->d_head;
  a.causal = d->causal; a.window = d->window; a.tiles = T / SA_ROWS + d->n_seqs;
  a.c = fabsf(d->scale) * SA_LOG2E;
  a.scale = d->scale;
  a.row_start = row_start;
  return a;
}

int allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& asked) {
  if (bytes <= 65536) return PQ_OK;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return pq_set_error(PQ_ERR_HIP, "hipGetDevice failed");
  const uint64_t bit = (uint64_t)1 << (dev & 63);
  if (asked.load(std::memory_order_relaxed) & bit) return PQ_OK;
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)
    return pq_set_error(PQ_ERR_HIP, "hipFuncSetAttribute failed for an attention kernel");
  asked.fetch_or(bit, std::memory_order_relaxed);
  return PQ_OK;
}

template <int DP, bool DIRECT> int launch_forward(const self_args& a, hipStream_t s) {
  static std::atomic<uint64_t> asked;
  constexpr int lds = 4 * stage_t<DP, DIRECT>::BYTES;
  if (int e = allow_lds((const void*)self_forward_kernel<DP, DIRECT>, lds, asked)) return e;
  self_forward_kernel<DP, DIRECT><<<(unsigned)(a.tiles * a.heads), 256, lds, s>>>(a);
  PQ_CHECK_LAUNCH("self_forward_kernel");
  return PQ_OK;
}
template <int DP, bool DIRECT> int launch_backward(const self_args& a, hipStream_t s) {
  static std::atomic<uint64_t> asked[2];
  constexpr int lds = 4 * stage_t<DP, DIRECT>::BYTES;
  if (int e = allow_lds((const void*)self_query_kernel<DP, DIRECT>, lds, asked[0])) return e;
  if (int e = allow_lds((const void*)self_token_kernel<DP, DIRECT>, lds + SA_STAGE * 16, asked[1])) return e;
  self_query_kernel<DP, DIRECT><<<(unsigned)(a.tiles * a.heads), 256, lds, s>>>(a);
  PQ_CHECK_LAUNCH("self_query_kernel");
  self_token_kernel<DP, DIRECT><<<(unsigned)(a.tiles * a.kv_heads * a.pieces), 256, lds + SA_STAGE * 16, s>>>(a);
  PQ_CHECK_LAUNCH("self_token_kernel");
  if (a.pieces > 1) {
    self_join_kernel<<<(unsigned)(((int64_t)a.T * a.kv_heads * a.d + 255) / 256), 256, 0, s>>>(a);
    PQ_CHECK_LAUNCH("self_join_kernel");
  }
  return PQ_OK;
}
template <bool DIRECT> int launch_forward_d(const self_args& a, hipStream_t s) {
  switch ((a.d + 31) / 32) {
    case 1: return launch_forward<32, DIRECT>(a, s);
    case 2: return launch_forward<64, DIRECT>(a, s);
    case 3: return launch_forward<96, DIRECT>(a, s);
    default: return launch_forward<128, DIRECT>(a, s);
  }
}
template <bool DIRECT> int launch_backward_d(const self_args& a, hipStream_t s) {
  switch ((a.d + 31) / 32) {
    case 1: return launch_backward<32, DIRECT>(a, s);
    case 2: return launch_backward<64, DIRECT>(a, s);
    case 3: return launch_backward<96, DIRECT>(a, s);
    default: return launch_backward<128, DIRECT>(a, s);
  }
}

}  // namespace

extern "C" int pq_self_attn_fwd(const pq_self_attn_desc* d, const void* Q, int64_t q_stride, const void* K, int64_t k_stride, const void* V,
                                int64_t v_stride, int32_t T, const int32_t* row_start, void* O, float* lse, void* stream) {
  if (int e = check_self(d)) return e;
  if (int e = check_rows(d, T)) return e;
  if (T == 0 || d->n_seqs == 0) return PQ_OK;
  PQ_REQUIRE(Q && K && V && O && lse && row_start, PQ_ERR_BAD_ARG, "NULL buffer");
  if (int e = check_stride("Q", q_stride, d->n_heads, d->d_head)) return e;
  if (int e = check_stride("K", k_stride, d->n_kv_heads, d->d_head)) return e;
  if (int e = check_stride("V", v_stride, d->n_kv_heads, d->d_head)) return e;
  PQ_REQUIRE(at16(Q) && at16(K) && at16(V) && at16(O), PQ_ERR_SHAPE, "buffers must be 16-byte aligned");
  const int H = d->n_heads, Hk = d->n_kv_heads, dh = d->d_head;
  const pq_region written[] = {rows_region("O", O, T, (int64_t)H * dh, H, dh), pq_flat_region("lse", lse, (int64_t)T * H * 4)};
  const pq_region read[] = {rows_region("Q", Q, T, q_stride, H, dh), rows_region("K", K, T, k_stride, Hk, dh), rows_region("V", V, T, v_stride, Hk, dh),
                            row_start_region(d, row_start)};
  if (int e = pq_refuse_overlap(written, 2, read, 4)) return e;
  self_args a = make_args(d, T, row_start);
  a.Q = (const uint16_t*)Q; a.K = (const uint16_t*)K; a.V = (const uint16_t*)V;
  a.qs = q_stride; a.ks = k_stride; a.vs = v_stride;
  a.out = (uint16_t*)O; a.lse = lse;
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_SELF_ATTN_FWD, s);
  const bool direct = a.d % 8 == 0 && q_stride % 8 == 0 && k_stride % 8 == 0 && v_stride % 8 == 0;
  return direct ? launch_forward_d<true>(a, s) : launch_forward_d<false>(a, s);
}

extern "C" size_t pq_self_attn_bwd_workspace_bytes(const pq_self_attn_desc* d, int32_t T) {
  if (check_self(d) || check_rows(d, T)) return 0;
  const int pieces = token_pieces(d, T);
  return stats_bytes(d, T) + (pieces > 1 ? pieces * part_bytes(d, T) : 0) + 256;
}

extern "C" int pq_self_attn_bwd(const pq_self_attn_desc* d, const void* dO, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                                const void* V, int64_t v_stride, const void* O, const float* lse, int32_t T, const int32_t* row_start, void* dQ,
                                int64_t dq_stride, void* dK, int64_t dk_stride, void* dV, int64_t dv_stride, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (int e = check_self(d)) return e;
  if (int e = check_rows(d, T)) return e;
  if (T == 0 || d->n_seqs == 0) return PQ_OK;
  PQ_REQUIRE(dO && Q && K && V && O && lse && row_start && dQ && dK && dV && workspace, PQ_ERR_BAD_ARG, "NULL buffer");
  if (int e = check_stride("Q", q_stride, d->n_heads, d->d_head)) return e;
  if (int e = check_stride("K", k_stride, d->n_kv_heads, d->d_head)) return e;
  if (int e = check_stride("V", v_stride, d->n_kv_heads, d->d_head)) return e;
  if (int e = check_stride("dQ", dq_stride, d->n_heads, d->d_head)) return e;
  if (int e = check_stride("dK", dk_stride, d->n_kv_heads, d->d_head)) return e;
  if (int e = check_stride("dV", dv_stride, d->n_kv_heads, d->d_head)) return e;
  PQ_REQUIRE(at16(dO) && at16(Q) && at16(K) && at16(V) && at16(O) && at16(dQ) && at16(dK) && at16(dV) && at16(workspace), PQ_ERR_SHAPE,
             "buffers must be 16-byte aligned");
  // (fewer rows may want more pieces and more room for them: a workspace for more rows serves fewer with the pieces that it holds)
  const size_t least = stats_bytes(d, T) + 256;
  PQ_REQUIRE(workspace_bytes >= least, PQ_ERR_WORKSPACE, "workspace %zu < %zu", workspace_bytes, least);
  const int pieces = (int)std::max<size_t>(1, std::min<size_t>(token_pieces(d, T), (workspace_bytes - least) / part_bytes(d, T)));
  const int H = d->n_heads, Hk = d->n_kv_heads, dh = d->d_head;
  const pq_region written[] = {rows_region("dQ", dQ, T, dq_stride, H, dh), rows_region("dK", dK, T, dk_stride, Hk, dh), rows_region("dV", dV, T, dv_stride, Hk, dh),
                               pq_flat_region("workspace", workspace, (int64_t)(stats_bytes(d, T) + (pieces > 1 ? pieces * part_bytes(d, T) : 0)))};
  const pq_region read[] = {rows_region("dO", dO, T, (int64_t)H * dh, H, dh), rows_region("Q", Q, T, q_stride, H, dh), rows_region("K", K, T, k_stride, Hk, dh),
                            rows_region("V", V, T, v_stride, Hk, dh), rows_region("O", O, T, (int64_t)H * dh, H, dh),
                            pq_flat_region("lse", lse, (int64_t)T * H * 4), row_start_region(d, row_start)};
  if (int e = pq_refuse_overlap(written, 4, read, 7)) return e;
  self_args a = make_args(d, T, row_start);
  a.Q = (const uint16_t*)Q; a.K = (const uint16_t*)K; a.V = (const uint16_t*)V; a.O = (const uint16_t*)O; a.dO = (const uint16_t*)dO;
  a.qs = q_stride; a.ks = k_stride; a.vs = v_stride;
  a.dQ = (uint16_t*)dQ; a.dK = (uint16_t*)dK; a.dV = (uint16_t*)dV;
  a.dqs = dq_stride; a.dks = dk_stride; a.dvs = dv_stride;
  a.lse = const_cast<float*>(lse);
  a.stats = (float2*)workspace;
  a.parts = (float*)((char*)workspace + stats_bytes(d, T));
  a.pieces = pieces;
  hipStream_t s = (hipStream_t)stream;
  pq_prof_scope prof(PQP_SELF_ATTN_BWD, s);
  const bool direct = a.d % 8 == 0 && q_stride % 8 == 0 && k_stride % 8 == 0 && v_stride % 8 == 0;
  return direct ? launch_backward_d<true>(a, s) : launch_backward_d<false>(a, s);
}
