// qsl_residual.h -- kernels on a layer's residual stream: dropout whose mask is formed again wherever it is needed, the root-mean-square norm
// of residual + dropout(x), whole or in 8 bits with scales, and its gradient.
//
// Row n with totals h of C columns, r = (sum h^2 / C + eps)^(-1/2), u = r h:
//   y = w u                  dh = r (g - u mean_j(g_j u_j)) + what arrives at h from elsewhere, g = w dy           dw = sum over rows of dy u
//   drop(v)_i = v_i 65536 / T where the row's 16-bit random piece i is below T, else 0
// A row is read once and held in registers between its sums and its results: every array that a call has to read or write passes the
// memory once.  All of it is computed in 32 bits.
// Part of the translation unit residual.hip; not a public header.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "qsl_device.h"

using namespace qsl;

namespace {

__device__ __forceinline__ uint64_t block_number() { return static_cast<uint64_t>(blockIdx.y) * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------------------------------------
// units: N columns of a row, 16 bytes of the arrays' type E, eight 16-bit values or four floats: lanes side by side read 16 bytes side by side.  (Eight
// floats a lane in two loads: the norm of 6,000 fp32 rows of 785, without a residual, 9.7 us instead of 7.9.)  They begin at every N-th column of the row, wherever
// that lies: the loads need no more than the elements' alignment.  Weights and sums in floats beside 16-bit arrays have units of eight too.
// ---------------------------------------------------------------------------------------------
template <class E> constexpr int COLS = 16 / sizeof(E);
template <class W, int N> struct Unit { uint32_t w[N * sizeof(W) / 4]; };

template <int N> __device__ __forceinline__ void unpack(const Unit<float, N>& q, float* v) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __uint_as_float(q.w[i]);
}
__device__ __forceinline__ void unpack(const Unit<__bf16, 8>& q, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(q.w[i] << 16); v[2 * i + 1] = __uint_as_float(q.w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void unpack(const Unit<_Float16, 8>& q, float* v) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) { const h2 x = __builtin_bit_cast(h2, q.w[i]); v[2 * i] = static_cast<float>(x[0]); v[2 * i + 1] = static_cast<float>(x[1]); }
}
// rounded once, to nearest even
template <int N> __device__ __forceinline__ void pack(const float* v, Unit<float, N>& q) {
#pragma unroll
  for (int i = 0; i < N; ++i) q.w[i] = __float_as_uint(v[i]);
}
template <class W, class = typename std::enable_if<sizeof(W) == 2>::type> __device__ __forceinline__ void pack(const float* v, Unit<W, 8>& q) {
  typedef W w2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) { const w2 x = {static_cast<W>(v[2 * i]), static_cast<W>(v[2 * i + 1])}; q.w[i] = __builtin_bit_cast(uint32_t, x); }
}

// 16 bytes with the elements' alignment, and the parts of a unit that is short of columns; an element's bits
template <class W> struct Raw {
  typedef uint32_t mem __attribute__((ext_vector_type(4), aligned(2)));
  typedef uint32_t four __attribute__((ext_vector_type(2), aligned(2)));
  typedef uint32_t two __attribute__((aligned(2)));
  typedef uint16_t bits;
};
template <> struct Raw<float> {
  typedef uint32_t mem __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t four __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t two __attribute__((ext_vector_type(2), aligned(4)));
  typedef uint32_t bits;
};
// the first n < N of a unit's elements away, zeros behind the rest
template <class W, int N> __device__ __forceinline__ void shift_out(Unit<W, N>& q, uint32_t n) {
  constexpr int WORDS = N * sizeof(W) / 4;
  auto away = [&](int words) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) q.w[i] = i + words < WORDS ? q.w[i + words] : 0;
  };
  if (N == 8 && n & 4) away(WORDS / 2);
  if (n & 2) away(2 * sizeof(W) / 4);
  if (n & 1) {
    if constexpr (sizeof(W) == 4) away(1);
    else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) q.w[i] = __builtin_amdgcn_alignbit(i + 1 < WORDS ? q.w[i + 1] : 0, q.w[i], 16);
    }
  }
}
// PAST: what is written is all that the caches hold, or more, and what is read comes on top, so that little of it is found there by what runs next: it need
// not pass through them.  us for 16,384 rows of 4,096, through them / past them: the norm bf16 91 / 88, fp32 182 / 175, and bf16 with a reader of its results behind it
// 161 / 158 (of 8,192 rows, which the caches hold, 81 / 83); the gradient bf16 125.5 / 120, fp32 246 / 230; dropout with a residual fp32 135.5 / 128.
template <bool PAST, class M> __device__ __forceinline__ M load16(const M* p) {
  if constexpr (PAST) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool PAST, class M> __device__ __forceinline__ void store16(M* p, M m) {
  if constexpr (PAST) __builtin_nontemporal_store(m, p);
  else *p = m;
}
// U units of a row of `cols` columns, from column c0 on, `step` columns apart; zeros where there is no row (`live`) or none of it left.  A row's last
// unit, where it is short, is cut from the row's last N columns, so that its load is one with the others (by single elements: the gradient
// of 30,000 rows of 785 bf16 71 instead of 61 us): cut_units has to follow.  It waits for the values, so it follows when all
// arrays' loads are under way (else 2,047 rows of 12,289 70 instead of 64 us).  TINY: rows of less than N are taken by elements.
template <int U, bool TINY, bool PAST, class W, int N>
__device__ __forceinline__ void load_units(const W* row, uint32_t c0, uint32_t step, uint32_t cols, bool live, Unit<W, N>* q) {
  constexpr int WORDS = N * sizeof(W) / 4;
  const uint32_t end = live ? cols : 0;
  if (!TINY || cols >= N) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = c0 + u * step;
      const W* p = row + min(c, cols - N);
#pragma unroll
      for (int k = 0; k < WORDS / 4; ++k) {
        typename Raw<W>::mem m = {0, 0, 0, 0};
        if (c < end) m = load16<PAST>(reinterpret_cast<const typename Raw<W>::mem*>(p) + k);
#pragma unroll
        for (int i = 0; i < 4; ++i) q[u].w[4 * k + i] = m[i];
      }
    }
  } else {
    typedef typename Raw<W>::bits bits;
    const bits* p = reinterpret_cast<const bits*>(row);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) q[u].w[i] = 0;
    }
    if (c0 < end) {                                                         // (c0 = 0)
#pragma unroll
      for (uint32_t i = 0; i < N - 1; ++i) {
        const uint32_t x = i < cols ? static_cast<uint32_t>(p[i]) : 0u;
        if constexpr (sizeof(W) == 4) q[0].w[i] = x;
        else q[0].w[i / 2] |= x << 16 * (i & 1);
      }
    }
  }
}
template <int U, bool TINY, class W, int N> __device__ __forceinline__ void cut_units(uint32_t c0, uint32_t step, uint32_t cols, Unit<W, N>* q) {
  if ((cols & (N - 1)) == 0 || (TINY && cols < N)) return;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (c0 + u * step < cols && c0 + u * step + N > cols) shift_out(q[u], N - (cols & (N - 1)));      // (no row: zeros stay zeros)
}
// a unit's columns below `end`: cols, or 0 where there is no row
template <bool PAST, int N, class W> __device__ __forceinline__ void store_unit(W* row, uint32_t c, uint32_t end, const float* v) {
  Unit<W, N> q;
  pack(v, q);
  if (c + N <= end) {
#pragma unroll
    for (int k = 0; k < N * static_cast<int>(sizeof(W)) / 16; ++k) {
      typename Raw<W>::mem m = {q.w[4 * k], q.w[4 * k + 1], q.w[4 * k + 2], q.w[4 * k + 3]};
      store16<PAST>(reinterpret_cast<typename Raw<W>::mem*>(row + c) + k, m);
    }
  } else if (c < end) {                                                     // four, two, one
    uint32_t n = end - c;
    W* p = row + c;
    if (N == 8 && n & 4) {
      typename Raw<W>::four m;
      __builtin_memcpy(&m, q.w, sizeof(m));
      *reinterpret_cast<typename Raw<W>::four*>(p) = m;
      shift_out(q, 4);
      p += 4;
    }
    if (n & 2) {
      typename Raw<W>::two m;
      __builtin_memcpy(&m, q.w, sizeof(m));
      *reinterpret_cast<typename Raw<W>::two*>(p) = m;
      shift_out(q, 2);
      p += 2;
    }
    if (n & 1) *reinterpret_cast<typename Raw<W>::bits*>(p) = static_cast<typename Raw<W>::bits>(q.w[0]);
  }
}

// ---------------------------------------------------------------------------------------------
// which values are kept
// ---------------------------------------------------------------------------------------------
constexpr uint32_t DROP_STREAM = 2, KEEP_ALL = 65536;      // (streams 0 and 1: Rand_k, QSGD)
struct Drop {
  uint32_t T;                   // of 65,536; KEEP_ALL: nothing is dropped, nothing formed
  float factor;                 // 65536 / T
  uint32_t row0, seed_lo, seed_hi;
  uint64_t round;
  const uint64_t* round_at;
};
struct Key { uint32_t lo, hi; };
__device__ __forceinline__ Key key_of(const Drop& d) {
  uint64_t r = d.round;
  if (d.T != KEEP_ALL && d.round_at) r += *d.round_at;
  return Key{static_cast<uint32_t>(r), (static_cast<uint32_t>(r >> 32) & 0x3FFFFFFFu) | DROP_STREAM << 30};
}
// philox4x32_10 with its exclusive-ors in one instruction of three operands each (two: dropout of 65,536 rows of 4,096 bf16 182 us instead of 175.5, what
// it takes without a mask)
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ Words4 random_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c0, p1 = static_cast<uint64_t>(0xCD9E8D57u) * c2;
    c0 = xor3(static_cast<uint32_t>(p1 >> 32), c1, k0); c1 = static_cast<uint32_t>(p1);
    c2 = xor3(static_cast<uint32_t>(p0 >> 32), c3, k1); c3 = static_cast<uint32_t>(p0);
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return Words4{{c0, c1, c2, c3}};
}
// v <- drop(v) of a row's unit: 16-bit pieces of the Philox block of its eight columns, of which a unit of four takes its half.  (A word of 32 bits for
// each: those 175.5 us become 200.  The share that is kept is a multiple of 2^-16, and the factor belongs to that share, so that what is kept has the
// right mean.)
template <int N> __device__ __forceinline__ void drop_unit(const Drop& d, const Key& k, uint32_t row, uint32_t unit, float* v) {
  Words4 o = random_words(N == 8 ? unit : unit / 2, d.row0 + row, k.lo, k.hi, d.seed_lo, d.seed_hi);
  if (N == 4 && unit & 1) { o.w[0] = o.w[2]; o.w[1] = o.w[3]; }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t piece = i & 1 ? o.w[i / 2] >> 16 : o.w[i / 2] & 0xFFFFu;
    v[i] = piece < d.T ? v[i] * d.factor : 0.0f;
  }
}

// ---------------------------------------------------------------------------------------------
// sums and maxima over the L lanes that hold a row (16, 64, or a block), the same bits in each of them
// ---------------------------------------------------------------------------------------------
constexpr int DPP_ROW_ROR = 0x120, DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141;      // quad_perm [1,0,3,2], [2,3,0,1]
template <int CTRL> __device__ __forceinline__ uint32_t dpp_move(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xF, 0xF, false));
}
template <int CTRL> __device__ __forceinline__ float dpp_move(float x) { return __uint_as_float(dpp_move<CTRL>(__float_as_uint(x))); }
// Rotations by 8, 4, 2, 1: both lanes of a pair add the same two numbers, so all sixteen end with the same bits.
__device__ __forceinline__ float sum16(float x) {
  x += dpp_move<DPP_ROW_ROR + 8>(x);
  x += dpp_move<DPP_ROW_ROR + 4>(x);
  x += dpp_move<DPP_ROW_ROR + 2>(x);
  return x + dpp_move<DPP_ROW_ROR + 1>(x);
}
__device__ __forceinline__ float lane_float(float x, int lane) { return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(x)), lane))); }
__device__ __forceinline__ float wave_total(float x) {
  x = sum16(x);
  return (lane_float(x, 0) + lane_float(x, 16)) + (lane_float(x, 32) + lane_float(x, 48));
}
// The W waves' values of a row, joined by every W neighbouring lanes: each pair of lanes adds the same two numbers.  (Every thread reading all W:
// the gradient of 16,384 rows of 4,096 bf16 130.5 us instead of 128.9, of 30,000 of 785 55.9 / 55.4.)
template <int W> __device__ __forceinline__ float join_sum(float x) {
  if constexpr (W >= 2) x += dpp_move<DPP_XOR1>(x);
  if constexpr (W >= 4) x += dpp_move<DPP_XOR2>(x);
  if constexpr (W >= 8) x += dpp_move<DPP_HALF_MIRROR>(x);
  if constexpr (W >= 16) x += dpp_move<DPP_ROW_ROR + 8>(x);
  return x;
}
// `at`: places in LDS for the row's waves that no thread still reads from an earlier call
template <int L> __device__ __forceinline__ float row_sum(float x, float* at) {
  if constexpr (L == 16) return sum16(x);
  x = wave_total(x);
  if constexpr (L <= 64) return x;
  if (lane_id() == 0) at[threadIdx.x / WAVE] = x;
  __syncthreads();
  return join_sum<L / 64>(at[threadIdx.x % (L / 64)]);
}
// two sums at once
struct Two { float a, b; };
template <int L> __device__ __forceinline__ Two row_sums(Two x, Two* at) {
  if constexpr (L == 16) return Two{sum16(x.a), sum16(x.b)};
  x = Two{wave_total(x.a), wave_total(x.b)};
  if constexpr (L <= 64) return x;
  if (lane_id() == 0) at[threadIdx.x / WAVE] = x;
  __syncthreads();
  x = at[threadIdx.x % (L / 64)];
  return Two{join_sum<L / 64>(x.a), join_sum<L / 64>(x.b)};
}
// over 4, 8, 16 or 32 neighbouring lanes
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t x, uint32_t lanes) {
  x = max(x, dpp_move<DPP_XOR1>(x));
  x = max(x, dpp_move<DPP_XOR2>(x));
  if (lanes >= 8) x = max(x, dpp_move<DPP_HALF_MIRROR>(x));
  if (lanes >= 16) x = max(x, dpp_move<DPP_ROW_ROR + 8>(x));
  if (lanes >= 32) x = max(x, static_cast<uint32_t>(__builtin_amdgcn_ds_swizzle(static_cast<int>(x), 0x401F)));      // from lane ^ 16
  return x;
}
template <int L> __device__ __forceinline__ uint32_t row_max(uint32_t x, uint32_t* at) {
  x = max_of_lanes(x, 16);
  if constexpr (L == 16) return x;
  x = max(max(lane_value(x, 0), lane_value(x, 16)), max(lane_value(x, 32), lane_value(x, 48)));
  if constexpr (L <= 64) return x;
  if (lane_id() == 0) at[threadIdx.x / WAVE] = x;
  __syncthreads();
  constexpr int W = L / 64;
  x = at[threadIdx.x % W];
  if constexpr (W >= 2) x = max(x, dpp_move<DPP_XOR1>(x));
  if constexpr (W >= 4) x = max(x, dpp_move<DPP_XOR2>(x));
  if constexpr (W >= 8) x = max(x, dpp_move<DPP_HALF_MIRROR>(x));
  if constexpr (W >= 16) x = max(x, dpp_move<DPP_ROW_ROR + 8>(x));
  return x;
}

// Squares of totals from 2^64 on do not fit into a float: such rows are taken times this, eps times its square.  (2^56 squared times QSL_NORM_COLS_MAX fits.  Of
// a usual eps nothing is left, but 2^100 counts beside a mean of 2^113, from where on a sum over QSL_NORM_COLS_MAX columns may not fit.)
constexpr float SMALLER = 0x1p-72f;
// Totals below 2^64, or taken times that, times gradients below 2^128 divided by this fit, and their sums.  (What is lost below 2^-149 is nothing beside the
// sum of sizes, 2^-40 and more where the products themselves do not fit.)
constexpr float LARGER = 0x1p96f;
constexpr float INF = __builtin_inff();

template <int L> constexpr int THREADS = L <= 64 ? 256 : L;      // rows of a wave and less share a block
template <int L> constexpr bool TINY = L == 16;                  // rows of less than a unit's columns go there
template <int L> constexpr int WAVES = L <= 64 ? 1 : L / 64;     // of a row
// a row's number within the block, for the compiler the same in a wave where it is
template <int L> __device__ __forceinline__ uint32_t row_in_block() {
  if constexpr (L > 64) return 0;
  else if constexpr (L == 64) return __builtin_amdgcn_readfirstlane(threadIdx.x / L);
  else return threadIdx.x / L;
}

// ---------------------------------------------------------------------------------------------
// dropout by itself
// ---------------------------------------------------------------------------------------------
struct DropArgs {
  const void *x, *res;
  void* y;
  uint64_t x_stride, res_stride, y_stride, rows;
  uint32_t cols, units;          // units of a row
  Drop drop;
};
constexpr int DROP_THREADS = 256;

// Read and written once each, bound by memory: 8,192 rows of 4,096 bf16 with a residual 37.6 us, 5.35 TB/s (a copy of 1 GiB: 5.2).
// A unit a thread, the rows' units one behind the other: the shortest way from a load to a store, eight waves on a
// SIMD unit.  (Four a thread, whose loads are under way together: 8,192 rows of 4,096 bf16 28.7 us instead of 25.3, 4,095 of 11,009 40.9 / 34.2; eight 30.5.)
template <class E, bool PAST> __global__ __launch_bounds__(DROP_THREADS) void k_dropout(DropArgs a) {
  const uint64_t first = block_number() * DROP_THREADS, row_b = first / a.units;
  const uint32_t i = static_cast<uint32_t>(first - row_b * a.units) + threadIdx.x, r = i / a.units;
  const uint64_t row = row_b + r;
  constexpr int N = COLS<E>;
  const uint32_t unit = i - r * a.units, c = unit * N;
  if (row >= a.rows) return;
  Unit<E, N> x, res;
  load_units<1, true, PAST>(static_cast<const E*>(a.x) + row * a.x_stride, c, 0, a.cols, true, &x);
  if (a.res) load_units<1, true, PAST>(static_cast<const E*>(a.res) + row * a.res_stride, c, 0, a.cols, true, &res);
  cut_units<1, true>(c, 0, a.cols, &x);
  float v[N];
  unpack(x, v);
  if (a.drop.T != KEEP_ALL) drop_unit<N>(a.drop, key_of(a.drop), static_cast<uint32_t>(row), unit, v);
  if (a.res) {
    float b[N];
    cut_units<1, true>(c, 0, a.cols, &res);
    unpack(res, b);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += b[k];
  }
  store_unit<PAST, N>(static_cast<E*>(a.y) + row * a.y_stride, c, a.cols, v);
}

// ---------------------------------------------------------------------------------------------
// the norm
// ---------------------------------------------------------------------------------------------
struct NormArgs {
  const void *x, *res, *weight;
  void *total, *y;
  float* scales;
  uint64_t x_stride, res_stride, total_stride, y_stride, rows;
  uint32_t cols, weight_is_float, is_e4m3, group_bits;      // 2^group_bits columns have a scale, 0: the row
  float eps;
  Drop drop;
};

template <class E, int U, bool TINY> __device__ __forceinline__ void load_weight(const void* weight, uint32_t is_float, uint32_t c0, uint32_t step, uint32_t cols, float* w) {
  constexpr int N = COLS<E>;
  auto load = [&](auto* at) {
    Unit<typename std::remove_const<typename std::remove_reference<decltype(*at)>::type>::type, N> q[U];
    load_units<U, TINY, false>(at, c0, step, cols, true, q);
    cut_units<U, TINY>(c0, step, cols, q);
#pragma unroll
    for (int u = 0; u < U; ++u) unpack(q[u], w + N * u);
  };
  if (!weight) {
#pragma unroll
    for (int i = 0; i < N * U; ++i) w[i] = 1.0f;
  } else if (sizeof(E) == 4 || is_float) {
    load(static_cast<const float*>(weight));
  } else {
    load(static_cast<const E*>(weight));
  }
}
// 8-bit codes of a unit, N bytes.  y = m t with t = w (h 2^e), r = m 2^e, 1 <= m < 2, and the product's rounding error t_lo: that power of two is exact, and
// t fits where y does, large weights and small ones; `most`: the bits of the group's largest |t|.  y Q / a =
// t Q / max |t|: m does not enter, and with the errors of t and of the quotient the code is that of the exact value for all that h allows.  (Of 24.6 million
// e4m3 codes of rows of 4,096 with a residual 48 are not those of 64 bits, by elementary operations in 32 bits 67; fp32 8 and 16.)
template <int N> __device__ __forceinline__ void store_codes(uint8_t* row, uint32_t c, uint32_t cols, const float* t, const float* t_lo, uint32_t most, float m, bool is_e4m3,
                                            float* scale_at) {
  const float Q = is_e4m3 ? 448.0f : 127.0f, t_max = __uint_as_float(most), y_max = t_max * m, a = fmaxf(y_max, 0x1p-100f);
  const bool bad = !(y_max < INF);                    // an infinity or a NaN
  const bool plain = !(y_max >= 0x1p-100f);           // next to nothing: by y itself, |y| Q / a <= Q
  const float div = plain ? a : t_max, q = Q / div, inv = plain ? q * m : q, lo_inv = plain ? 0.0f : q, inv_lo = __builtin_fmaf(-q, div, Q) * (lo_inv / Q);
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __builtin_fmaf(t[i], inv, __builtin_fmaf(t[i], inv_lo, t_lo[i] * lo_inv));
  uint32_t code[N / 4];
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    const float* f = v + 4 * k;
    uint32_t x = 0;
    if (is_e4m3) {
      x = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], x, false);
      x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], x, true);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x |= (static_cast<uint32_t>(static_cast<int>(rintf(f[i]))) & 0xFFu) << 8 * i;
    }
    code[k] = bad ? 0 : x;
  }
  if (scale_at) *scale_at = bad ? __builtin_nanf("") : a / Q;
  typedef uint32_t eight __attribute__((ext_vector_type(2), aligned(1)));
  typedef uint32_t four __attribute__((aligned(1)));
  typedef uint16_t two __attribute__((aligned(1)));
  uint8_t* p = row + c;
  if (c + N <= cols) {
    if constexpr (N == 8) { const eight q = {code[0], code[1]}; *reinterpret_cast<eight*>(p) = q; }
    else *reinterpret_cast<four*>(p) = code[0];
  } else {
    const uint32_t n = cols - c;
    uint32_t x = code[0];
    if (N == 8 && n & 4) { *reinterpret_cast<four*>(p) = x; x = code[N / 4 - 1]; p += 4; }
    if (n & 2) { *reinterpret_cast<two*>(p) = static_cast<uint16_t>(x); x >>= 16; p += 2; }
    if (n & 1) *p = static_cast<uint8_t>(x);
  }
}

// A row by L lanes with U units each: loads of all arrays, the totals and their squares, one sum over the lanes, results from registers.  Bound by
// memory: 16,384 rows of 4,096 bf16 (x, residual, total, y) with a mask 87 us, 6.2 TB/s; 8,192 rows of 8,192 to e4m3 83.5 us, 5.65 TB/s; a row by itself
// 2.4 us, the way from its loads over one barrier to its stores.
template <class E, int L, int U, bool BITS8, bool PAST>
__global__ __launch_bounds__(THREADS<L>) void k_rms_norm(NormArgs a) {
  __shared__ float sums[2][WAVES<L>];
  __shared__ uint32_t maxima[WAVES<L>];
  constexpr int N = COLS<E>;
  constexpr bool LATE_WEIGHT = L * U * N > 16384;      // (the registers do not hold them beside the rest)
  const uint64_t row = block_number() * (THREADS<L> / L) + row_in_block<L>();
  const uint32_t lane = threadIdx.x % L, c0 = lane * N, end = row < a.rows ? a.cols : 0;
  Unit<E, N> x[U], res[U];
  load_units<U, TINY<L>, PAST>(static_cast<const E*>(a.x) + row * a.x_stride, c0, L * N, a.cols, end != 0, x);
  if (a.res) load_units<U, TINY<L>, PAST>(static_cast<const E*>(a.res) + row * a.res_stride, c0, L * N, a.cols, end != 0, res);
  float h[N * U], w[N * U];
  if constexpr (!LATE_WEIGHT) load_weight<E, U, TINY<L>>(a.weight, a.weight_is_float, c0, L * N, a.cols, w);
  const Key key = key_of(a.drop);
  cut_units<U, TINY<L>>(c0, L * N, a.cols, x);
  if (a.res) cut_units<U, TINY<L>>(c0, L * N, a.cols, res);
  float ss = 0.0f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float* v = h + N * u;
    unpack(x[u], v);
    if (a.drop.T != KEEP_ALL) drop_unit<N>(a.drop, key, static_cast<uint32_t>(row), u * L + lane, v);
    if (a.res) {
      float b[N];
      unpack(res[u], b);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += b[i];
    }
    if (a.total) store_unit<PAST, N>(static_cast<E*>(a.total) + row * a.total_stride, c0 + u * L * N, end, v);
#pragma unroll
    for (int i = 0; i < N; ++i) ss = __builtin_fmaf(v[i], v[i], ss);
  }
  ss = row_sum<L>(ss, sums[0]);
  float f = 1.0f;
  if (__any(ss == INF)) {      // (the same answer in all waves of a row)
    f = ss == INF ? SMALLER : 1.0f;
    ss = 0.0f;
#pragma unroll
    for (int i = 0; i < N * U; ++i) { h[i] *= f; ss = __builtin_fmaf(h[i], h[i], ss); }
    ss = row_sum<L>(ss, sums[1]);
  }
  const float r = 1.0f / sqrtf(ss / static_cast<float>(a.cols) + a.eps * f * f);
  const float two_e = __uint_as_float(__float_as_uint(r) & 0x7F800000u), m = __uint_as_float((__float_as_uint(r) & 0x007FFFFFu) | 0x3F800000u);      // (r NaN: 2^e infinite)
  float lo[BITS8 ? N * U : 1];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if constexpr (LATE_WEIGHT) load_weight<E, 1, false>(a.weight, a.weight_is_float, c0 + u * L * N, 0, a.cols, w + N * u);
#pragma unroll
    for (int k = N * u; k < N * u + N; ++k) {
      if constexpr (BITS8) {
        const float x2 = h[k] * two_e, t = x2 * w[k];
        lo[k] = __builtin_fmaf(x2, w[k], -t);
        h[k] = t;
      } else {
        h[k] = h[k] * r * w[k];
      }
    }
  }
  if constexpr (!BITS8) {
#pragma unroll
    for (int u = 0; u < U; ++u) store_unit<PAST, N>(static_cast<E*>(a.y) + row * a.y_stride, c0 + u * L * N, end, h + N * u);
  } else {
    uint32_t most[U], all = 0;      // of the bits of |t|: a NaN is above the infinities; 0 behind the row
#pragma unroll
    for (int u = 0; u < U; ++u) {
      most[u] = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) most[u] = max(most[u], __float_as_uint(h[N * u + i]) & 0x7FFFFFFFu);
      if (a.group_bits) most[u] = max_of_lanes(most[u], (1u << a.group_bits) / N);
      all = max(all, most[u]);
    }
    if (!a.group_bits) all = row_max<L>(all, maxima);
    const uint32_t in_group = (1u << a.group_bits) - 1, of_row = a.group_bits ? (a.cols + in_group) >> a.group_bits : 1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t c = c0 + u * L * N;
      float* const scale_at = a.scales + row * of_row + (a.group_bits ? c >> a.group_bits : 0);
      if (c < end) store_codes<N>(static_cast<uint8_t*>(a.y) + row * a.y_stride, c, end, h + N * u, lo + N * u, a.group_bits ? most[u] : all, m, a.is_e4m3,
                                  (a.group_bits ? (c & in_group) == 0 : c == 0) ? scale_at : nullptr);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// its gradient
// ---------------------------------------------------------------------------------------------
struct BackArgs {
  const void *total, *dy, *dtotal, *weight;
  void *dres, *dx;
  float* part;                   // [blocks, cols]: every block's sum of dy u over its rows (dweight itself, if there is one block); or nullptr
  uint64_t total_stride, dy_stride, dtotal_stride, dres_stride, dx_stride, rows;
  uint32_t cols, weight_is_float;
  float eps;
  Drop drop;
};

// Both sums over a row at once, then the results from registers.  Bound by memory: 16,384 rows of 4,096 bf16 with a mask (five arrays) 112 us, 6.0 TB/s, and
// 4.5 for k_sum_parts; rows of more than 8,192 columns, a block to a compute unit, by the way from loads to stores that little else runs beside
// (2,047 rows of 12,289 fp16, four arrays, 44.5 us, 4.5 TB/s, and 5.3).
// A block goes through rows that lie a grid apart and keeps its sum for dw in registers.  A unit's registers take the next row's as soon as this row's is
// unpacked for its results, so that these loads are under way beside the masks and the stores and few waves are enough (us, bf16, loads at a row's
// beginning / ahead: 16,384 rows of 4,096 128.8 / 120.7, of 2,048 70 / 65, 2,047 rows of 12,288 58.8 / 56.3).
// Where 1024 threads leave a thread 128 registers, the weights are held in LDS, every thread's own; where that is not enough (TIGHT), nothing is loaded
// ahead, and what else arrives at the totals is loaded where it is added (fp32, 2,047 rows of 12,288: 104 us, with loads ahead 127).
// There too the compiler is kept from holding what it can form again: offsets and the first rounds of the masks, which depend on the lane alone, and unpacked
// 16-bit values (4,096 rows of 32,768 bf16 456 us without, 333 without the last, 272; 2,048 of fp32 368 / 275).  Rows of more than 16,384 columns still have 12
// (fp32), 20 (bf16) and 32 bytes (fp16) of a lane's registers in memory: 2,048 of 32,768 fp32 260 us (floor 258), bf16 145 (129).
template <class E, int L, int U> constexpr bool WEIGHT_IN_LDS = L * U * COLS<E> >= 16384;
template <int L, int U> constexpr bool TIGHT_ROW = L * U >= 4096;
template <class E, int L, int U, bool PAST>
__global__ __launch_bounds__(THREADS<L>) void k_rms_norm_backward(BackArgs a) {
  constexpr int ROWS = THREADS<L> / L;
  constexpr int N = COLS<E>;
  constexpr bool LDS = WEIGHT_IN_LDS<E, L, U>, TIGHT = TIGHT_ROW<L, U>;
  typedef float quad __attribute__((ext_vector_type(4)));
  __shared__ quad weights[LDS ? N / 4 * U : 1][LDS ? L : 1];
  __shared__ Two sums[2][2][WAVES<L>];
  __shared__ float joined[ROWS > 1 ? ROWS * N * U * L : 1];
  uint32_t lane = threadIdx.x % L, c0 = lane * N;
  const Key key = key_of(a.drop);
  float w_all[LDS ? N : N * U], dw[N * U];
  if constexpr (LDS) {
    for (int u = 0; u < U; ++u) {
      load_weight<E, 1, false>(a.weight, a.weight_is_float, c0 + u * L * N, 0, a.cols, w_all);
#pragma unroll
      for (int k = 0; k < N / 4; ++k) weights[N / 4 * u + k][lane] = quad{w_all[4 * k], w_all[4 * k + 1], w_all[4 * k + 2], w_all[4 * k + 3]};
    }
  } else {
    load_weight<E, U, TINY<L>>(a.weight, a.weight_is_float, c0, L * N, a.cols, w_all);
  }
  // what is formed of the lane's number is formed again behind this, not held in registers from row to row
  auto lane_again = [&]() {
    if constexpr (TIGHT) {
      asm volatile("" : "+v"(lane));
      c0 = lane * N;
    }
  };
  auto weight_of = [&](int u, float* w) {
    if constexpr (LDS) {
#pragma unroll
      for (int k = 0; k < N / 4; ++k) {
        const quad q = weights[N / 4 * u + k][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * k + i] = q[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = w_all[N * u + i];
    }
  };
#pragma unroll
  for (int i = 0; i < N * U; ++i) dw[i] = 0.0f;
  Unit<E, N> hq[U], dyq[U], dtq[TIGHT ? 1 : U];
  auto load_unit = [&](uint64_t row, int u) {
    const uint32_t c = c0 + u * L * N;
    const bool live = row < a.rows;
    load_units<1, TINY<L>, PAST>(static_cast<const E*>(a.total) + row * a.total_stride, c, 0, a.cols, live, hq + u);
    load_units<1, TINY<L>, PAST>(static_cast<const E*>(a.dy) + row * a.dy_stride, c, 0, a.cols, live, dyq + u);
    if constexpr (!TIGHT)
      if (a.dtotal) load_units<1, TINY<L>, PAST>(static_cast<const E*>(a.dtotal) + row * a.dtotal_stride, c, 0, a.cols, live, dtq + u);
  };
  const uint64_t step = static_cast<uint64_t>(gridDim.x) * ROWS;
  uint64_t row = static_cast<uint64_t>(blockIdx.x) * ROWS + row_in_block<L>();
  if constexpr (!TIGHT) {
#pragma unroll
    for (int u = 0; u < U; ++u) load_unit(row, u);
  }
  uint32_t turn = 0;             // a row's sums go where those before last stood: there is a barrier between reading these and writing them
  for (uint64_t base = static_cast<uint64_t>(blockIdx.x) * ROWS; base < a.rows; base += step, row += step) {
    const uint32_t end = row < a.rows ? a.cols : 0;
    lane_again();
    if constexpr (TIGHT) {
#pragma unroll
      for (int u = 0; u < U; ++u) load_unit(row, u);
    }
    cut_units<U, TINY<L>>(c0, L * N, a.cols, hq);
    cut_units<U, TINY<L>>(c0, L * N, a.cols, dyq);
    if constexpr (!TIGHT)
      if (a.dtotal) cut_units<U, TINY<L>>(c0, L * N, a.cols, dtq);
    auto sum = [&](auto&& g_of) {
      Two s = {0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float h[N], d[N], w[N];
        unpack(hq[u], h);
        unpack(dyq[u], d);
        weight_of(u, w);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          s.a = __builtin_fmaf(h[i], h[i], s.a);
          s.b = __builtin_fmaf(g_of(d[i] * w[i]), h[i], s.b);
        }
        if constexpr (TIGHT && sizeof(E) == 2) {      // (unpacked again for the results)
#pragma unroll
          for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(hq[u].w[i]), "+v"(dyq[u].w[i]));
        }
      }
      return s;
    };
    Two s = row_sums<L>(sum([](float g) { return g; }), sums[turn][0]);
    float f = 1.0f, up = 1.0f;
    if (__any(!(s.a + fabsf(s.b) < INF))) {
      if (s.a == INF) {      // the totals times f, in their type: what that rounds is nothing beside the row's largest
        f = SMALLER;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float h[N];
          unpack(hq[u], h);
#pragma unroll
          for (int i = 0; i < N; ++i) h[i] *= f;
          pack(h, hq[u]);
        }
      }
      if (!(fabsf(s.b) < INF)) up = LARGER;
      s = row_sums<L>(sum([down = up == 1.0f ? 1.0f : 1.0f / LARGER](float g) { return g * down; }), sums[turn][1]);
    }
    turn ^= 1;
    const float r = 1.0f / sqrtf(s.a / static_cast<float>(a.cols) + a.eps * f * f);
    const float mean = s.b * r / static_cast<float>(a.cols) * up, rf = r * f;
    lane_again();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float h[N], d[N], t[N], w[N];
      unpack(hq[u], h);
      unpack(dyq[u], d);
      weight_of(u, w);
      if (a.dtotal) {
        if constexpr (TIGHT) {
          load_units<1, false, PAST>(static_cast<const E*>(a.dtotal) + row * a.dtotal_stride, c0 + u * L * N, 0, a.cols, end != 0, dtq);
          cut_units<1, false>(c0 + u * L * N, 0, a.cols, dtq);
        }
        unpack(dtq[TIGHT ? 0 : u], t);
      }
      if constexpr (!TIGHT) load_unit(row + step, u);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float un = h[i] * r;
        dw[N * u + i] = __builtin_fmaf(d[i], un, dw[N * u + i]);
        d[i] = rf * (d[i] * w[i] - un * mean);
        if (a.dtotal) d[i] += t[i];
      }
      if (a.dres) store_unit<PAST, N>(static_cast<E*>(a.dres) + row * a.dres_stride, c0 + u * L * N, end, d);
      if (a.dx) {
        if (a.drop.T != KEEP_ALL) drop_unit<N>(a.drop, key, static_cast<uint32_t>(row), u * L + lane, d);
        store_unit<PAST, N>(static_cast<E*>(a.dx) + row * a.dx_stride, c0 + u * L * N, end, d);
      }
    }
  }
  if (!a.part) return;
  float* out = a.part + static_cast<uint64_t>(blockIdx.x) * a.cols;
  if constexpr (ROWS == 1) {
#pragma unroll
    for (int u = 0; u < U; ++u) store_unit<false, N>(out, c0 + u * L * N, a.cols, dw + N * u);
  } else {
    const uint32_t mine = row_in_block<L>();
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) joined[mine * (N * U * L) + c0 + u * L * N + i] = dw[N * u + i];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.cols; c += THREADS<L>) {
      float s = joined[c];
#pragma unroll
      for (int k = 1; k < ROWS; ++k) s += joined[k * (N * U * L) + c];
      out[c] = s;
    }
  }
}

// dw: every PARTS-th of the blocks' sums in turn, then the sums of these, always in the same order.  Eight loads of a thread are under way at once.
template <uint32_t COLS, uint32_t PARTS>
__global__ __launch_bounds__(COLS * PARTS) void k_sum_parts(const float* part, uint32_t blocks, uint32_t cols, float* dweight) {
  __shared__ float at[PARTS][COLS + 1];
  const uint32_t x = threadIdx.x % COLS, y = threadIdx.x / COLS, c = blockIdx.x * COLS + x;
  float s = 0.0f;
  for (uint32_t b = y; b < blocks; b += 8 * PARTS) {
    float v[8];
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
      const uint32_t n = b + k * PARTS;
      v[k] = c < cols && n < blocks ? part[static_cast<uint64_t>(n) * cols + c] : 0.0f;
    }
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) s += v[k];
  }
  at[y][x] = s;
  __syncthreads();
  // the sums of a column: by sixteen lanes
  if (threadIdx.x < 16 * COLS) {
    const uint32_t l = threadIdx.x % 16, col = threadIdx.x / 16;
    s = at[l][col];
#pragma unroll
    for (uint32_t k = 16; k < PARTS; k += 16) s += at[l + k][col];
    s = sum16(s);
    if (l == 0 && blockIdx.x * COLS + col < cols) dweight[blockIdx.x * COLS + col] = s;
  }
}

}  // namespace
