// qsl_logits.h -- kernels on the rows of a model's logits: log probabilities of given tokens with the entropy and the top
// alternatives, their gradient, and the loss against a teacher's top logits with its gradient.
//
// Row n with logits z, factor c (`scale`), natural logarithms; m = max z, s = sum exp(c (z_i - m)), L = ln s:
//   logp_i = c (z_i - m) - L        p_i = exp(logp_i)        lse = c m + L        H = -sum p_i logp_i
//   d logp_t / dz_i = c ([i = t] - p_i)                      dH / dz_i = -c p_i (logp_i + H)
// A thread keeps (m, s, w) of the values that it has met, w = sum e_i y_i with y_i = c log2(e) (z_i - m), e_i = exp2(y_i): when m
// grows by a step, y falls by delta = c log2(e) (m_old - m_new), hence s <- s 2^delta, w <- (w + s delta) 2^delta; H = L - ln 2 w / s.
// All of it is held in 32 bits.  m starts at the lowest finite float, so a value of -inf has e = 0 and a row of them s = 0.
// Part of the translation unit logits.hip; not a public header.  (It stands in a folder of its own beside the compression kernels'.)
#pragma once

#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "qsl_device.h"

using namespace qsl;

namespace {

constexpr float LOWEST = -FLT_MAX, LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;
constexpr float Y_MIN = -1e4f;             // exp2 of this is 0; keeps 0 * -inf out of w
// Blocks are numbered over a grid of two dimensions, whose last row may be short of work.  (A loop over rows in the kernel would have its
// offsets held in registers from row to row: 127 VGPRs instead of 93 to 95 for 16 vectors of 16-bit values.)
__device__ __forceinline__ uint64_t block_number() { return static_cast<uint64_t>(blockIdx.y) * gridDim.x + blockIdx.x; }

constexpr uint32_t TOP_MAX = 128;          // alternatives of a row at most
constexpr uint32_t TEACHER_MAX = 256;      // entries of a teacher's row at most
constexpr uint32_t CAND_CAP = 512;         // candidates for the alternatives that are ranked at once
constexpr uint32_t REFINE = 256;           // ... of which so many give the next bound when there are more
// K alternatives of a row of few vectors: almost every vector's largest value is above the K-th largest of them, if there are K
constexpr __host__ __device__ bool maxima_say_little(uint64_t K, uint64_t nvec) { return K > nvec - nvec / 8; }
constexpr uint32_t GROUPS = 256;           // maxima of groups of threads that the threshold is taken from, at most
constexpr uint32_t HASH_SIZE = 4 * TEACHER_MAX;   // slots in which a teacher's entries are looked up, at most
constexpr uint32_t MASK_SPAN = 1u << 18;   // classes whose membership in the teacher's entries is held in LDS at once (32 KB)

// ---------------------------------------------------------------------------------------------
// elements: 16 bytes at a time, aligned to 4 bytes where reading (a row of 16-bit values may start between two words: its first value
// is then taken by itself; read at odd places, 4,096 rows of 128,001 take 211 us instead of 171), to the element where writing
// ---------------------------------------------------------------------------------------------
typedef uint32_t raw_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t raw_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t raw4 __attribute__((ext_vector_type(4)));

template <class E> struct Elem;
template <> struct Elem<float> {
  static constexpr int N = 4;
  typedef uint32_t bits;
  static __device__ __forceinline__ float from_bits(uint32_t b) { return __uint_as_float(b); }
  static constexpr uint32_t MINUS_INF = 0xFF800000u;
  typedef raw_a4 mem;
  static __device__ __forceinline__ void unpack(raw4 r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ float of_word(uint32_t x, uint32_t q) { (void)q; return __uint_as_float(x); }      // value q from its word
  static __device__ __forceinline__ void erase(raw4& r, uint32_t bits) {      // -inf where a bit is set
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = bits >> i & 1 ? MINUS_INF : r[i];
  }
  static __device__ __forceinline__ raw4 pack(const float* v) {
    raw4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
    return r;
  }
};
template <> struct Elem<__bf16> {
  static constexpr int N = 8;
  typedef uint16_t bits;
  static __device__ __forceinline__ float from_bits(uint32_t b) { return __uint_as_float(b << 16); }
  static constexpr uint32_t MINUS_INF = 0xFF80FF80u;
  typedef raw_a2 mem;
  static __device__ __forceinline__ void unpack(raw4 r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r[i] << 16); v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ float of_word(uint32_t x, uint32_t q) { (void)q; return __uint_as_float(q & 1 ? x & 0xFFFF0000u : x << 16); }      // value q from its word
  static __device__ __forceinline__ void erase(raw4& r, uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = (bits >> 2 * i & 1 ? 0x0000FFFFu : 0u) | (bits >> 2 * i & 2 ? 0xFFFF0000u : 0u);
      r[i] = (r[i] & ~m) | (MINUS_INF & m);
    }
  }
  static __device__ __forceinline__ raw4 pack(const float* v) {      // rounded once, to nearest even
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    raw4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) { b2 x = {static_cast<__bf16>(v[2 * i]), static_cast<__bf16>(v[2 * i + 1])}; r[i] = __builtin_bit_cast(uint32_t, x); }
    return r;
  }
};
template <> struct Elem<_Float16> {
  static constexpr int N = 8;
  typedef uint16_t bits;
  static __device__ __forceinline__ float from_bits(uint32_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(b))); }
  static constexpr uint32_t MINUS_INF = 0xFC00FC00u;
  typedef raw_a2 mem;
  static __device__ __forceinline__ void unpack(raw4 r, float* v) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) { const h2 x = __builtin_bit_cast(h2, static_cast<uint32_t>(r[i])); v[2 * i] = static_cast<float>(x[0]); v[2 * i + 1] = static_cast<float>(x[1]); }
  }
  static __device__ __forceinline__ float of_word(uint32_t x, uint32_t q) { (void)q; return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(q & 1 ? x >> 16 : x))); }      // value q from its word
  static __device__ __forceinline__ void erase(raw4& r, uint32_t bits) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = (bits >> 2 * i & 1 ? 0x0000FFFFu : 0u) | (bits >> 2 * i & 2 ? 0xFFFF0000u : 0u);
      r[i] = (r[i] & ~m) | (MINUS_INF & m);
    }
  }
  static __device__ __forceinline__ raw4 pack(const float* v) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    raw4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) { h2 x = {static_cast<_Float16>(v[2 * i]), static_cast<_Float16>(v[2 * i + 1])}; r[i] = __builtin_bit_cast(uint32_t, x); }
    return r;
  }
};

// values before the first whole word
template <class E> __device__ __forceinline__ uint32_t odd_ones(const E* z) { return sizeof(E) == 2 && (reinterpret_cast<uintptr_t>(z) & 2) ? 1 : 0; }
// LAST: the value is not read again, so it need not be kept in the caches (k_score, 4,096 rows of 256 KB 191 / 181 us; k_gradient_apply
// behind k_score 584 / 555 together).  Not where a second kernel reads the row (slices and pieces of 300 rows of 600 KB 106 / 98).
template <bool LAST, class E> __device__ __forceinline__ raw4 load16(const E* p) {
  const typename Elem<E>::mem* m = reinterpret_cast<const typename Elem<E>::mem*>(p);
  if constexpr (LAST) return __builtin_nontemporal_load(m);
  else return *m;
}
// gradients are not read here again (8,192 rows of 64 KB 177 / 171 us, 300 of 400 KB in pieces 73 / 61)
template <class E> __device__ __forceinline__ void store16(E* p, raw4 r) {
  __builtin_nontemporal_store(static_cast<typename Elem<E>::mem>(r), reinterpret_cast<typename Elem<E>::mem*>(p));
}

// ---------------------------------------------------------------------------------------------
// statistics
// ---------------------------------------------------------------------------------------------
struct Stat { float m, s, w; };
struct __align__(16) Stat4 { float m, s, w, pad; };

__device__ __forceinline__ Stat stat_none() { return Stat{LOWEST, 0.0f, 0.0f}; }
__device__ __forceinline__ float exp2_(float y) { return __builtin_amdgcn_exp2f(y); }

// takes n values in and returns the largest; -inf adds nothing, NaN and +inf make s NaN
template <bool ENT, int N>
__device__ __forceinline__ float take(Stat& o, const float* v, float cl) {
  float vm = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) vm = fmaxf(vm, v[i]);
  const float m = fmaxf(o.m, vm), dl = fmaxf((o.m - m) * cl, Y_MIN), f = exp2_(dl);      // f = 1 where m stays: cheaper than a branch
  if (ENT) o.w = (o.w + o.s * dl) * f;
  o.s *= f;
  o.m = m;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = (v[i] - o.m) * cl, e = exp2_(y);
    o.s += e;
    if (ENT) o.w = __builtin_fmaf(e, fmaxf(y, Y_MIN), o.w);
  }
  return vm;
}

// lanes of a quad 1 0 3 2 and 2 3 0 1, lanes of 8 and of 16 backwards
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_keep(float x, float old) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float lane_float(float x, uint32_t lane) { return __uint_as_float(lane_value(__float_as_uint(x), lane)); }
__device__ __forceinline__ float wave_max_f(float x) {
  x = fmaxf(x, dpp_keep<DPP_ROW_SHR + 1, 0xF>(x, x));
  x = fmaxf(x, dpp_keep<DPP_ROW_SHR + 2, 0xF>(x, x));
  x = fmaxf(x, dpp_keep<DPP_ROW_SHR + 4, 0xF>(x, x));
  x = fmaxf(x, dpp_keep<DPP_ROW_SHR + 8, 0xF>(x, x));
  x = fmaxf(x, dpp_keep<DPP_BCAST15, 0xA>(x, x));
  x = fmaxf(x, dpp_keep<DPP_BCAST31, 0xC>(x, x));
  return lane_float(x, 63);
}
__device__ __forceinline__ float wave_sum_f(float x) {
  x += dpp_keep<DPP_ROW_SHR + 1, 0xF>(x, 0.0f);
  x += dpp_keep<DPP_ROW_SHR + 2, 0xF>(x, 0.0f);
  x += dpp_keep<DPP_ROW_SHR + 4, 0xF>(x, 0.0f);
  x += dpp_keep<DPP_ROW_SHR + 8, 0xF>(x, 0.0f);
  x += dpp_keep<DPP_BCAST15, 0xA>(x, 0.0f);
  x += dpp_keep<DPP_BCAST31, 0xC>(x, 0.0f);
  return lane_float(x, 63);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_zero_d(double x) {
  return __builtin_bit_cast(double, dpp_or_zero64<CTRL, ROWS>(__builtin_bit_cast(uint64_t, x)));
}
__device__ __forceinline__ double wave_sum_d(double x) {
  x += dpp_zero_d<DPP_ROW_SHR + 1, 0xF>(x);
  x += dpp_zero_d<DPP_ROW_SHR + 2, 0xF>(x);
  x += dpp_zero_d<DPP_ROW_SHR + 4, 0xF>(x);
  x += dpp_zero_d<DPP_ROW_SHR + 8, 0xF>(x);
  x += dpp_zero_d<DPP_BCAST15, 0xA>(x);
  x += dpp_zero_d<DPP_BCAST31, 0xC>(x);
  return __builtin_bit_cast(double, lane_value64(__builtin_bit_cast(uint64_t, x), 63));
}

// (m, s, w) brought to a larger maximum
template <bool ENT>
__device__ __forceinline__ Stat raised(Stat o, float m, float cl) {
  const float dl = fmaxf((o.m - m) * cl, Y_MIN), f = exp2_(dl);
  if (ENT) o.w = (o.w + o.s * dl) * f;
  o.s *= f;
  o.m = m;
  return o;
}

// the statistics of all lanes
template <bool ENT>
__device__ __forceinline__ Stat wave_stat(Stat o, float cl) {
  o = raised<ENT>(o, wave_max_f(o.m), cl);
  o.s = wave_sum_f(o.s);
  if (ENT) o.w = wave_sum_f(o.w);
  return o;
}

// the statistics of N = 2 .. 16 waves, lane i % N holding wave i's: sums over N neighbours by moves within the rows of 16 lanes
template <bool ENT, int N>
__device__ __forceinline__ Stat row16_stat(Stat o, float cl) {
  float m = o.m;
  if (N >= 2) m = fmaxf(m, dpp_keep<DPP_XOR1, 0xF>(m, m));
  if (N >= 4) m = fmaxf(m, dpp_keep<DPP_XOR2, 0xF>(m, m));
  if (N >= 8) m = fmaxf(m, dpp_keep<DPP_HALF_MIRROR, 0xF>(m, m));
  if (N >= 16) m = fmaxf(m, dpp_keep<DPP_MIRROR, 0xF>(m, m));
  o = raised<ENT>(o, m, cl);
  auto sum = [](float x) {
    if (N >= 2) x += dpp_keep<DPP_XOR1, 0xF>(x, 0.0f);
    if (N >= 4) x += dpp_keep<DPP_XOR2, 0xF>(x, 0.0f);
    if (N >= 8) x += dpp_keep<DPP_HALF_MIRROR, 0xF>(x, 0.0f);
    if (N >= 16) x += dpp_keep<DPP_MIRROR, 0xF>(x, 0.0f);
    return lane_float(x, 0);
  };
  o.m = lane_float(m, 0);
  o.s = sum(o.s);
  if (ENT) o.w = sum(o.w);
  return o;
}

// the statistics of all threads of a block of TH, in every thread; `box` holds TH / 64 of them
template <bool ENT, int TH>
__device__ __forceinline__ Stat block_stat(Stat o, float cl, Stat* box) {
  o = wave_stat<ENT>(o, cl);
  if (TH == 64) return o;
  if (lane_id() == 0) box[threadIdx.x >> 6] = o;
  __syncthreads();
  o = box[lane_id() % (TH / 64)];                                     // every row of 16 lanes holds all of them, once each or more
  return row16_stat<ENT, TH / 64>(o, cl);
}

// Of a finished row's sums: the logarithm is taken where an output needs it (the gradient does not, unless the entropy's).
__device__ __forceinline__ float row_entropy(const Stat& o) { return o.s == 0.0f ? 0.0f : logf(o.s) - LN2 * (o.w / o.s); }
__device__ __forceinline__ float row_lse(const Stat& o, float c) { return o.s == 0.0f ? -INFINITY : o.m * c + logf(o.s); }
// also where the row holds nothing else (s = 0)
__device__ __forceinline__ float log_prob(const Stat& o, float z, float c) {
  return z == -INFINITY && o.s == o.s ? -INFINITY : (z - o.m) * c - logf(o.s);
}

// ---------------------------------------------------------------------------------------------
// walking along a row: U loads of 16 bytes of a thread are under way at a time
// ---------------------------------------------------------------------------------------------
// whole(v, r): the thread's vectors v, v + TH, ...; vector v begins at value first + v N, those from nvec on hold -inf.  Then at most one call
// single(index, value) for the thread's value before or behind the vectors.
template <bool LAST, class E, int TH, int U, class F, class G>
__device__ __forceinline__ void walk(const E* z, uint32_t n, uint32_t first, F&& whole, G&& single) {
  constexpr int N = Elem<E>::N;
  const uint32_t nvec = (n - first) / N;
  for (uint32_t v0 = threadIdx.x; v0 < nvec; v0 += TH * U) {
    raw4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = raw4{Elem<E>::MINUS_INF, Elem<E>::MINUS_INF, Elem<E>::MINUS_INF, Elem<E>::MINUS_INF};
      const uint32_t v = v0 + u * TH;
      if (v < nvec) r[u] = load16<LAST>(z + first + static_cast<uint64_t>(v) * N);
    }
    whole(v0, r);
  }
  const uint32_t i = threadIdx.x < first ? threadIdx.x : nvec * N + threadIdx.x;
  if (i < n) single(i, static_cast<float>(z[i]));
}

template <bool LAST, class E, int TH, bool ENT>
__device__ __forceinline__ Stat pass_stat(const E* z, uint32_t n, float cl) {
  constexpr int N = Elem<E>::N, U = 4;
  Stat o = stat_none();
  walk<LAST, E, TH, U>(z, n, odd_ones(z),
    [&](uint32_t, const raw4* r) {
      float v[U * N];
#pragma unroll
      for (int u = 0; u < U; ++u) Elem<E>::unpack(r[u], v + u * N);
      take<ENT, U * N>(o, v, cl);
    },
    [&](uint32_t, float x) { take<ENT, 1>(o, &x, cl); });
  return o;
}

// dz = e (A + B y) with y = (x - m) cl, e = exp2(y): the gradient in a class that nothing is given for, A and B divided by s
struct Gradient { float cl, m, A, B; };
template <bool ENT>
__device__ __forceinline__ float gradient_value(const Gradient& f, float x) {
  const float y = (x - f.m) * f.cl, e = exp2_(y);
  return ENT ? e * __builtin_fmaf(f.B, fmaxf(y, Y_MIN), f.A) : e * f.A;
}

struct NoneOut { __device__ __forceinline__ uint32_t operator()(uint32_t) const { return 0; } };

// an integer that orders like the value (not for NaN; -0 counts as +0)
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t u = __float_as_uint(z + 0.0f);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// A piece of a row that the block holds in registers, NV vectors a thread and the values behind the last whole vector one a thread: it
// is read from memory once, whatever is made of it.  load() only starts the loads; loads past the end go to the last vector, and
// settle() makes -inf of them.
template <bool LAST, class E, int TH, int NV>
struct Held {
  static constexpr int N = Elem<E>::N;
  static constexpr uint32_t SIZE = TH * NV * N;                        // values in whole vectors
  raw4 r[NV];
  uint32_t last;                                                       // its bits
  uint32_t first, nvec, n;                                             // vector v begins at value first + v N
  __device__ __forceinline__ uint32_t vec(int u) const { return threadIdx.x + u * TH; }
  __device__ __forceinline__ uint32_t last_index() const { return threadIdx.x < first ? threadIdx.x : nvec * N + threadIdx.x; }
  __device__ __forceinline__ void load(const E* z, uint32_t n_) {
    n = n_; first = odd_ones(z); nvec = (n - first) / N;
    if (nvec) {
#pragma unroll
      for (int u = 0; u < NV; ++u) r[u] = load16<LAST>(z + first + static_cast<uint64_t>(min(vec(u), nvec - 1)) * N);
    }
    last = *reinterpret_cast<const typename Elem<E>::bits*>(z + min(last_index(), n - 1));
  }
  // What is made of vector u comes after `y` is known: keeps the compiler from waiting for all loads before the first sum, and from
  // holding all values unpacked from one use to the next.  (The branches that pass over empty pieces do so too: with both, 16 vectors of
  // 16-bit values take 93 to 95 VGPRs, and this alone is one or two of them in the kernels of few vectors.)
  __device__ __forceinline__ void in_order(int u, float& y) { asm volatile("" : "+v"(r[u]), "+v"(y)); }
  __device__ __forceinline__ float last_value(float& y) {              // (the last load: waiting for it is waiting for all)
    asm volatile("" : "+v"(last), "+v"(y));
    return Elem<E>::from_bits(last);
  }
  __device__ __forceinline__ void settle(int u) {
    if ((u + 1) * TH <= nvec) return;                                  // the same for all threads
    asm volatile("");                                                  // ... and a branch: the four selections below are not for every vector
    const bool out = vec(u) >= nvec;
#pragma unroll
    for (int q = 0; q < 4; ++q) r[u][q] = out ? Elem<E>::MINUS_INF : r[u][q];
  }
  static constexpr int U = NV < 16 / N ? NV : 16 / N;                  // vectors that are taken in together: 16 values
  // out(v): the bits of the values of vector v - 1 that are left out (v = 0: of the values before vector 0).  most[i]: the largest of vectors i U .. i U + U - 1
  template <bool ENT, class F>
  __device__ __forceinline__ Stat stat(float cl, F&& out, float (&most)[NV / U]) {
    Stat o = stat_none();
#pragma unroll
    for (int u0 = 0; u0 < NV; u0 += U) {
      most[u0 / U] = -INFINITY;
      if (u0 * TH >= nvec) continue;                                   // the same for all threads: nothing of the piece is left
      float v[U * N];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        in_order(u0 + u, o.s);
        if (ENT) in_order(u0 + u, o.w);
        settle(u0 + u);
        const uint32_t bits = out(min(vec(u0 + u), nvec) + 1);
        if (bits) Elem<E>::erase(r[u0 + u], bits);
        Elem<E>::unpack(r[u0 + u], v + u * N);
      }
      most[u0 / U] = take<ENT, U * N>(o, v, cl);
    }
    const float xl = last_value(o.s);
    const bool left_out = threadIdx.x < N && out(threadIdx.x < first ? 0 : nvec + 1) >> (threadIdx.x < first ? N - first : threadIdx.x - first) & 1;
    const float x = last_index() < n && !left_out ? xl : -INFINITY;
    take<ENT, 1>(o, &x, cl);
    return o;
  }
  template <bool ENT>
  __device__ __forceinline__ Stat stat(float cl) {
    float most[NV / U];
    return stat<ENT>(cl, NoneOut(), most);
  }
  // f(index, value) for the values that are at least `tau`, found by their chunk's largest.  A thread has few such chunks, and goes
  // through them one by one while the others go through theirs (chunk by chunk for all threads, almost every chunk has one
  // somewhere in the wave).  Where tau is -inf, the values of -inf only from the vectors that begin before `keep`.
  template <class F>
  __device__ __forceinline__ void at_least(float tau, uint32_t keep, const float (&most)[NV / U], F&& f) {
    constexpr int C = NV / U, W = 4 * U;                               // chunks, words of one
    uint32_t chunks = 0;
#pragma unroll
    for (int i = 0; i < C; ++i) chunks |= most[i] >= (first + vec(i * U) * N < keep ? tau : fmaxf(tau, LOWEST)) ? 1u << i : 0u;
    while (chunks) {
      const uint32_t i = __builtin_ctz(chunks);
      chunks &= chunks - 1;
      uint32_t w[W];
#pragma unroll
      for (int x = 0; x < W; ++x) {
        w[x] = r[x / 4][x % 4];
#pragma unroll
        for (int j = 1; j < C; ++j) w[x] = i == static_cast<uint32_t>(j) ? r[j * U + x / 4][x % 4] : w[x];
      }
      uint32_t hits = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t v = threadIdx.x + (i * U + u) * TH;
        const float least = first + v * N < keep ? tau : fmaxf(tau, LOWEST);
        float x[N];
        Elem<E>::unpack(raw4{w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]}, x);
        uint32_t h = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) h |= x[q] >= least ? 1u << q : 0u;
        if (v < nvec) hits |= h << u * N;
      }
      while (hits) {
        const uint32_t q = __builtin_ctz(hits);
        hits &= hits - 1;
        uint32_t x = w[0];
#pragma unroll
        for (int j = 1; j < W; ++j) x = q / (N / 4) == static_cast<uint32_t>(j) ? w[j] : x;
        f(first + (threadIdx.x + (i * U + q / N) * TH) * N + q % N, Elem<E>::of_word(x, q));
      }
    }
    const float x = Elem<E>::from_bits(last);
    if (last_index() < n && x >= (last_index() < keep ? tau : fmaxf(tau, LOWEST))) f(last_index(), x);
  }
  // how many values reach `least` (above -inf), of a wave that holds the piece; after stat()
  __device__ __forceinline__ uint32_t count(float least) {
    uint32_t c = __popcll(__ballot(last_index() < n && Elem<E>::from_bits(last) >= least));
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (u / U * U * TH >= nvec) continue;                            // (what stat() has passed over)
      asm volatile("" : "+v"(r[u]));                                   // unpacked anew for every count: the values would not leave room for other waves
      float v[N];
      Elem<E>::unpack(r[u], v);
#pragma unroll
      for (int q = 0; q < N; ++q) c += __popcll(__ballot(v[q] >= least));
    }
    return c;
  }
  // the gradient of the piece; where class t is in it, `add` comes on top and given(its logit) is called
  template <bool ENT, class F>
  __device__ __forceinline__ void gradient(E* dz, Gradient f, uint32_t t, float add, F&& given) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (u * TH >= nvec) continue;
      in_order(u, f.A);
      float v[N];
      Elem<E>::unpack(r[u], v);
      const uint32_t q0 = t - first - vec(u) * N;
      if (q0 < static_cast<uint32_t>(N) && vec(u) < nvec) {
        float x = v[0];
#pragma unroll
        for (int q = 0; q < N; ++q) x = q0 == static_cast<uint32_t>(q) ? v[q] : x;
        given(x);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = gradient_value<ENT>(f, v[q]) + (q0 == static_cast<uint32_t>(q) ? add : 0.0f);
      } else {
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = gradient_value<ENT>(f, v[q]);
      }
      if (vec(u) < nvec) store16((dz + first + u * TH * N) + threadIdx.x * N, Elem<E>::pack(v));      // one offset for all u
    }
    if (last_index() < n) {
      const float x = last_value(f.A);
      if (t == last_index()) given(x);
      dz[last_index()] = static_cast<E>(gradient_value<ENT>(f, x) + (t == last_index() ? add : 0.0f));
    }
  }
};
// a barrier for what is in LDS: loads from memory stay under way
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ---------------------------------------------------------------------------------------------
// the K largest values of a row, ties to the lower index
// ---------------------------------------------------------------------------------------------
// orders like (value, lower index first); no two entries of a row have the same key, and 0 is none's
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o >> 31 ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ uint64_t top_key(float z, uint32_t i) { return static_cast<uint64_t>(ordered(z)) << 32 | (0xFFFFFFFFu - i); }
__device__ __forceinline__ float key_value(uint64_t k) { return from_ordered(static_cast<uint32_t>(k >> 32)); }
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xFFFFFFFFu - static_cast<uint32_t>(k); }

template <uint32_t CAP>
struct TopBox {
  __align__(16) uint64_t list[CAP + 8];    // zeros behind the last one up to a multiple of 8
  uint16_t above[CAP], place[CAP];
  uint32_t equal[CAP];
  __align__(16) float group[GROUPS];
  float tau;
  uint32_t n;
  uint64_t kth;
};

// f(key, rank) for list[0 .. held), all of them different.  Upper halves are compared with all others (64 bits at a time cost twice as
// much), whole keys with the few that have the same upper half (or with all, where they are many).
template <int TH, uint32_t CAP, class F>
__device__ __forceinline__ void ranked(TopBox<CAP>& b, uint32_t held, F&& f) {
  if (threadIdx.x < 8) b.list[held + threadIdx.x] = 0;
  for (uint32_t i = threadIdx.x; i < held; i += TH) b.equal[i] = 0;
  __syncthreads();
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < held; i += TH) {
    const uint32_t k = static_cast<uint32_t>(b.list[i] >> 32);
    uint32_t above = 0;
#pragma unroll 1
    for (uint32_t j = 0; j < held; j += 8) {                          // 8 at a time: one at a time every comparison waits for its own read
#pragma unroll
      for (uint32_t q = 0; q < 8; q += 2) {
        const uint4 o = *reinterpret_cast<const uint4*>(b.list + j + q);
        above += (o.y > k) + (o.w > k);
      }
    }
    b.above[i] = above;
    b.place[above + atomicAdd(&b.equal[above], 1u)] = i;
  }
  __syncthreads();
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < held; i += TH) {
    const uint64_t k = b.list[i];
    const uint32_t above = b.above[i], equal = b.equal[above];
    uint32_t rank = above;
    if (equal > 16) {
      rank = 0;
#pragma unroll 1
      for (uint32_t j = 0; j < held; j += 8) {
#pragma unroll
        for (uint32_t q = 0; q < 8; q += 2) {
          const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(b.list + j + q);
          rank += (o.x > k) + (o.y > k);
        }
      }
    } else if (equal > 1) {
      for (uint32_t j = above; j < above + equal; ++j) rank += b.list[b.place[j]] > k;
    }
    f(k, rank);
  }
}

// The K-th largest of a wave's values but for the lower 16 bits of its ordered(), which are 0: less than it, found bit by bit, with
// reach(trial) values of the wave reaching a trial.  -inf where fewer than K are above -inf.
template <class F>
__device__ __forceinline__ float wave_kth(uint32_t K, F&& reach) {
  uint32_t T = 0;
#pragma unroll 1
  for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1)
    if (reach(T | bit) >= K) T |= bit;
  return T > ordered(-INFINITY) ? from_ordered(T) : -INFINITY;
}

// The last part of block_top: the K largest of the entries that scan() offers from `bound` on; at least K are.
template <int TH, uint32_t CAP, class S, class F>
__device__ __forceinline__ void block_top_from(uint64_t bound, uint32_t K, TopBox<CAP>& b, S&& scan, F&& out) {
  for (;;) {
    scan([&](uint64_t k) {
      if (k < bound) return;
      const uint32_t at = atomicAdd(&b.n, 1u);
      if (at < CAP) b.list[at] = k;
    });
    __syncthreads();
    const uint32_t found = b.n;
    if (found <= CAP) {
      ranked<TH>(b, found, [&](uint64_t k, uint32_t rank) { if (rank < K) out(rank, k); });
      return;
    }
    __syncthreads();                                                  // (list[REFINE] is about to be cleared)
    ranked<TH>(b, REFINE, [&](uint64_t k, uint32_t rank) { if (rank == K - 1) b.kth = k; });
    __syncthreads();
    bound = b.kth;
    if (threadIdx.x == 0) b.n = 0;
    __syncthreads();
  }
}

// The K largest of n entries that the threads of a block hold, through out(rank, key); `most`: the thread's largest value (-inf:
// none); scan(tau, f): f(key) for each of the thread's entries whose value is at least tau.
// Groups of threads hold distinct entries, so the K-th largest of the groups' maxima is at most the K-th largest value: only what
// reaches it is a candidate (for values in no particular order a few more than K, in the few threads whose maximum reaches it).  One
// wave finds its upper 16 bits; less than it will do as well.  Values of -inf count only where fewer than K others are left; of those the lowest indices are wanted, and they are among the first
// K entries: a mask that leaves less than K classes does not make all others candidates.  If more than CAP entries are candidates (many equal or ordered values), the K-th largest of the first REFINE that found room
// is the next bound: a larger one, since keys differ, and for entries in no particular order it leaves K / REFINE of them.
// OWN: `most` is the largest of what the thread's scan() goes through (else of any entries, no two threads' the same).
template <int TH, uint32_t CAP, class OWN, class S, class F>
__device__ __forceinline__ void block_top(uint32_t n, uint32_t K, float most, TopBox<CAP>& b, OWN, S&& scan, F&& out) {
  constexpr uint32_t PER = TH > GROUPS ? TH / GROUPS : 1, G = TH / PER, M = G / 64;
  static_assert(PER == 1 || PER == 2 || PER == 4, "a group is a thread, or two or four lanes of a quad");
  float gm = most;
  if (PER >= 2) gm = fmaxf(gm, dpp_keep<DPP_XOR1, 0xF>(gm, gm));          // the lanes of a quad: 1 0 3 2, then 2 3 0 1
  if (PER == 4) gm = fmaxf(gm, dpp_keep<DPP_XOR2, 0xF>(gm, gm));
  if (TH > 64 && threadIdx.x % PER == 0) b.group[threadIdx.x / PER] = gm;
  if (threadIdx.x == 0) b.n = 0;
  __syncthreads();
  if (threadIdx.x < 64) {
    float tau = -INFINITY;
    if (K <= G && n > 2 * K) {
      uint32_t o[M];
#pragma unroll
      for (uint32_t j = 0; j < M; ++j) o[j] = ordered(TH > 64 ? b.group[lane_id() + 64 * j] : gm);
      tau = wave_kth(K, [&](uint32_t trial) {
        uint32_t c = 0;
#pragma unroll
        for (uint32_t j = 0; j < M; ++j) c += __popcll(__ballot(o[j] >= trial));
        return c;
      });
    }
    if (threadIdx.x == 0) b.tau = tau;
  }
  __syncthreads();
  const float tau = b.tau;
  block_top_from<TH>(0, K, b, [&](auto&& f) { if (!OWN::value || most >= tau) scan(tau, f); }, out);
}

// the same for a row in memory
template <class E, int TH, uint32_t CAP, class F>
__device__ __forceinline__ void row_top(const E* z, uint32_t n, uint32_t K, float most, TopBox<CAP>& b, F&& out) {
  constexpr int N = Elem<E>::N, U = 4;
  const uint32_t first = odd_ones(z), nvec = (n - first) / N;
  block_top<TH, CAP>(n, K, most, b, std::true_type(), [&](float tau, auto&& f) {
    walk<true, E, TH, U>(z, n, first,
      [&](uint32_t v0, const raw4* r) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (v0 + u * TH >= nvec) continue;
          float v[N];
          Elem<E>::unpack(r[u], v);
          const uint32_t i = first + (v0 + u * TH) * N;
          const float least = i < K ? tau : fmaxf(tau, LOWEST);
#pragma unroll
          for (int q = 0; q < N; ++q) if (v[q] >= least) f(top_key(v[q], i + q));
        }
      },
      [&](uint32_t i, float x) { if (x >= (i < K ? tau : fmaxf(tau, LOWEST))) f(top_key(x, i)); });
  }, out);
}

// ---------------------------------------------------------------------------------------------
// log probabilities of given tokens
// ---------------------------------------------------------------------------------------------
struct ScoreArgs {
  const void* z;
  uint64_t stride;
  uint32_t rows, vocab, K;
  float c;
  const int64_t* target;
  float *logprob, *entropy, *lse;
  int32_t* top_index;
  float* top_logprob;
  float* stats;
};

// the given class and its logit, read by one thread ahead of the row: two reads, one behind the other
template <class E>
struct Given {
  int64_t t;
  E x;
  __device__ __forceinline__ void load(const ScoreArgs& a, uint32_t row, const E* z) {
    if (!a.logprob || threadIdx.x != 0) return;
    t = a.target[row];
    x = z[t >= 0 && t < static_cast<int64_t>(a.vocab) ? t : 0];
  }
  __device__ __forceinline__ float logprob(const ScoreArgs& a, const Stat& o) const {
    return t < 0 ? 0.0f : t >= static_cast<int64_t>(a.vocab) ? NAN : log_prob(o, static_cast<float>(x), a.c);
  }
};

template <class E>
__device__ __forceinline__ void score_outputs(const ScoreArgs& a, uint32_t row, const Given<E>& g, const Stat& o) {
  if (a.logprob) a.logprob[row] = g.logprob(a, o);
  if (a.entropy) a.entropy[row] = row_entropy(o);
  if (a.lse) a.lse[row] = row_lse(o, a.c);
  if (a.stats) { float* s = a.stats + 4ull * row; s[0] = o.m; s[1] = o.s; s[2] = row_entropy(o); s[3] = 0.0f; }
}
// f(out) with out(rank, key) writing an alternative; where the row has no order (a NaN or +inf in it) the outputs say so instead
template <int TH, class F>
__device__ __forceinline__ void alternatives(const ScoreArgs& a, uint32_t row, const Stat& o, F&& f) {
  int32_t* ti = a.top_index ? a.top_index + static_cast<uint64_t>(row) * a.K : nullptr;
  float* tl = a.top_logprob ? a.top_logprob + static_cast<uint64_t>(row) * a.K : nullptr;
  if (o.s != o.s) {
    for (uint32_t k = threadIdx.x; k < a.K; k += TH) { if (ti) ti[k] = -1; if (tl) tl[k] = NAN; }
    return;
  }
  if (o.s == 0.0f) {                                                  // nothing but -inf
    for (uint32_t k = threadIdx.x; k < a.K; k += TH) { if (ti) ti[k] = static_cast<int32_t>(k); if (tl) tl[k] = -INFINITY; }
    return;
  }
  f([&](uint32_t rank, uint64_t k) {
    if (ti) ti[rank] = static_cast<int32_t>(key_index(k));
    if (tl) tl[rank] = log_prob(o, key_value(k), a.c);
  });
}

// A block per row, which it walks along once: bound by memory, and as near by its instructions (4,096 rows of 128,000 bf16 with the entropy
// 154 - 160 us, 6.6 - 6.8 TB/s; 9.9 vector instructions per 64 values (SQ_INSTS_VALU), of four cycles each 131 us of issue on 1,024 SIMDs at
// 2.4 GHz, to which comes what the exponential takes longer).  Eight loads a thread under way instead of four cost registers, hence
// waves: 214 us.  With alternatives (rows of more than 64 slices only) the threads that hold candidates read their shares again.
template <bool LAST, class E, int TH, bool ENT, bool TOP>
__global__ __launch_bounds__(TH) void k_score(ScoreArgs a) {
  __shared__ Stat box[16];
  __shared__ TopBox<TOP ? CAND_CAP : 1> tb;
  const float cl = a.c * LOG2E;
  const uint64_t row = block_number();
  if (row >= a.rows) return;
  const E* z = static_cast<const E*>(a.z) + row * a.stride;
  Given<E> given;
  given.load(a, row, z);
  const Stat mine = pass_stat<LAST && !TOP, E, TH, ENT>(z, a.vocab, cl);
  const Stat o = block_stat<ENT, TH>(mine, cl, box);
  if (threadIdx.x == 0) score_outputs(a, row, given, o);
  if (TOP)
    alternatives<TH>(a, row, o, [&](auto&& out) {
      row_top<E, TH, TOP ? CAND_CAP : 1>(z, a.vocab, a.K, mine.s > 0.0f ? mine.m : -INFINITY, tb, out);
    });
}

// Alternatives of a row that fits the block's registers: read once, ranked from there.  What ranking costs comes on top of the memory's time, as
// far as other rows of the compute unit do not fill the gap: 4,096 rows of 32,000 bf16, 20 alternatives 48 us (their bytes 43), 128
// alternatives 67; short rows are bound by the ranking's issue slots (16,384 rows of 2,000: 25 us, their bytes 11).
template <class E, int TH, int NV, bool ENT>
__global__ __launch_bounds__(TH) void k_score_held(ScoreArgs a) {
  constexpr uint32_t CAP = TH == 64 ? REFINE : CAND_CAP;               // (one wave: LDS would limit how many are resident)
  __shared__ Stat box[16];
  __shared__ TopBox<CAP> tb;
  const float cl = a.c * LOG2E;
  const uint64_t row = block_number();
  if (row >= a.rows) return;
  const E* z = static_cast<const E*>(a.z) + row * a.stride;
  Given<E> given;
  Held<true, E, TH, NV> h;
  h.load(z, a.vocab);
  given.load(a, row, z);
  float most[NV / Held<true, E, TH, NV>::U];
  const Stat mine = h.template stat<ENT>(cl, NoneOut(), most);
  const Stat o = block_stat<ENT, TH>(mine, cl, box);
  if (threadIdx.x == 0) score_outputs(a, row, given, o);
  alternatives<TH>(a, row, o, [&](auto&& out) {
    auto scan = [&](float tau, auto&& f) { h.at_least(tau, a.K, most, [&](uint32_t i, float x) { f(top_key(x, i)); }); };
    if constexpr (TH == 64) {
      // All values counted instead of the vectors' maxima (16 times), unless ranking all is little.  us, 12,000 rows of bf16, with maxima /
      // this: 210 values, 32 and 128 alternatives 65 / 23, 70 / 43; 500, 128 208 / 42; 800, 128 236 / 54.  Where there are more vectors:
      // 500, 32 16 / 21; 210, 20 15 / 20.  Ranking all: 64, 20 19 / 23; 70, 64 23 / 27.
      if (maxima_say_little(a.K, h.nvec) && a.vocab > min(max(2 * a.K, 64u), 128u)) {
        const float tau = wave_kth(a.K, [&](uint32_t trial) { return h.count(from_ordered(trial)); });
        if (threadIdx.x == 0) tb.n = 0;
        __syncthreads();
        block_top_from<TH>(0, a.K, tb, [&](auto&& f) { scan(tau, f); }, out);
        return;
      }
    }
    block_top<TH, CAP>(a.vocab, a.K, mine.s > 0.0f ? mine.m : -INFINITY, tb, std::true_type(), scan, out);
  });
}

// ---------------------------------------------------------------------------------------------
// rows split into slices, a block each, where there are few rows or they do not fit a block's registers
// ---------------------------------------------------------------------------------------------
constexpr uint32_t SLICES_MAX = 64;        // slices of a row at most: a wave joins them

struct Slices {
  uint32_t S, len;                         // slices of a row, values in each but the last
  Stat4* part;                             // [rows, S]
  uint64_t* key;                           // [rows, S, K] the slice's largest, largest first; 0: none
};

// NV = 0: the slice is walked along, without alternatives.  2,048 rows of 50,001 fp32 in four slices each, 64 alternatives: 78 us (5.2
// TB/s), by one block of 1024 x 16 a row 110, since nothing fills the time in which that block ranks.
template <class E, int NV, bool ENT>
__global__ __launch_bounds__(256) void k_slice_stats(ScoreArgs a, Slices sl) {
  __shared__ Stat box[4];
  __shared__ TopBox<NV ? CAND_CAP : 1> tb;
  const float cl = a.c * LOG2E;
  const uint64_t pieces = static_cast<uint64_t>(a.rows) * sl.S;
  const uint64_t p = block_number();
  if (p >= pieces) return;
  const uint32_t row = static_cast<uint32_t>(p / sl.S), i0 = static_cast<uint32_t>(p % sl.S) * sl.len, n = min(a.vocab - i0, sl.len);
  const E* z = static_cast<const E*>(a.z) + row * a.stride + i0;
  auto hand_over = [&](const Stat& mine) {
    const Stat o = block_stat<ENT, 256>(mine, cl, box);
    if (threadIdx.x == 0) sl.part[p] = Stat4{o.m, o.s, o.w, 0.0f};
  };
  if constexpr (NV == 0) hand_over(pass_stat<false, E, 256, ENT>(z, n, cl));
  else {
    Held<true, E, 256, NV> h;
    h.load(z, n);
    float most[NV / Held<true, E, 256, NV>::U];
    const Stat mine = h.template stat<ENT>(cl, NoneOut(), most);
    hand_over(mine);
    uint64_t* key = sl.key + p * a.K;
    for (uint32_t k = threadIdx.x; k < a.K; k += 256) if (k >= n) key[k] = 0;      // (of a slice with a NaN nobody looks at the keys)
    block_top<256, CAND_CAP>(n, a.K, mine.s > 0.0f ? mine.m : -INFINITY, tb, std::true_type(),
                             [&](float tau, auto&& f) { h.at_least(tau, a.K, most, [&](uint32_t i, float x) { f(top_key(x, i0 + i)); }); },
                             [&](uint32_t rank, uint64_t k) { key[rank] = k; });
  }
}

// every wave: the statistics of a row from those of its slices
template <bool ENT>
__device__ __forceinline__ Stat joined(const Slices& sl, uint32_t row, float cl) {
  Stat o = stat_none();
  if (lane_id() < sl.S) { const Stat4 p = sl.part[static_cast<uint64_t>(row) * sl.S + lane_id()]; o = Stat{p.m, p.s, p.w}; }
  return wave_stat<ENT>(o, cl);
}

// A block per row: a chain of reads and barriers, 5 us for 64 rows, 8 for 2,048.
template <class E, bool ENT>
__global__ __launch_bounds__(256) void k_score_join(ScoreArgs a, Slices sl) {
  __shared__ TopBox<CAND_CAP> tb;
  const float cl = a.c * LOG2E;
  const uint64_t row = block_number();
  if (row >= a.rows) return;
  const uint32_t n = sl.S * a.K;
  const uint64_t* key = sl.key + row * n;
  constexpr uint32_t M = 8;
  uint64_t mine[M];
#pragma unroll
  for (uint32_t j = 0; j < M; ++j) mine[j] = threadIdx.x + 256 * j < n ? key[threadIdx.x + 256 * j] : 0;
  // The bound comes from the first 256 / S of every slice, 208 of them or more (S = 52), or from all S K where K is less: hardly ever are more
  // of a slice's among the K.
  const uint32_t place = threadIdx.x / sl.S;
  const uint64_t sample = place < a.K && place < 256 / sl.S ? key[threadIdx.x % sl.S * a.K + place] : 0;
  Given<E> given;
  given.load(a, row, static_cast<const E*>(a.z) + row * a.stride);
  const Stat o = joined<ENT>(sl, row, cl);
  if (threadIdx.x == 0) score_outputs(a, row, given, o);
  if (a.K == 0) return;
  alternatives<256>(a, row, o, [&](auto&& out) {
    block_top<256, CAND_CAP>(n, a.K, sample ? key_value(sample) : -INFINITY, tb, std::false_type(), [&](float tau, auto&& f) {
      auto offer = [&](uint64_t k) { if (k && key_value(k) >= tau) f(k); };
#pragma unroll
      for (uint32_t j = 0; j < M; ++j) offer(mine[j]);
      for (uint32_t i = threadIdx.x + 256 * M; i < n; i += 256) offer(key[i]);
    }, out);
  });
}

// ---------------------------------------------------------------------------------------------
// the gradient of log probabilities and entropies
// ---------------------------------------------------------------------------------------------
struct GradArgs {
  const void* z;
  void* dz;
  uint64_t stride, dstride;
  uint32_t rows, vocab;
  float c;
  const int64_t* target;
  const float *g, *h;
  const float* stats;
  float *logprob, *entropy;
};

struct RowGradient {
  Gradient f;
  uint32_t t;                              // the given class, or 2^32 - 1
  float add;                               // what it gets on top
};

// what is given for a row, read ahead of it
struct RowWeights { int64_t t; float g, h; };
template <bool ENT>
__device__ __forceinline__ RowWeights row_weights(const GradArgs& a, uint32_t row) {
  RowWeights w;
  w.t = a.target ? a.target[row] : -1;
  w.g = a.g ? a.g[row] : 0.0f;
  w.h = ENT && a.h ? a.h[row] : 0.0f;
  if (w.t < 0) w.g = 0.0f;
  if (w.t >= static_cast<int64_t>(a.vocab)) w.g = NAN;
  return w;
}
template <bool ENT>
__device__ __forceinline__ RowGradient row_gradient(const GradArgs& a, const RowWeights& w, const Stat& o, float H) {
  const bool empty = o.s == 0.0f;
  RowGradient r;
  r.f.cl = a.c * LOG2E; r.f.m = o.m;
  r.f.A = empty ? (w.t >= static_cast<int64_t>(a.vocab) ? NAN : 0.0f) : -a.c * (ENT ? w.g + w.h * (H - logf(o.s)) : w.g) / o.s;
  r.f.B = ENT && !empty ? -a.c * w.h * LN2 / o.s : 0.0f;
  r.t = w.t >= 0 && w.t < static_cast<int64_t>(a.vocab) ? static_cast<uint32_t>(w.t) : 0xFFFFFFFFu;
  r.add = empty ? 0.0f : a.c * w.g;
  return r;
}
// what a row hands out besides its gradient; the log probability of a given class comes from the thread that holds it
__device__ __forceinline__ void gradient_outputs(const GradArgs& a, uint32_t row, float H, const RowGradient& r, int64_t given) {
  if (a.entropy) a.entropy[row] = H;
  if (a.logprob && r.t == 0xFFFFFFFFu) a.logprob[row] = given < 0 ? 0.0f : NAN;
}

// A block per row, held in its registers: one read, one write, and bound by them (8,192 rows of 32,000 bf16 170 us, 6.2 TB/s, where a copy
// reaches 5.2; walking along the row twice, the second time mostly in the caches, 214).
template <class E, int TH, int NV, bool ENT>
__global__ __launch_bounds__(TH) void k_gradient_held(GradArgs a) {
  __shared__ Stat box[16];
  const float cl = a.c * LOG2E;
  const uint64_t row = block_number();
  if (row >= a.rows) return;
  const RowWeights w = row_weights<ENT>(a, row);
  Held<false, E, TH, NV> h;
  h.load(static_cast<const E*>(a.z) + row * a.stride, a.vocab);
  const Stat o = block_stat<ENT, TH>(h.template stat<ENT>(cl), cl, box);
  const float H = ENT ? row_entropy(o) : 0.0f;
  const RowGradient r = row_gradient<ENT>(a, w, o, H);
  h.template gradient<ENT>(static_cast<E*>(a.dz) + row * a.dstride, r.f, r.t, r.add,
                           [&](float x) { if (a.logprob) a.logprob[row] = log_prob(o, x, a.c); });
  if (threadIdx.x == 0) gradient_outputs(a, row, H, r, w.t);
}

// A piece of a row per block, the statistics known: the caller's, or (a.stats = NULL) joined from the slices'.  4,096 rows of 131,072 bf16
// with the entropy 348 us, 6.2 TB/s.  (Rows from the last to the first, so that what the forward call read last is still in a cache:
// 350.)
template <class E, bool ENT>
__global__ __launch_bounds__(256) void k_gradient_apply(GradArgs a, Slices sl) {
  constexpr int NV = 4;
  typedef Held<true, E, 256, NV> H;
  const uint32_t per = (a.vocab + H::SIZE - 1) / H::SIZE;
  const uint64_t pieces = static_cast<uint64_t>(a.rows) * per;
  const uint64_t p = block_number();
  if (p >= pieces) return;
  const uint32_t row = static_cast<uint32_t>(p / per), i0 = static_cast<uint32_t>(p % per) * H::SIZE, n = min(a.vocab - i0, H::SIZE);
  const RowWeights w = row_weights<ENT>(a, row);
  H h;
  h.load(static_cast<const E*>(a.z) + row * a.stride + i0, n);
  Stat o;
  float entropy;
  if (a.stats) { const float* s = a.stats + 4ull * row; o.m = s[0]; o.s = s[1]; entropy = s[2]; }
  else { o = joined<ENT>(sl, row, a.c * LOG2E); entropy = ENT ? row_entropy(o) : 0.0f; }
  const RowGradient r = row_gradient<ENT>(a, w, o, entropy);
  h.template gradient<ENT>(static_cast<E*>(a.dz) + row * a.dstride + i0, r.f, r.t - i0, r.add,
                           [&](float x) { if (a.logprob) a.logprob[row] = log_prob(o, x, a.c); });
  if (threadIdx.x == 0 && i0 == 0) gradient_outputs(a, row, entropy, r, w.t);
}

// ---------------------------------------------------------------------------------------------
// a teacher's top logits
// ---------------------------------------------------------------------------------------------
struct DistillArgs {
  const void* z;
  void* dz;
  uint64_t stride, dstride;
  uint32_t rows, vocab, K;
  float c, ct;
  const int32_t* index;
  const float *value, *tlse;
  const float* g;
  const float* stats_in;
  float *loss, *stats;
};

struct TeacherBox {
  int32_t key[HASH_SIZE];          // the classes, each in the first free slot from its own on
  uint32_t first[HASH_SIZE];       // where a class stands first
  int32_t index[TEACHER_MAX];      // -1: no entry
  float value[TEACHER_MAX];        // the teacher's logits
  float z[TEACHER_MAX];            // the student's logits there
  float q[TEACHER_MAX];            // the teacher's probabilities
  uint32_t bad, some;              // an index outside; whether the row teaches anything (a NaN counts)
  double lse, sum_q;               // of the teacher's logits
  float m, s, F, m_all;
  double t_all;                    // sum of exp(c (z_i - m_all)) over the whole row
};
template <int TH> constexpr int entries_of() { return (TEACHER_MAX + TH - 1) / TH; }

// The teacher's entries of a row: their classes in the box; entries that are none, and classes that stood earlier in the row, have
// index -1.  The student's logits there are on their way to x: teacher_logits() puts them into the box.  Ends behind a barrier.
template <int TH>
struct Entries {
  int32_t index[entries_of<TH>()];
  float value[entries_of<TH>()];
  __device__ __forceinline__ void load(const DistillArgs& a, uint64_t row) {
#pragma unroll
    for (int j = 0; j < entries_of<TH>(); ++j) {
      const uint64_t at = row * a.K + min(threadIdx.x + j * TH, a.K - 1);
      index[j] = a.index[at];
      value[j] = a.value[at];
    }
  }
};
template <class E, int TH>
__device__ __forceinline__ void teacher_entries(const DistillArgs& a, const E* z, TeacherBox& b, Entries<TH>& e, E (&x)[entries_of<TH>()]) {
  int32_t (&idx)[entries_of<TH>()] = e.index;
  constexpr int M = entries_of<TH>();
  uint32_t shift = 26;                                                // 4 slots per entry, 64 at least
  while (1u << (32 - shift) < 4 * a.K) --shift;
  const uint32_t slots = 1u << (32 - shift);
  for (uint32_t i = threadIdx.x; i < slots; i += TH) { b.key[i] = -1; b.first[i] = 0xFFFFFFFFu; }
  if (threadIdx.x == 0) b.bad = 0;
  lds_barrier();
  uint32_t slot[M];
#pragma unroll
  for (int j = 0; j < M; ++j) {
    const uint32_t k = threadIdx.x + j * TH;
    slot[j] = 0;
    if (k >= a.K) idx[j] = -1;
    if (idx[j] >= 0 && static_cast<uint32_t>(idx[j]) >= a.vocab) { b.bad = 1; idx[j] = -1; }
    x[j] = z[max(idx[j], 0)];
    if (idx[j] >= 0) {
      uint32_t s = (static_cast<uint32_t>(idx[j]) * 2654435761u) >> shift;
      for (;;) {                                                      // at most a quarter of the slots is taken
        const int32_t old = atomicCAS(&b.key[s], -1, idx[j]);
        if (old == -1 || old == idx[j]) break;
        s = (s + 1) & (slots - 1);
      }
      slot[j] = s;
      atomicMin(&b.first[s], k);
    }
  }
  lds_barrier();
#pragma unroll
  for (int j = 0; j < M; ++j) {
    const uint32_t k = threadIdx.x + j * TH;
    if (k < a.K) { b.index[k] = idx[j] >= 0 && b.first[slot[j]] == k ? idx[j] : -1; b.value[k] = e.value[j]; }
  }
  lds_barrier();
}
template <class E, int TH>
__device__ __forceinline__ void teacher_logits(const DistillArgs& a, TeacherBox& b, const E (&x)[entries_of<TH>()]) {
#pragma unroll
  for (int j = 0; j < entries_of<TH>(); ++j) {
    const uint32_t k = threadIdx.x + j * TH;
    if (k < a.K) b.z[k] = static_cast<float>(x[j]);
  }
}

// Marks the classes of [i0, i0 + len) that are entries: bits v N .. v N + N - 1 of the mask are vector v - 1's, those before `first` stand
// right before vector 0's.  index(k): entry k.
constexpr uint32_t mask_words(uint32_t len) { return (len + 8) / 32 + 1; }
template <int TH, int N, class F>
__device__ __forceinline__ void mark(uint32_t* mask, uint32_t i0, uint32_t len, uint32_t first, uint32_t K, F&& index) {
  for (uint32_t i = threadIdx.x; i < mask_words(len); i += TH) mask[i] = 0;
  lds_barrier();
  for (uint32_t k = threadIdx.x; k < K; k += TH) {
    const int32_t e = index(k);
    const uint32_t i = static_cast<uint32_t>(e) - i0, at = i + N - first;      // classes before the span are huge
    if (e >= 0 && i < len) atomicOr(&mask[at / 32], 1u << at % 32);
  }
  lds_barrier();
}
template <int N>
__device__ __forceinline__ uint32_t marks(const uint32_t* mask, uint32_t v) { return mask[v * N / 32] >> v * N % 32 & ((1u << N) - 1); }

// The statistics of a row's slice without the teacher's classes, whose places are marked in LDS, a span of the slice at a time.
template <class E, int TH, class F>
__device__ __forceinline__ Stat pass_rest(const E* z, uint32_t i0, uint32_t n, uint32_t K, float cl, uint32_t* mask, F&& index) {
  constexpr int N = Elem<E>::N, U = 4;
  Stat o = stat_none();
  for (uint32_t s0 = 0; s0 < n; s0 += MASK_SPAN) {
    const uint32_t len = min(n - s0, MASK_SPAN), first = odd_ones(z + s0), nvec = (len - first) / N;
    if (s0) __syncthreads();
    mark<TH, N>(mask, i0 + s0, len, first, K, index);
    walk<false, E, TH, U>(z + s0, len, first,
      [&](uint32_t v0, const raw4* r) {
        float v[U * N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t bits = v0 + u * TH < nvec ? marks<N>(mask, v0 + u * TH + 1) : 0;
          raw4 x = r[u];
          if (bits) Elem<E>::erase(x, bits);
          Elem<E>::unpack(x, v + u * N);
        }
        take<false, U * N>(o, v, cl);
      },
      [&](uint32_t i, float x) {
        const uint32_t at = i + N - first;
        if (!(mask[at / 32] >> at % 32 & 1)) take<false, 1>(o, &x, cl);
      });
  }
  return o;
}

// what lanes of a wave have written to LDS is there for its other lanes
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What follows is one wave's, K entries at most four times its lanes, in 64 bits: the loss is a difference of logarithms that nearly agree
// when the student is good.  The loops stay loops, to leave the registers to the row.

// the teacher's probabilities.  A row teaches nothing whose entries have no mass (none, or all of them -inf) and that leaves nothing over:
// without the rest as a class, or where its normaliser says that the teacher's row held nothing but -inf.
template <bool REST>
__device__ __forceinline__ void teacher_probabilities(const DistillArgs& a, uint64_t row, TeacherBox& b) {
  double lse = 0.0, top = 0.0;
  bool some = true;
  if (REST) {
    top = lse = a.tlse[row];
    some = lse != -INFINITY;
  } else {
    float most = -INFINITY;
    bool any = false;
#pragma unroll 1
    for (uint32_t k = lane_id(); k < a.K; k += 64)
      if (b.index[k] >= 0) { most = fmaxf(most, b.value[k]); any |= !(b.value[k] == -INFINITY); }
    some = __any(any);                                                // (a NaN is not -inf)
    top = static_cast<double>(wave_max_f(most)) * a.ct;
  }
  double* e = reinterpret_cast<double*>(b.key);                       // (the slots have done their work)
  static_assert(sizeof b.key >= TEACHER_MAX * sizeof(double), "room for an exponential per entry");
  double sum = 0.0;
#pragma unroll 1
  for (uint32_t k = lane_id(); k < a.K; k += 64)
    if (b.index[k] >= 0) {
      const double x = some ? exp(static_cast<double>(b.value[k]) * a.ct - top) : REST && b.value[k] != b.value[k] ? NAN : 0.0;
      if (REST) b.q[k] = static_cast<float>(x);
      else e[k] = x;
      sum += x;
    }
  sum = wave_sum_d(sum);
  if (sum != sum) some = true;
  if (!REST) {
#pragma unroll 1
    for (uint32_t k = lane_id(); k < a.K; k += 64) if (b.index[k] >= 0) b.q[k] = some ? static_cast<float>(e[k] / sum) : 0.0f;
    lse = top + log(sum);
  }
  if (lane_id() == 0) { b.lse = lse; b.sum_q = sum; b.some = some; }
  wave_lds_fence();
}

// What the row's statistics `o` (of the whole row, or with REST of the classes outside) make of it: m, s, F (dz_i = c g F softmax_i over
// what `o` covers), m_all, t_all.  Statistics that the caller kept (a.stats_in) take the place of `o`.
template <bool REST>
__device__ __forceinline__ void student_sums(const DistillArgs& a, uint64_t row, Stat o, TeacherBox& b) {
  const double c = a.c;
  double F = b.some ? 1.0 : 0.0, t = o.s;
  float m_all = o.m;
  if (a.stats_in) {
    const float* s = a.stats_in + 8ull * row;
    o.m = s[0]; o.s = s[1]; F = s[2]; m_all = s[3];
    t = s[4];                                                         // as taught() rounds it: nothing is lost
  } else if (REST) {
    float most = -INFINITY;
#pragma unroll 1
    for (uint32_t k = lane_id(); k < a.K; k += 64) if (b.index[k] >= 0) most = fmaxf(most, b.z[k]);
    m_all = fmaxf(wave_max_f(most), o.m);
    double inside = 0.0;
#pragma unroll 1
    for (uint32_t k = lane_id(); k < a.K; k += 64) if (b.index[k] >= 0) inside += exp((static_cast<double>(b.z[k]) - m_all) * c);
    inside = wave_sum_d(inside);
    const double outside = o.s == 0.0f ? 0.0 : o.s * exp((static_cast<double>(o.m) - m_all) * c);
    t = inside + outside;
    F = outside / t - fmax(1.0 - b.sum_q, 0.0);
    if (o.s == 0.0f) F = 0.0;                                         // nothing outside: the rest is left out
  }
  if (b.sum_q != b.sum_q) F = NAN;                                    // a NaN among the teacher's entries
  if (t == 0.0 || !b.some) F = 0.0;                                   // a row that leaves nothing, or teaches nothing
  if (b.bad || t != t) F = NAN;                                       // (t has met every logit: also the entries', where nothing else is left)
  if (lane_id() == 0) { b.m = o.m; b.s = o.s; b.F = static_cast<float>(F); b.m_all = m_all; b.t_all = t; }
  wave_lds_fence();
}

template <bool REST>
__device__ __forceinline__ float distill_loss(const DistillArgs& a, Stat o, const TeacherBox& b) {
  const double c = a.c, m_all = b.m_all, t = b.t_all, L = log(t);
  double loss = 0.0;
  if (b.some) {
#pragma unroll 1
    for (uint32_t k = lane_id(); k < a.K; k += 64) {
      if (b.index[k] < 0 || b.q[k] == 0.0f) continue;
      const double x = b.z[k], lp = t == t && x == -INFINITY ? -INFINITY : (x - m_all) * c - L;
      loss += b.q[k] * (static_cast<double>(b.value[k]) * a.ct - b.lse - lp);
    }
  }
  loss = wave_sum_d(loss);
  const double left = fmax(1.0 - b.sum_q, 0.0);
  if (REST && b.some && o.s != 0.0f && left != 0.0) {
    // what the student leaves over, t being the sum over all: its share's logarithm, but where the share is small that of its parts, which
    // does not underflow
    const double outside = o.s * exp((o.m - m_all) * c) / t;
    const double lp = outside > 0.5 ? log(outside) : (o.m - m_all) * c + log(o.s / t);
    loss += left * (log1p(-b.sum_q) - lp);
  }
  return b.bad || t != t ? NAN : static_cast<float>(loss);
}

// the gradient in an entry's class
__device__ __forceinline__ float taught(const TeacherBox& b, uint32_t k, float g, float cl) {
  if (b.bad || b.t_all != b.t_all) return NAN;
  if (b.t_all == 0.0 || !b.some) return 0.0f;                          // a row that leaves nothing, or teaches nothing
  if (b.sum_q != b.sum_q) return NAN;
  const float p = exp2_((b.z[k] - b.m_all) * cl) / static_cast<float>(b.t_all);
  return g * (p - b.q[k]);
}

// A of Gradient for what the row's sums cover; 0 where nothing is taught, whatever the row's weight
__device__ __forceinline__ float untaught(const TeacherBox& b, float g) { return b.F == 0.0f || b.s == 0.0f ? 0.0f * b.F : g * b.F / b.s; }

__device__ __forceinline__ void distill_outputs(const DistillArgs& a, uint32_t row, const TeacherBox& b, float loss) {
  if (a.loss) a.loss[row] = loss;
  if (a.stats) {
    float* s = a.stats + 8ull * row;
    s[0] = b.m; s[1] = b.s; s[2] = b.F; s[3] = b.m_all; s[4] = static_cast<float>(b.t_all); s[5] = s[6] = s[7] = 0.0f;
  }
}

// A block per row, held in its registers.  REST: what the teacher's entries leave over is one more class.  8,192 rows of 32,000 bf16, 64 entries
// and the rest (1024 x 4) 196 - 199 us, without the rest 194, against 170 of the gradient alone: between the sums and the gradient one wave
// works on the entries, and two rows a compute unit do not hide all of it.  (Loss and entries' gradient before the stores, values read where
// they are needed: 212.)
template <class E, int TH, int NV, bool REST>
__global__ __launch_bounds__(TH) void k_distill_held(DistillArgs a) {
  typedef Held<false, E, TH, NV> H;
  __shared__ Stat box[16];
  __shared__ TeacherBox b;
  __shared__ uint32_t mask[REST ? mask_words(H::SIZE + 8) : 1];
  const float cl = a.c * LOG2E;
  const uint64_t row = block_number();
  if (row >= a.rows) return;
  const E* z = static_cast<const E*>(a.z) + row * a.stride;
  const float g = a.c * (a.g ? a.g[row] : 1.0f);
  Entries<TH> e;
  e.load(a, row);                                                     // first: they come back first
  H h;
  h.load(z, a.vocab);
  E x[entries_of<TH>()];
  teacher_entries<E, TH>(a, z, b, e, x);
  if (REST && !a.stats_in) mark<TH, H::N>(mask, 0, a.vocab, h.first, a.K, [&](uint32_t k) { return b.index[k]; });
  if (threadIdx.x < 64) teacher_probabilities<REST>(a, row, b);       // while the others sum
  Stat o = stat_none();
  if (!a.stats_in) {
    float most[NV / H::U];
    o = h.template stat<false>(cl, [&](uint32_t v) { return REST ? marks<H::N>(mask, v) : 0u; }, most);
  }
  teacher_logits<E, TH>(a, b, x);
  o = block_stat<false, TH>(o, cl, box);
  if (TH == 64) __syncthreads();
  if (threadIdx.x < 64) student_sums<REST>(a, row, o, b);
  __syncthreads();
  E* dz = static_cast<E*>(a.dz) + row * a.dstride;
  if (a.dz) h.template gradient<false>(dz, Gradient{cl, b.m, untaught(b, g), 0.0f}, 0xFFFFFFFFu, 0.0f, [](float) {});
  if (threadIdx.x < 64 && !a.stats_in) {                              // while the stores are on their way
    const float loss = distill_loss<REST>(a, o, b);
    if (threadIdx.x == 0) distill_outputs(a, row, b, loss);
  }
  if (a.dz) {
    __syncthreads();                                                  // the entries' classes are written again
    for (uint32_t k = threadIdx.x; k < a.K; k += TH)
      if (b.index[k] >= 0) dz[b.index[k]] = static_cast<E>(taught(b, k, g, cl));
  }
}

// Rows split into slices: their statistics; what the teacher makes of a row; the gradient, a piece of a row per block.  300 rows of 151,001 fp32,
// 200 entries: 32 + 8 + 57 us; a row of 604 KB fits no block's registers, so it is read twice, the second time in part from the last cache.
template <class E, bool REST>
__global__ __launch_bounds__(256) void k_distill_slices(DistillArgs a, Slices sl) {
  __shared__ Stat box[4];
  extern __shared__ uint32_t mask[];
  const float cl = a.c * LOG2E;
  const uint64_t pieces = static_cast<uint64_t>(a.rows) * sl.S;
  const uint64_t p = block_number();
  if (p >= pieces) return;
  const uint32_t row = static_cast<uint32_t>(p / sl.S), i0 = static_cast<uint32_t>(p % sl.S) * sl.len, n = min(a.vocab - i0, sl.len);
  const E* z = static_cast<const E*>(a.z) + row * a.stride + i0;
  const int32_t* index = a.index + static_cast<uint64_t>(row) * a.K;
  Stat o = REST ? pass_rest<E, 256>(z, i0, n, a.K, cl, mask, [&](uint32_t k) { return index[k]; }) : pass_stat<false, E, 256, false>(z, n, cl);
  o = block_stat<false, 256>(o, cl, box);
  if (threadIdx.x == 0) sl.part[p] = Stat4{o.m, o.s, o.w, 0.0f};
}

struct Taught {                            // what k_distill_join leaves for k_distill_apply
  Stat4* row;                              // [rows] m, A of Gradient
  int32_t* index;                          // [rows, K] classes, -1: none
  float* value;                            // [rows, K] the gradient there
};

template <class E, bool REST>
__global__ __launch_bounds__(256) void k_distill_join(DistillArgs a, Slices sl, Taught w) {
  __shared__ TeacherBox b;
  const float cl = a.c * LOG2E;
  const uint64_t row = block_number();
  if (row >= a.rows) return;
  const float g = a.c * (a.g ? a.g[row] : 1.0f);
  Entries<256> e;
  e.load(a, row);
  E x[1];
  teacher_entries<E, 256>(a, static_cast<const E*>(a.z) + row * a.stride, b, e, x);
  Stat o = stat_none();
  if (threadIdx.x < 64) {
    if (!a.stats_in) o = joined<false>(sl, row, cl);
    teacher_probabilities<REST>(a, row, b);
  }
  teacher_logits<E, 256>(a, b, x);
  __syncthreads();
  if (threadIdx.x < 64) student_sums<REST>(a, row, o, b);
  __syncthreads();
  if (w.row) {
    if (threadIdx.x == 0) w.row[row] = Stat4{b.m, untaught(b, g), 0.0f, 0.0f};
    const uint32_t k = threadIdx.x;
    if (k < a.K) {
      w.index[static_cast<uint64_t>(row) * a.K + k] = b.index[k];
      w.value[static_cast<uint64_t>(row) * a.K + k] = b.index[k] >= 0 ? taught(b, k, g, cl) : 0.0f;
    }
  }
  if (threadIdx.x < 64 && !a.stats_in) {
    const float loss = distill_loss<REST>(a, o, b);
    if (threadIdx.x == 0) distill_outputs(a, row, b, loss);
  }
}

template <class E>
__global__ __launch_bounds__(256) void k_distill_apply(DistillArgs a, Taught w) {
  constexpr int NV = 4;
  typedef Held<true, E, 256, NV> H;
  const uint32_t per = (a.vocab + H::SIZE - 1) / H::SIZE;
  const uint64_t pieces = static_cast<uint64_t>(a.rows) * per;
  const uint64_t p = block_number();
  if (p >= pieces) return;
  const uint32_t row = static_cast<uint32_t>(p / per), i0 = static_cast<uint32_t>(p % per) * H::SIZE, n = min(a.vocab - i0, H::SIZE);
  E* dz = static_cast<E*>(a.dz) + row * a.dstride + i0;
  H h;
  h.load(static_cast<const E*>(a.z) + row * a.stride + i0, n);
  const Stat4 r = w.row[row];
  h.template gradient<false>(dz, Gradient{a.c * LOG2E, r.m, r.s, 0.0f}, 0xFFFFFFFFu, 0.0f, [](float) {});
  __syncthreads();
  const uint32_t k = threadIdx.x;
  if (k < a.K) {
    const int32_t e = w.index[static_cast<uint64_t>(row) * a.K + k];
    const uint32_t i = static_cast<uint32_t>(e) - i0;
    if (e >= 0 && i < n) dz[i] = static_cast<E>(w.value[static_cast<uint64_t>(row) * a.K + k]);
  }
}

}  // namespace
