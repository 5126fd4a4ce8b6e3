// qsl_logits.h -- kernels on the rows of a model's logits: log probabilities of given tokens with the entropy and the top
// alternatives, their gradient, and the loss against a teacher's top logits with its gradient.
//
// Row n with logits z, factor c (`scale`), natural logarithms; m = max z, s = sum exp(c (z_i - m)), L = ln s:
//   logp_i = c (z_i - m) - L        p_i = exp(logp_i)        lse = c m + L        H = -sum p_i logp_i
//   d logp_t / dz_i = c ([i = t] - p_i)                      dH / dz_i = -c p_i (logp_i + H)
// A thread keeps (m, s, w) of the values that it has met, w = sum e_i y_i with y_i = c log2(e) (z_i - m), e_i = exp2(y_i): when m
// grows by a step, y falls by delta = c log2(e) (m_old - m_new), hence s <- s 2^delta, w <- (w + s delta) 2^delta; H = L - ln 2 w / s.
// All of it is held in 32 bits.  m starts at the lowest finite float, so a value of -inf has e = 0 and a row of them s = 0.
// Part of the translation unit logits.hip; not a public header.
#pragma once

#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qsl_device.h"

using namespace qsl;

namespace {

constexpr float LOWEST = -FLT_MAX, LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;
constexpr float Y_MIN = -1e4f;             // exp2 of this is 0; keeps 0 * -inf out of w
constexpr uint32_t TOP_MAX = 128;          // alternatives of a row at most
constexpr uint32_t TEACHER_MAX = 256;      // entries of a teacher's row at most
constexpr uint32_t CAND_CAP = 1024;        // candidates for the alternatives that are ranked at once
constexpr uint32_t GROUPS = 256;           // maxima of groups of threads that the threshold is taken from, at most
constexpr uint32_t HASH_SIZE = 1024;       // slots in which a teacher's entries are looked up: at most a quarter is used
constexpr uint32_t MASK_SPAN = 1u << 18;   // classes whose membership in the teacher's entries is held in LDS at once (32 KB)

// ---------------------------------------------------------------------------------------------
// elements: 16 bytes at a time, aligned to the element only (rows of an odd length start anywhere)
// ---------------------------------------------------------------------------------------------
typedef uint32_t raw_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t raw_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t raw4 __attribute__((ext_vector_type(4)));

template <class E> struct Elem;
template <> struct Elem<float> {
  static constexpr int N = 4;
  static constexpr uint32_t MINUS_INF = 0xFF800000u;
  typedef raw_a4 mem;
  static __device__ __forceinline__ void unpack(raw4 r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
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
  static constexpr uint32_t MINUS_INF = 0xFF80FF80u;
  typedef raw_a2 mem;
  static __device__ __forceinline__ void unpack(raw4 r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r[i] << 16); v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u); }
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
  static constexpr uint32_t MINUS_INF = 0xFC00FC00u;
  typedef raw_a2 mem;
  static __device__ __forceinline__ void unpack(raw4 r, float* v) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) { const h2 x = __builtin_bit_cast(h2, static_cast<uint32_t>(r[i])); v[2 * i] = static_cast<float>(x[0]); v[2 * i + 1] = static_cast<float>(x[1]); }
  }
  static __device__ __forceinline__ raw4 pack(const float* v) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    raw4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) { h2 x = {static_cast<_Float16>(v[2 * i]), static_cast<_Float16>(v[2 * i + 1])}; r[i] = __builtin_bit_cast(uint32_t, x); }
    return r;
  }
};

template <class E> __device__ __forceinline__ raw4 load16(const E* p) { return *reinterpret_cast<const typename Elem<E>::mem*>(p); }
template <class E> __device__ __forceinline__ void store16(E* p, raw4 r) { *reinterpret_cast<typename Elem<E>::mem*>(p) = r; }

// ---------------------------------------------------------------------------------------------
// statistics
// ---------------------------------------------------------------------------------------------
struct Stat { float m, s, w; };

__device__ __forceinline__ Stat stat_none() { return Stat{LOWEST, 0.0f, 0.0f}; }
__device__ __forceinline__ float exp2_(float y) { return __builtin_amdgcn_exp2f(y); }

// takes n values in; -inf adds nothing, NaN and +inf make s NaN
template <bool ENT, int N>
__device__ __forceinline__ void take(Stat& o, const float* v, float cl) {
  float vm = v[0];
#pragma unroll
  for (int i = 1; i < N; ++i) vm = fmaxf(vm, v[i]);
  if (vm > o.m) {
    const float dl = fmaxf((o.m - vm) * cl, Y_MIN), f = exp2_(dl);
    if (ENT) o.w = (o.w + o.s * dl) * f;
    o.s *= f;
    o.m = vm;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = (v[i] - o.m) * cl, e = exp2_(y);
    o.s += e;
    if (ENT) o.w = __builtin_fmaf(e, fmaxf(y, Y_MIN), o.w);
  }
}

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
__device__ __forceinline__ double wave_sum_d(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ double wave_max_d(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = fmax(x, __shfl_xor(x, o, 64));
  return x;
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

// the statistics of all threads of a block of TH, in every thread; `box` holds TH / 64 of them
template <bool ENT, int TH>
__device__ __forceinline__ Stat block_stat(Stat o, float cl, Stat* box) {
  o = wave_stat<ENT>(o, cl);
  if (TH == 64) return o;
  if (lane_id() == 0) box[threadIdx.x >> 6] = o;
  __syncthreads();
  o = lane_id() < TH / 64 ? box[lane_id()] : stat_none();
  return wave_stat<ENT>(o, cl);
}

// what the outputs need of a finished row
struct RowStat { float m, L, H; };
template <bool ENT>
__device__ __forceinline__ RowStat row_stat(Stat o) {
  RowStat r;
  r.m = o.m; r.L = logf(o.s);
  r.H = !ENT ? 0.0f : o.s == 0.0f ? 0.0f : r.L - LN2 * (o.w / o.s);
  return r;
}

// ---------------------------------------------------------------------------------------------
// walking along a row: U loads of 16 bytes of a thread are under way at a time
// ---------------------------------------------------------------------------------------------
// f(first index, N values): vectors that lie wholly in the row; then at most one call for the thread's single value behind them
template <class E, int TH, int U, class F, class G>
__device__ __forceinline__ void walk(const E* z, uint32_t n, F&& whole, G&& single) {
  constexpr int N = Elem<E>::N;
  const uint32_t nvec = n / N;
  for (uint32_t v0 = threadIdx.x; v0 < nvec; v0 += TH * U) {
    raw4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u] = raw4{Elem<E>::MINUS_INF, Elem<E>::MINUS_INF, Elem<E>::MINUS_INF, Elem<E>::MINUS_INF};
      const uint32_t v = v0 + u * TH;
      if (v < nvec) r[u] = load16(z + static_cast<uint64_t>(v) * N);
    }
    whole(v0, r);
  }
  const uint32_t i = nvec * N + threadIdx.x;
  if (i < n) single(i, static_cast<float>(z[i]));
}

template <class E, int TH, bool ENT>
__device__ __forceinline__ Stat pass_stat(const E* z, uint32_t n, float cl) {
  constexpr int N = Elem<E>::N, U = 4;
  Stat o = stat_none();
  walk<E, TH, U>(z, n,
    [&](uint32_t, const raw4* r) {
      float v[U * N];
#pragma unroll
      for (int u = 0; u < U; ++u) Elem<E>::unpack(r[u], v + u * N);
      take<ENT, U * N>(o, v, cl);
    },
    [&](uint32_t, float x) { take<ENT, 1>(o, &x, cl); });
  return o;
}

// ---------------------------------------------------------------------------------------------
// the K largest values of a row, ties to the lower index
// ---------------------------------------------------------------------------------------------
// orders like (value, lower index first); no two entries of a row have the same key, and 0 is none's
__device__ __forceinline__ uint64_t top_key(float z, uint32_t i) {
  const uint32_t u = __float_as_uint(z + 0.0f);                       // -0 counts as +0
  const uint32_t o = u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
  return static_cast<uint64_t>(o) << 32 | (0xFFFFFFFFu - i);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o >> 31 ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xFFFFFFFFu - static_cast<uint32_t>(k); }

struct TopBox {
  uint64_t list[CAND_CAP];
  float group[GROUPS];
  float tau;
  uint32_t n;
  uint64_t kth;
};

// The K largest of a row whose threads have met `most` as their largest value (-inf: none), through out(rank, key).
// Groups of threads hold distinct values, so the K-th largest of the groups' maxima is at most the K-th largest value: only what
// reaches it is a candidate (for values in no particular order a few more than K, in the few threads whose maximum reaches it).  If
// more than CAND_CAP do (many equal or ordered values), the K-th largest of those that found room is the next bound; keys differ,
// so it is a larger one.
template <class E, int TH, class F>
__device__ __forceinline__ void block_top(const E* z, uint32_t n, uint32_t K, float most, TopBox& b, F&& out) {
  constexpr int N = Elem<E>::N, U = 4;
  constexpr uint32_t PER = TH > GROUPS ? TH / GROUPS : 1, G = TH / PER;
  float gm = most;
  if (PER == 4) {
    gm = fmaxf(gm, dpp_keep<0xB1, 0xF>(gm, gm));                      // the lanes of a quad: 1 0 3 2, then 2 3 0 1
    gm = fmaxf(gm, dpp_keep<0x4E, 0xF>(gm, gm));
  }
  if (threadIdx.x % PER == 0) b.group[threadIdx.x / PER] = gm;
  if (threadIdx.x == 0) { b.tau = -INFINITY; b.n = 0; }
  __syncthreads();
  if (K <= G && threadIdx.x < G) {
    const float mine = b.group[threadIdx.x];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < G; ++j) { const float o = b.group[j]; rank += o > mine || (o == mine && j < threadIdx.x); }
    if (rank == K - 1) b.tau = mine;
  }
  __syncthreads();
  const float tau = b.tau;
  uint64_t bound = top_key(tau, 0xFFFFFFFFu);
  for (;;) {
    auto offer = [&](uint32_t i, float x) {
      const uint64_t k = top_key(x, i);
      if (k < bound) return;
      const uint32_t at = atomicAdd(&b.n, 1u);
      if (at < CAND_CAP) b.list[at] = k;
    };
    if (most >= tau)
      walk<E, TH, U>(z, n,
        [&](uint32_t v0, const raw4* r) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const uint32_t i = (v0 + u * TH) * N;
            if (v0 + u * TH >= n / N) continue;
            float v[N];
            Elem<E>::unpack(r[u], v);
#pragma unroll
            for (int q = 0; q < N; ++q) if (v[q] >= tau) offer(i + q, v[q]);
          }
        },
        [&](uint32_t i, float x) { if (x >= tau) offer(i, x); });
    __syncthreads();
    const uint32_t found = b.n, held = min(found, CAND_CAP);
    for (uint32_t i = threadIdx.x; i < held; i += TH) {
      const uint64_t k = b.list[i];
      uint32_t rank = 0;
      for (uint32_t j = 0; j < held; ++j) rank += b.list[j] > k;
      if (found <= CAND_CAP) { if (rank < K) out(rank, k); }
      else if (rank == K - 1) b.kth = k;
    }
    if (found <= CAND_CAP) break;
    __syncthreads();
    bound = b.kth;
    if (threadIdx.x == 0) b.n = 0;
    __syncthreads();
  }
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

__device__ __forceinline__ float log_prob(const RowStat& r, float z, float c) {
  return z == -INFINITY && r.L == r.L ? -INFINITY : (z - r.m) * c - r.L;       // also where the row holds nothing else (L = -inf)
}

template <class E>
__device__ __forceinline__ float target_logprob(const RowStat& r, const E* z, uint32_t vocab, int64_t t, float c) {
  if (t < 0) return 0.0f;
  if (t >= static_cast<int64_t>(vocab)) return NAN;
  return log_prob(r, static_cast<float>(z[t]), c);
}

template <class E, int TH, bool ENT, bool TOP>
__global__ __launch_bounds__(TH) void k_score(ScoreArgs a) {
  __shared__ Stat box[16];
  __shared__ TopBox tb;
  const float cl = a.c * LOG2E;
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* z = static_cast<const E*>(a.z) + row * a.stride;
    const Stat mine = pass_stat<E, TH, ENT>(z, a.vocab, cl);
    const Stat o = block_stat<ENT, TH>(mine, cl, box);
    const RowStat r = row_stat<ENT>(o);
    if (threadIdx.x == 0) {
      if (a.logprob) a.logprob[row] = target_logprob(r, z, a.vocab, a.target[row], a.c);
      if (ENT && a.entropy) a.entropy[row] = r.H;
      if (a.lse) a.lse[row] = o.s == 0.0f ? -INFINITY : r.m * a.c + r.L;
      if (a.stats) { float* s = a.stats + 4ull * row; s[0] = r.m; s[1] = r.L; s[2] = r.H; s[3] = 0.0f; }
    }
    if (TOP) {
      int32_t* ti = a.top_index ? a.top_index + static_cast<uint64_t>(row) * a.K : nullptr;
      float* tl = a.top_logprob ? a.top_logprob + static_cast<uint64_t>(row) * a.K : nullptr;
      if (r.L != r.L) {                                              // a NaN or +inf in the row: no order to speak of
        for (uint32_t k = threadIdx.x; k < a.K; k += TH) { if (ti) ti[k] = -1; if (tl) tl[k] = NAN; }
      } else {
        block_top<E, TH>(z, a.vocab, a.K, mine.s > 0.0f ? mine.m : -INFINITY, tb, [&](uint32_t rank, uint64_t k) {
          if (ti) ti[rank] = static_cast<int32_t>(key_index(k));
          if (tl) tl[rank] = log_prob(r, key_value(k), a.c);
        });
      }
    }
    __syncthreads();                                                  // box and tb are used again
  }
}

// ---------------------------------------------------------------------------------------------
// gradients: dz_i = p_i (A + B y_i) for every class, the given token's or the teacher's classes written again behind a barrier
// ---------------------------------------------------------------------------------------------
template <class E, int TH, bool ENT>
__device__ __forceinline__ void pass_gradient(const E* z, E* dz, uint32_t n, float cl, float m, float l2, float A, float B) {
  constexpr int N = Elem<E>::N, U = 4;
  auto value = [&](float x) {
    const float y = (x - m) * cl, p = exp2_(y - l2);
    return ENT ? p * __builtin_fmaf(B, fmaxf(y, Y_MIN), A) : p * A;
  };
  walk<E, TH, U>(z, n,
    [&](uint32_t v0, const raw4* r) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[N];
        Elem<E>::unpack(r[u], v);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = value(v[q]);
        if (v0 + u * TH < n / N) store16(dz + static_cast<uint64_t>(v0 + u * TH) * N, Elem<E>::pack(v));
      }
    },
    [&](uint32_t i, float x) { dz[i] = static_cast<E>(value(x)); });
}

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

// A block per row: without `stats` it walks along the row twice, the second time mostly through the caches.
template <class E, int TH, bool ENT>
__global__ __launch_bounds__(TH) void k_logprob_gradient(GradArgs a) {
  __shared__ Stat box[16];
  const float cl = a.c * LOG2E;
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* z = static_cast<const E*>(a.z) + row * a.stride;
    E* dz = static_cast<E*>(a.dz) + row * a.dstride;
    const int64_t t = a.target ? a.target[row] : -1;
    const bool given = t >= 0 && t < static_cast<int64_t>(a.vocab);
    const float zt = given ? static_cast<float>(z[t]) : 0.0f;         // before anything is written: dz may be z
    RowStat r;
    if (a.stats) {
      const float* s = a.stats + 4ull * row;
      r.m = s[0]; r.L = s[1]; r.H = s[2];
      __syncthreads();
    } else {
      r = row_stat<ENT>(block_stat<ENT, TH>(pass_stat<E, TH, ENT>(z, a.vocab, cl), cl, box));
      if (threadIdx.x == 0) {
        if (a.logprob) a.logprob[row] = t < 0 ? 0.0f : given ? log_prob(r, zt, a.c) : NAN;
        if (ENT && a.entropy) a.entropy[row] = r.H;
      }
      __syncthreads();
    }
    float g = a.g && t >= 0 ? a.g[row] : 0.0f;
    if (t >= static_cast<int64_t>(a.vocab)) g = NAN;
    const float h = ENT && a.h ? a.h[row] : 0.0f;
    const bool empty = r.L == -INFINITY;
    const float l2 = empty ? 0.0f : r.L * LOG2E;
    const float A = empty ? 0.0f : -a.c * (g + h * (r.H - r.L)), B = -a.c * h * LN2;
    pass_gradient<E, TH, ENT>(z, dz, a.vocab, cl, r.m, l2, A, B);
    __syncthreads();
    if (threadIdx.x == 0 && given && !empty) {
      const float y = (zt - r.m) * cl, p = exp2_(y - l2);
      dz[t] = static_cast<E>(a.c * g + p * __builtin_fmaf(B, fmaxf(y, Y_MIN), A));
    }
  }
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
  float z[TEACHER_MAX];            // the student's logits there
  float q[TEACHER_MAX];            // the teacher's probabilities
  uint32_t bad;
  float m, L, F, m_all, L_all;
};

// The teacher's entries of a row: their classes, the student's logits there; entries that are none, and classes that stood earlier
// in the row, have index -1.  Ends behind a barrier.
template <class E, int TH>
__device__ __forceinline__ void teacher_entries(const DistillArgs& a, uint32_t row, const E* z, TeacherBox& b) {
  for (uint32_t i = threadIdx.x; i < HASH_SIZE; i += TH) { b.key[i] = -1; b.first[i] = 0xFFFFFFFFu; }
  if (threadIdx.x == 0) b.bad = 0;
  __syncthreads();
  constexpr uint32_t M = (TEACHER_MAX + TH - 1) / TH;
  int32_t idx[M];
  uint32_t slot[M];
#pragma unroll
  for (uint32_t j = 0; j < M; ++j) {
    const uint32_t k = threadIdx.x + j * TH;
    idx[j] = -1; slot[j] = 0;
    if (k < a.K) {
      const int32_t i = a.index[static_cast<uint64_t>(row) * a.K + k];
      if (i >= 0 && static_cast<uint32_t>(i) >= a.vocab) b.bad = 1;
      else if (i >= 0) {
        idx[j] = i;
        uint32_t s = (static_cast<uint32_t>(i) * 2654435761u) >> 22;
        for (;;) {                                                    // at most TEACHER_MAX of the HASH_SIZE slots are taken
          const int32_t old = atomicCAS(&b.key[s], -1, i);
          if (old == -1 || old == i) break;
          s = (s + 1) % HASH_SIZE;
        }
        slot[j] = s;
        atomicMin(&b.first[s], k);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t j = 0; j < M; ++j) {
    const uint32_t k = threadIdx.x + j * TH;
    if (k < a.K) {
      const int32_t i = idx[j] >= 0 && b.first[slot[j]] == k ? idx[j] : -1;
      b.index[k] = i;
      b.z[k] = i >= 0 ? static_cast<float>(z[i]) : 0.0f;
    }
  }
  __syncthreads();
}

// The statistics of the row without the teacher's classes: their places are marked in LDS, a span of the row at a time.
template <class E, int TH>
__device__ __forceinline__ Stat pass_rest(const E* z, uint32_t n, uint32_t K, float cl, const TeacherBox& b, uint32_t* mask) {
  constexpr int N = Elem<E>::N, U = 4;
  Stat o = stat_none();
  for (uint32_t s0 = 0; s0 < n; s0 += MASK_SPAN) {
    const uint32_t len = min(n - s0, MASK_SPAN);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < (len + 31) / 32; i += TH) mask[i] = 0;
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < K; k += TH) {
      const uint32_t i = static_cast<uint32_t>(b.index[k]) - s0;      // -1 and classes before the span are huge
      if (b.index[k] >= 0 && i < len) atomicOr(&mask[i / 32], 1u << i % 32);
    }
    __syncthreads();
    walk<E, TH, U>(z + s0, len,
      [&](uint32_t v0, const raw4* r) {
        float v[U * N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          Elem<E>::unpack(r[u], v + u * N);
          const uint32_t i = (v0 + u * TH) * N;
          const uint32_t bits = i < len ? mask[i / 32] >> i % 32 & ((1u << N) - 1) : 0;
          if (bits) {
#pragma unroll
            for (int q = 0; q < N; ++q) if (bits >> q & 1) v[u * N + q] = -INFINITY;
          }
        }
        take<false, U * N>(o, v, cl);
      },
      [&](uint32_t i, float x) { if (!(mask[i / 32] >> i % 32 & 1)) take<false, 1>(o, &x, cl); });
  }
  return o;
}

// By one wave: what the teacher's entries and the row's statistics `o` (of the whole row, or with `rest` of the classes outside)
// make of the row.  In 64 bits: the loss is a difference of logarithms that nearly agree when the student is good, and there are
// only K of them.  Leaves q, m, L, F (dz_i = c g F softmax_i over what `o` covers), m_all, L_all in the box; returns the loss.
__device__ __forceinline__ float teach(const DistillArgs& a, uint32_t row, Stat o, bool from_stats, TeacherBox& b) {
  constexpr int M = TEACHER_MAX / 64;
  const bool rest = a.tlse != nullptr;
  const double c = a.c;
  double u[M], x[M];
  bool has[M];
  double umax = -INFINITY, zmax = -INFINITY;
  bool some = false, nan = false;
#pragma unroll
  for (int j = 0; j < M; ++j) {
    const uint32_t k = lane_id() + 64 * j;
    has[j] = k < a.K && b.index[k] >= 0;
    u[j] = has[j] ? static_cast<double>(a.value[static_cast<uint64_t>(row) * a.K + k]) * a.ct : -INFINITY;
    x[j] = has[j] ? static_cast<double>(b.z[k]) : -INFINITY;
    umax = fmax(umax, u[j]);
    zmax = fmax(zmax, x[j]);
    some |= has[j];
    nan |= u[j] != u[j];
  }
  some = __any(some);
  // the teacher's probabilities; without any mass (no entries, or all of them -inf) the row teaches nothing
  double lse_t = 0.0;
  if (rest) lse_t = a.tlse[row];
  else {
    umax = wave_max_d(umax);
    some = some && (umax > -INFINITY || __any(nan));
    double t = 0.0;
#pragma unroll
    for (int j = 0; j < M; ++j) if (has[j] && some) t += exp(u[j] - umax);
    t = wave_sum_d(t);
    lse_t = some ? umax + log(t) : 0.0;
  }
  double m_all, L_all, m_o = o.m, L_o = log(static_cast<double>(o.s));
  if (from_stats) {
    const float* s = a.stats_in + 8ull * row;
    m_o = s[0]; L_o = s[1]; m_all = s[3]; L_all = s[4];
  } else if (!rest) {
    m_all = m_o; L_all = L_o;
  } else {
    zmax = wave_max_d(zmax);
    m_all = fmax(zmax, m_o);
    double t = 0.0;
#pragma unroll
    for (int j = 0; j < M; ++j) if (has[j]) t += exp((x[j] - m_all) * c);
    t = wave_sum_d(t) + (o.s == 0.0f ? 0.0 : o.s * exp((m_o - m_all) * c));
    L_all = log(t);
  }
  const bool empty = L_all == -INFINITY;
  double loss = 0.0, sum_q = 0.0, sum_p = 0.0;
#pragma unroll
  for (int j = 0; j < M; ++j) {
    if (!has[j]) continue;
    const double lq = u[j] - lse_t, q = some ? exp(lq) : 0.0;
    const double lp = empty || x[j] == -INFINITY ? (L_all == L_all ? -INFINITY : NAN) : (x[j] - m_all) * c - L_all;
    if (!(q == 0.0)) loss += q * (lq - lp);
    sum_q += q;
    sum_p += exp(lp);
    b.q[lane_id() + 64 * j] = static_cast<float>(q);
  }
  double F = some ? 1.0 : 0.0;
  if (rest && !from_stats) {
    sum_q = wave_sum_d(sum_q); sum_p = wave_sum_d(sum_p);
    const double left = fmax(1.0 - sum_q, 0.0);
    F = 0.0;
    if (L_o != -INFINITY) {                                           // nothing outside: the rest is left out
      // the student's rest: from what is inside where that is the smaller part
      const double lp = sum_p < 0.5 ? log1p(-sum_p) : (m_o - m_all) * c + L_o - L_all;
      if (!(left == 0.0) && lane_id() == 0) loss += left * (log1p(-sum_q) - lp);
      F = exp(lp) - left;
      if (sum_q != sum_q) F = NAN;
    }
  }
  loss = wave_sum_d(loss);
  if (!from_stats && !rest && !some) loss = 0.0;
  if (b.bad) { loss = NAN; F = NAN; }
  if (lane_id() == 0) {
    b.m = static_cast<float>(m_o); b.L = static_cast<float>(L_o);
    b.m_all = static_cast<float>(m_all); b.L_all = static_cast<float>(L_all);
    b.F = from_stats ? a.stats_in[8ull * row + 2] : static_cast<float>(F);
    if (empty) { b.F = b.bad ? NAN : 0.0f; }
  }
  return static_cast<float>(loss);
}

// GRAD: the gradient too.  REST: what the teacher's entries leave over is one more class.
template <class E, int TH, bool REST, bool GRAD>
__global__ __launch_bounds__(TH) void k_distill(DistillArgs a) {
  __shared__ Stat box[16];
  __shared__ TeacherBox b;
  extern __shared__ uint32_t mask[];
  const float cl = a.c * LOG2E;
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* z = static_cast<const E*>(a.z) + row * a.stride;
    teacher_entries<E, TH>(a, row, z, b);
    Stat o = stat_none();
    const bool from_stats = GRAD && a.stats_in;
    if (!from_stats) {
      o = REST ? pass_rest<E, TH>(z, a.vocab, a.K, cl, b, mask) : pass_stat<E, TH, false>(z, a.vocab, cl);
      o = block_stat<false, TH>(o, cl, box);
    }
    if (threadIdx.x < 64) {
      const float loss = teach(a, row, o, from_stats, b);
      if (threadIdx.x == 0) {
        if (a.loss) a.loss[row] = loss;
        if (!GRAD && a.stats) {
          float* s = a.stats + 8ull * row;
          s[0] = b.m; s[1] = b.L; s[2] = b.F; s[3] = b.m_all; s[4] = b.L_all; s[5] = s[6] = s[7] = 0.0f;
        }
      }
    }
    __syncthreads();
    if (GRAD) {
      E* dz = static_cast<E*>(a.dz) + row * a.dstride;
      const float g = a.c * (a.g ? a.g[row] : 1.0f), L = b.L, L_all = b.L_all, m_all = b.m_all, F = b.F;
      pass_gradient<E, TH, false>(z, dz, a.vocab, cl, b.m, L == -INFINITY ? 0.0f : L * LOG2E, g * F, 0.0f);
      __syncthreads();
      for (uint32_t k = threadIdx.x; k < a.K; k += TH) {
        const int32_t i = b.index[k];
        if (i < 0) continue;
        const float p = L_all == -INFINITY ? 0.0f : expf((b.z[k] - m_all) * a.c - L_all), q = b.q[k];
        const bool none = L_all == -INFINITY || (!REST && F == 0.0f);
        dz[i] = static_cast<E>(b.bad ? NAN : none ? 0.0f : g * (p - q));
      }
    }
    __syncthreads();
  }
}

}  // namespace
