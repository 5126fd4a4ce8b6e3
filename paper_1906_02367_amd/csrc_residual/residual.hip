// residual.hip -- host side and C ABI of the operators on a layer's residual stream (include/qsl.h); their kernels are in qsl_residual.h.
//
// The calls keep no state: arguments are checked, one rule on the row's length picks the launch, the kernels go to the caller's stream.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "qsl.h"
#include "qsl_memory.h"
#include "qsl_residual.h"

namespace {

constexpr uint64_t CACHE_BYTES = 256ull << 20;     // the last cache before the memory
constexpr uint64_t GRID_X = 1u << 20;              // blocks in a row of the grid (a launch counts its threads in 32 bits)

uint32_t elem_size(uint32_t dtype) { return dtype == QSL_F32 ? 4 : dtype <= QSL_F16 ? 2 : 1; }

bool rows_ok(const qsl_rows& m, uint64_t rows, uint64_t cols, uint32_t dtype) {
  return !m.data || (stride_ok(rows, cols, m.stride) && aligned(m.data, elem_size(dtype)));
}
bool same(const qsl_rows& a, const qsl_rows& b, uint64_t rows) { return a.data == b.data && (a.stride == b.stride || rows == 1); }

bool drop_ok(const qsl_drop& d, uint64_t rows) {
  return d.p == 0.0 || (d.p > 0.0 && d.p <= 1.0 && d.round < 1ull << 62 && aligned(d.round_at, 8) && d.row0 + rows <= 1ull << 32);
}
Drop drop_of(const qsl_drop& d) {
  const uint32_t T = static_cast<uint32_t>(floor((1.0 - d.p) * 65536.0 + 0.5));
  return Drop{T, T ? static_cast<float>(65536.0 / T) : 0.0f, d.row0, static_cast<uint32_t>(d.seed), static_cast<uint32_t>(d.seed >> 32), d.round, d.round_at};
}
Memory round_of(const qsl_drop& d) { return array(d.p > 0.0 ? d.round_at : nullptr, 8); }

// f(the element type) as a type
template <class F>
void pick_type(uint32_t dtype, F&& f) {
  if (dtype == QSL_F32) f(float());
  else if (dtype == QSL_BF16) f(__bf16());
  else f(_Float16());
}
// f(whether what is read and written goes past the caches).  From what they hold written on: every call reads half as much beside it at least, so that its
// arrays together are more than that.
template <class F>
void pick_past(uint64_t written, F&& f) {
  if (written >= CACHE_BYTES) f(std::true_type());
  else f(std::false_type());
}
// What the norm writes may do so in rows of up to 32 KiB, in 8 bits of up to 8,192 columns (a lane with longer ones waits at its stores).  us through the
// caches / past them, whole and in 8 bits: bf16 16,384 rows of 8,192 180 / 175 and 161 / 158.5, 8,192 of 16,384 186 / 175 and 164 / 179, 3,000 of 32,768
// 151 / 166 and 158 / 185; fp32 8,192 of 8,192 188 / 176 and 158 / 150, 4,096 of 16,384 192 / 206 and 170 / 169.
template <class E, int L, int U, bool BITS8>
constexpr bool NORM_MAY_PASS = L * U * 16 <= 32768 && (!BITS8 || L * U * COLS<E> <= 8192);
template <int V> using Int = std::integral_constant<int, V>;

// f(lanes that hold a row, units each of them holds).  us, residual added, total and y written, through the caches, bf16 / fp32 (of which an array's unit is
// four columns: twice the lanes or units):
//   131,072 rows of 128    bf16 16 x 1 26, 64 x 1 48;                   fp32 16 x 2 47.6, 64 x 1 48.7
//   32,768 rows of 512     bf16 64 x 1 25, 128 x 1 27, 256 x 1 42;      fp32 64 x 2 48.5, 128 x 1 47.5, 256 x 1 49
//   30,000 rows of 1,024   bf16 64 x 2 44.5, 128 x 1 44, 256 x 1 47;    fp32 64 x 4 88, 128 x 2 85.6, 256 x 1 84, 512 x 1 84.6
//   30,000 rows of 785     bf16 64 x 2 38, 128 x 1 46;                  fp32 64 x 4 75, 128 x 2 71, 256 x 1 68, 256 x 2 74
//   16,384 rows of 2,048   bf16 128 x 2 46.5, 256 x 1 49, 512 x 1 51;   fp32 128 x 4 94, 256 x 2 92, 512 x 1 91.5, 1024 x 1 89 (with a mask 96)
//   16,384 rows of 4,096   bf16 256 x 2 91, 512 x 1 91.5, 1024 x 1 101; fp32 256 x 4 183, 512 x 2 184, 1024 x 1 179 (y alone 109, by 512 x 2 91)
//   8,192 rows of 8,192    bf16 512 x 2 91.5, 1024 x 1 92;              fp32 512 x 4 189, 1024 x 2 189
//   4,096 rows of 16,384   bf16 512 x 4 98.5, 1024 x 2 99;              fp32 1024 x 4 191, 1024 x 8 196
// So two units a lane, from 64 lanes to 1024, then more; short rows take eight columns a lane.
template <class E, class F>
void pick_row(uint32_t cols, F&& f) {
  constexpr uint32_t N = COLS<E>, K = 8 / N;      // K units: eight columns
  if (cols <= 16 * 8) f(Int<16>(), Int<K>());
  else if (cols <= 64 * 8) f(Int<64>(), Int<K>());
  else if (cols <= 64 * 2 * N) f(Int<64>(), Int<2>());
  else if (cols <= 128 * 2 * N) f(Int<128>(), Int<2>());
  else if (cols <= 256 * 2 * N) f(Int<256>(), Int<2>());
  else if (cols <= 512 * 2 * N) f(Int<512>(), Int<2>());
  else if (cols <= 1024 * 2 * N) f(Int<1024>(), Int<2>());
  else if (cols <= 1024 * 16) f(Int<1024>(), Int<2 * K>());
  else f(Int<1024>(), Int<4 * K>());
}
// The gradient's, which holds three arrays and the sum for dweight.  us with all of them, a mask and k_sum_parts, through the caches, with 1, 2, 3, 4 waves on
// a SIMD unit (1024 lanes: 4):
//   131,072 rows of 128    bf16 16 x 1 44, 36, 37, 39;                               fp32 16 x 2 98, 69, 66, 68
//   32,768 rows of 512     bf16 64 x 1 44, 37, 37, 39;                               fp32 64 x 2 69, 67, 67, 70
//   30,000 rows of 785     bf16 64 x 2 78, 56, 54, 62;  128 x 1 -, 75, 65;           fp32 64 x 4 103, 98, 108, 101;  256 x 1 157, 102, 97, 101
//   120 rows of 785                                                                  fp32 64 x 4 7.9;  256 x 1 6.6 (but up to 8 rows one launch, not two)
//   16,384 rows of 2,048   bf16 256 x 1 84, 65, 69, 71;  128 x 2 -, 69;              fp32 512 x 1 -, 122, -, 130;  256 x 2 136, 131, 132, 134
//   16,384 rows of 4,096   bf16 512 x 1 -, 121, -, 132;  256 x 2 -, 133, 135;        fp32 512 x 2 -, 247, -, 250;  1024 x 1 248
//   8,192 rows of 8,192    bf16 512 x 2 -, 128, -, 131;  1024 x 1 131;               fp32 512 x 4 -, 246, -, 250;  1024 x 2 243
//   4,096 rows of 16,384   bf16 1024 x 2 130;  512 x 4 -, 132;                       fp32 1024 x 4 263;  1024 x 8 407
//   2,048 rows of 32,768   bf16 1024 x 4 150;                                        fp32 1024 x 8 275
template <class E, class F>
void pick_row_back(uint32_t cols, F&& f) {
  constexpr uint32_t K = 8 / COLS<E>;
  if (cols <= 16 * 8) f(Int<16>(), Int<K>());
  else if (cols <= 64 * 8) f(Int<64>(), Int<K>());
  else if (cols <= 64 * 16) f(Int<64>(), Int<2 * K>());
  else if (cols <= 256 * 8) f(Int<256 * K>(), Int<1>());
  else if (cols <= 512 * 8) f(Int<512>(), Int<K>());
  else if (cols <= 512 * 16) f(Int<512 * K>(), Int<2>());
  else if (cols <= 1024 * 16) f(Int<1024>(), Int<2 * K>());
  else f(Int<1024>(), Int<4 * K>());
}

dim3 grid_of(uint64_t blocks) {
  return dim3(static_cast<uint32_t>(std::min(blocks, GRID_X)), static_cast<uint32_t>((blocks + GRID_X - 1) / GRID_X));
}

bool norm_ok(const qsl_norm* n) {
  if (!n || n->dtype > QSL_F16 || n->rows >= 1u << 31 || n->cols == 0 || n->cols > QSL_NORM_COLS_MAX) return false;
  if (n->weight && ((n->weight_dtype != n->dtype && n->weight_dtype != QSL_F32) || !aligned(n->weight, elem_size(n->weight_dtype)))) return false;
  return n->eps >= 0x1p-100f && n->eps <= 0x1p100f;
}
Memory weight_of(const qsl_norm* n) { return array(n->weight, static_cast<uint64_t>(n->cols) * elem_size(n->weight_dtype)); }

// Blocks of the backward pass: each goes through many rows, so that their sums for dweight are few.  Two rows (or two for each group of threads) are
// left to one block, whose sum is dweight: they take 1 to 2 us in it, another launch takes the host 4.
uint32_t back_blocks(const qsl_norm* n) {
  uint32_t blocks = 0;
  pick_type(n->dtype, [&](auto e) {
    pick_row_back<decltype(e)>(n->cols, [&](auto l, auto) {
      const uint64_t th = THREADS<l()>, per = th / l(), most = th == 256 ? 512 : 256;
      blocks = n->rows <= 2 * per ? (n->rows != 0) : static_cast<uint32_t>(std::min<uint64_t>((n->rows + per - 1) / per, most));
    });
  });
  return blocks;
}

// Launches kernel(args...).  (<<<...>>> takes the host 0.43 us more: it hands the launch's shape over by two calls of its own.)
template <class... A>
void launch(void (*kernel)(A...), dim3 grid, uint32_t threads, hipStream_t stream, std::common_type_t<A>... args) {
  void* at[] = {&args...};
  (void)hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, stream);      // what fails is the last error
}

// Narrow sums by blocks of 16 columns, of which there are more; wide ones by 32, whole lines of the caches, which else two compute dies read.  us behind a
// kernel that writes them, 16 / 32 columns: 768 blocks of 1,024 3.4 / 4.7, of 2,048 6.0 / 5.6, 512 of 4,096 7.1 / 5.7, 256 of 12,289 13.1 / 10.3
void sum_parts(const float* part, uint32_t blocks, uint32_t cols, float* dweight, hipStream_t stream) {
  if (cols <= 1024) launch(k_sum_parts<16, 64>, dim3((cols + 15) / 16), 1024, stream, part, blocks, cols, dweight);
  else launch(k_sum_parts<32, 32>, dim3((cols + 31) / 32), 1024, stream, part, blocks, cols, dweight);
}

qsl_status launched() { return hipGetLastError() == hipSuccess ? QSL_OK : QSL_ERR_DEVICE; }

}  // namespace

extern "C" qsl_status qsl_dropout(const qsl_dropout_args* args, void* hip_stream) {
  if (!args) return QSL_ERR_INVALID_ARG;
  const qsl_rows &x = args->x, &res = args->residual, &y = args->y;
  const uint64_t rows = args->rows, cols = args->cols, es = elem_size(args->dtype);
  if (args->dtype > QSL_F16 || rows >= 1u << 31 || cols == 0 || cols >= 1u << 31 || !drop_ok(args->drop, rows)) return QSL_ERR_INVALID_ARG;
  if (rows == 0) return QSL_OK;
  if (!x.data || !y.data) return QSL_ERR_INVALID_ARG;
  for (const qsl_rows* m : {&x, &res, &y}) if (!rows_ok(*m, rows, cols, args->dtype)) return QSL_ERR_INVALID_ARG;
  auto at = [&](const qsl_rows& m) { return rows_at(m.data, rows, cols, m.stride, es); };
  for (const qsl_rows* m : {&x, &res}) if (m->data && !same(*m, y, rows) && meet(at(*m), at(y))) return QSL_ERR_INVALID_ARG;
  if (meet(round_of(args->drop), at(y))) return QSL_ERR_INVALID_ARG;
  const uint32_t units = static_cast<uint32_t>((cols * es + 15) / 16);
  const DropArgs a = {x.data, res.data, y.data, x.stride, res.stride, y.stride, rows, args->cols, units, drop_of(args->drop)};
  const uint64_t blocks = (rows * units + DROP_THREADS - 1) / DROP_THREADS;
  pick_type(args->dtype, [&](auto e) {
    typedef decltype(e) E;
    pick_past(rows * cols * es, [&](auto past) { launch(k_dropout<E, past()>, grid_of(blocks), DROP_THREADS, static_cast<hipStream_t>(hip_stream), a); });
  });
  return launched();
}

extern "C" qsl_status qsl_rms_norm(const qsl_rms_norm_args* args, void* hip_stream) {
  if (!args || !norm_ok(&args->norm)) return QSL_ERR_INVALID_ARG;
  const qsl_norm* norm = &args->norm;
  const qsl_rows &x = args->x, &res = args->residual, &total = args->total, &y = args->y;
  const uint64_t rows = norm->rows, cols = norm->cols, es = elem_size(norm->dtype);
  const uint32_t out_dtype = args->out_dtype, group = args->group;
  const bool bits8 = out_dtype == QSL_E4M3 || out_dtype == QSL_I8;
  if (!drop_ok(args->drop, rows) || (!bits8 && out_dtype != norm->dtype)) return QSL_ERR_INVALID_ARG;
  if (bits8 ? group != 0 && group != 32 && group != 64 && group != 128 : group != 0 || args->scales) return QSL_ERR_INVALID_ARG;
  if (rows == 0) return QSL_OK;
  if (!x.data || !y.data || (bits8 && (!args->scales || !aligned(args->scales, 4)))) return QSL_ERR_INVALID_ARG;
  for (const qsl_rows* m : {&x, &res, &total}) if (!rows_ok(*m, rows, cols, norm->dtype)) return QSL_ERR_INVALID_ARG;
  if (!rows_ok(y, rows, cols, out_dtype)) return QSL_ERR_INVALID_ARG;
  auto at = [&](const qsl_rows& m, uint64_t size) { return rows_at(m.data, rows, cols, m.stride, size); };
  const Memory out_t = at(total, es), out_y = at(y, elem_size(out_dtype)), out_s = array(args->scales, 4 * rows * (group ? (cols + group - 1) / group : 1));
  if (!apart({out_t, out_y, out_s}, {weight_of(norm), round_of(args->drop)})) return QSL_ERR_INVALID_ARG;
  for (const qsl_rows* m : {&x, &res}) {      // a thread reads x and the residual where it writes the total and y, all of the row before any of it
    if (!m->data) continue;
    const Memory in = at(*m, es);
    if (!same(*m, total, rows) && meet(in, out_t)) return QSL_ERR_INVALID_ARG;
    if ((bits8 || !same(*m, y, rows)) && meet(in, out_y)) return QSL_ERR_INVALID_ARG;
    if (meet(in, out_s)) return QSL_ERR_INVALID_ARG;
  }
  // a group that holds the row is the row: so no group has more than the 16 lanes of a short one
  const uint32_t group_bits = group && group < cols ? 31u - __builtin_clz(group) : 0u;
  const NormArgs a = {x.data, res.data, norm->weight, total.data, y.data, args->scales, x.stride, res.stride, total.stride, y.stride, rows, norm->cols,
                      norm->weight_dtype == QSL_F32, out_dtype == QSL_E4M3, group_bits, norm->eps, drop_of(args->drop)};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const uint64_t written = rows * cols * ((total.data ? es : 0) + elem_size(out_dtype));
  pick_type(norm->dtype, [&](auto e) {
    typedef decltype(e) E;
    pick_row<E>(norm->cols, [&](auto l, auto u) {
      constexpr int th = THREADS<l()>, per = th / l();
      const dim3 grid = grid_of((rows + per - 1) / per);
      auto norm_of = [&](auto b8) {
        if constexpr (NORM_MAY_PASS<E, l(), u(), b8()>) pick_past(written, [&](auto past) { launch(k_rms_norm<E, l(), u(), b8(), past()>, grid, th, stream, a); });
        else launch(k_rms_norm<E, l(), u(), b8(), false>, grid, th, stream, a);
      };
      if (bits8) norm_of(std::true_type());
      else norm_of(std::false_type());
    });
  });
  return launched();
}

extern "C" size_t qsl_rms_norm_workspace_bytes(const qsl_norm* norm) {
  const uint64_t blocks = norm_ok(norm) ? back_blocks(norm) : 0;
  return blocks > 1 ? align_up(4 * blocks * norm->cols, 256) : 0;
}

extern "C" qsl_status qsl_rms_norm_backward(const qsl_rms_norm_backward_args* args, void* hip_stream) {
  if (!args || !norm_ok(&args->norm) || !drop_ok(args->drop, args->norm.rows) || !aligned(args->dweight, 4)) return QSL_ERR_INVALID_ARG;
  const qsl_norm* norm = &args->norm;
  const qsl_rows &total = args->total, &dy = args->dy, &dtotal = args->dtotal, &dres = args->dresidual, &dx = args->dx;
  const uint64_t rows = norm->rows, cols = norm->cols, es = elem_size(norm->dtype);
  float* const dweight = args->dweight;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const uint32_t blocks = back_blocks(norm);
  const bool parts_apart = dweight && blocks > 1;
  if (rows != 0) {
    if (!total.data || !dy.data || (!dres.data && !dx.data && !dweight)) return QSL_ERR_INVALID_ARG;
    for (const qsl_rows* m : {&total, &dy, &dtotal, &dres, &dx}) if (!rows_ok(*m, rows, cols, norm->dtype)) return QSL_ERR_INVALID_ARG;
    if (parts_apart && (!args->workspace || !aligned(args->workspace, 256))) return QSL_ERR_INVALID_ARG;
    if (parts_apart && args->workspace_bytes < qsl_rms_norm_workspace_bytes(norm)) return QSL_ERR_BUFFER_TOO_SMALL;
    auto at = [&](const qsl_rows& m) { return rows_at(m.data, rows, cols, m.stride, es); };
    const Memory dw = array(dweight, 4 * cols), parts = array(args->workspace, parts_apart ? 4 * blocks * cols : 0);
    if (!apart({at(dres), at(dx), dw, parts}, {weight_of(norm), round_of(args->drop)})) return QSL_ERR_INVALID_ARG;
    for (const qsl_rows* m : {&total, &dy, &dtotal}) {
      if (!m->data) continue;
      for (const qsl_rows* o : {&dres, &dx}) if (o->data && !same(*m, *o, rows) && meet(at(*m), at(*o))) return QSL_ERR_INVALID_ARG;
      if (meet(at(*m), dw) || meet(at(*m), parts)) return QSL_ERR_INVALID_ARG;
    }
    const BackArgs a = {total.data, dy.data, dtotal.data, norm->weight, dres.data, dx.data, parts_apart ? static_cast<float*>(args->workspace) : dweight,
                        total.stride, dy.stride, dtotal.stride, dres.stride, dx.stride, rows, norm->cols, norm->weight_dtype == QSL_F32, norm->eps,
                        drop_of(args->drop)};
    pick_type(norm->dtype, [&](auto e) {
      typedef decltype(e) E;
      pick_row_back<E>(norm->cols, [&](auto l, auto u) {
        pick_past(rows * cols * es * ((dres.data != nullptr) + (dx.data != nullptr)), [&](auto past) {
          launch(k_rms_norm_backward<E, l(), u(), past()>, dim3(blocks), THREADS<l()>, stream, a);
        });
      });
    });
  }
  if (parts_apart || (dweight && rows == 0)) sum_parts(static_cast<const float*>(args->workspace), blocks, norm->cols, dweight, stream);
  return rows || dweight ? launched() : QSL_OK;
}
