// logits.hip -- host side and C ABI of the operators on a model's logits (include/qsl.h); their kernels are in qsl_logits.h.
//
// The calls keep no state: arguments are checked, one rule on sizes picks the launch, the kernels go to the caller's stream.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "qsl.h"
#include "qsl_logits.h"
#include "qsl_memory.h"

static_assert(TOP_MAX == QSL_TOP_MAX && TEACHER_MAX == QSL_TEACHER_MAX, "the header's limits");
static_assert(REFINE >= 2 * TOP_MAX && CAND_CAP >= REFINE, "a bound from the first candidates must leave some of them out");

namespace {

constexpr uint64_t GRID_X = 1u << 20;              // blocks in a row of the grid (a launch counts its threads in 32 bits)
constexpr uint32_t FEW_ROWS = 256;                 // fewer rows than this leave compute units without a block
constexpr uint32_t WANTED_BLOCKS = 1024;           // blocks of 256 threads that keep the chip busy
constexpr uint64_t CACHE_BYTES = 256ull << 20;     // the last cache before the memory
constexpr uint64_t MIN_SLICE = 4096;               // bytes: 16 a thread

bool scale_ok(float c) { return c >= 0x1p-100f && c <= 0x1p100f; }
uint32_t elem_size(uint32_t dtype) { return dtype == QSL_F32 ? 4 : 2; }

bool stride_ok(const qsl_logits* z, uint64_t stride) { return stride_ok(z->rows, z->vocab, stride); }

bool logits_ok(const qsl_logits* z) {
  if (!z || z->dtype > QSL_F16 || z->vocab == 0 || z->vocab >= 1u << 31 || z->rows >= 1u << 31) return false;
  if (!stride_ok(z, z->stride) || !scale_ok(z->scale)) return false;
  return z->rows == 0 || (z->data && aligned(z->data, elem_size(z->dtype)));
}

Memory rows_at(const qsl_logits* z, const void* p, uint64_t stride) { return rows_at(p, z->rows, z->vocab, stride, elem_size(z->dtype)); }

// dlogits are the logits, or share no element with them
bool gradient_ok(const qsl_logits* z, const void* dz, uint64_t dstride) {
  const uint64_t es = elem_size(z->dtype);
  if (!stride_ok(z, dstride) || !aligned(dz, es)) return false;
  if (z->rows == 0) return true;
  if (!dz) return false;
  if (dz == z->data && (dstride == z->stride || z->rows == 1)) return true;
  return !meet(rows_at(z, z->data, z->stride), rows_at(z, dz, dstride));
}

bool teacher_ok(const qsl_logits* z, const qsl_teacher* t) {
  if (!t || t->top == 0 || t->top > QSL_TEACHER_MAX || !scale_ok(t->scale)) return false;
  if (z->rows == 0) return true;
  return t->index && t->value && aligned(t->index, 4) && aligned(t->value, 4) && aligned(t->lse, 4);
}

// f(the element type) as a type
template <class F>
void pick_type(const qsl_logits* z, F&& f) {
  if (z->dtype == QSL_F32) f(float());
  else if (z->dtype == QSL_BF16) f(__bf16());
  else f(_Float16());
}
template <class F>
void pick_bool(bool b, F&& f) {
  if (b) f(std::true_type());
  else f(std::false_type());
}
template <int V> using Int = std::integral_constant<int, V>;

constexpr uint64_t KB = 1024;
constexpr uint64_t HELD_MAX = 256 * KB;            // bytes of a row that 1024 threads hold in registers, 16 vectors each
constexpr uint64_t HELD_TOP_MAX = 128 * KB;        // ... from which alternatives are taken
constexpr uint64_t SLICE_MAX = 64 * KB;            // ... that 256 threads hold

uint64_t row_bytes(const qsl_logits* z) { return static_cast<uint64_t>(z->vocab) * elem_size(z->dtype); }

// f(threads, vectors a thread holds) for rows that a block holds (and the values before and behind their vectors).  Where a row can be
// held by few threads with many vectors or by many with few: many have the shorter way from the first load to the last store, few
// leave room for other rows while a row is being ranked; few rows have nothing to make room for.  us:
//   8,192 rows of 64 KB   gradient 256 x 16 198, 512 x 8 193, 1024 x 4 178
//   4,096 rows of 64 KB   20 alternatives 256 x 16 50, 512 x 8 53, 1024 x 4 70
//   8,192 rows of 32 KB   gradient 256 x 8 100, 512 x 4 95; entries 111 / 107; 20 alternatives 128 x 16 53, 256 x 8 54, 512 x 4 67
//   16 KB                 gradient (16,384 rows) 256 x 4 97, 128 x 8 100; 20 alternatives (8,192) 36 / 31
//   128 KB                gradient (4,000) 512 x 16 188, 1024 x 8 190, with the entropy 193 / 197; entries (2,000) 113 / 149; 20 alternatives
//                         (4,096) 99 / 148
template <class F>
void pick_for_gradient(uint64_t nvec, uint64_t rows, F&& f) {
  if (nvec <= 64) f(Int<64>(), Int<1>());
  else if (nvec <= 64 * 4) f(Int<64>(), Int<4>());
  else if (nvec <= 256 * 4) f(Int<256>(), Int<4>());
  else if (nvec <= 512 * 4) f(Int<512>(), Int<4>());
  else if (nvec <= 1024 * 4) f(Int<1024>(), Int<4>());
  else if (nvec <= 512 * 16 && rows >= FEW_ROWS) f(Int<512>(), Int<16>());
  else if (nvec <= 1024 * 8) f(Int<1024>(), Int<8>());
  else f(Int<1024>(), Int<16>());
}
// for a teacher's entries.  Summing 16-bit values without the entries' takes the most operations a vector: rows that leave a quarter of 1024 x 4
// empty go to 512 x 8, of which more are resident.  us, 8,192 rows of bf16, 1024 x 4 / 512 x 8: the rest as one class 17,000 155 / 124, 20,000
// 159 / 136, 24,000 167 / 153, 28,000 181 / 186, 32,000 198 / 210; the entries alone 20,000 133 / 138; fp32 of 10,000 125 / 138
template <bool REST16, class F>
void pick_for_teacher(uint64_t nvec, uint64_t rows, F&& f) {
  if constexpr (REST16) {
    if (nvec > 512 * 4 && nvec * 16 <= 48 * KB) { f(Int<512>(), Int<8>()); return; }
  }
  pick_for_gradient(nvec, rows, f);
}
// for alternatives, whose bound comes from the maxima of groups of threads, of which there have to be more than alternatives (a wave of 64 and
// 64 alternatives: 12,000 rows of 1,500 103 us, 128 x 8 37), or from all values of a wave
template <class F>
void pick_for_top(uint64_t nvec, uint64_t rows, uint32_t top, F&& f) {
  const bool few = rows < FEW_ROWS;
  if (nvec <= 64) f(Int<64>(), Int<1>());
  else if (nvec <= 64 * 4 && (top <= 32 || maxima_say_little(top, nvec))) f(Int<64>(), Int<4>());
  else if (nvec <= 128 * 8 && top <= 64 && !few) f(Int<128>(), Int<8>());
  else if (nvec <= 256 * 4) f(Int<256>(), Int<4>());
  else if (nvec <= 256 * 8 && !few) f(Int<256>(), Int<8>());
  else if (nvec <= 256 * 16 && !few) f(Int<256>(), Int<16>());
  else if (nvec <= 1024 * 4) f(Int<1024>(), Int<4>());
  else if (!few) f(Int<512>(), Int<16>());
  else f(Int<1024>(), Int<8>());
}

// How a call splits its rows.
struct Plan {
  bool split;
  uint32_t S, len;
};

Plan plan_slices(const qsl_logits* z, uint64_t least = MIN_SLICE) {
  const uint64_t bytes = row_bytes(z), es = elem_size(z->dtype);
  uint64_t S = std::max<uint64_t>((bytes + SLICE_MAX - 1) / SLICE_MAX, WANTED_BLOCKS / std::max(z->rows, 1u));
  S = std::min<uint64_t>({S, SLICES_MAX, (bytes + least - 1) / least});
  Plan p;
  p.split = true;
  // whole 4 KB: slices start where vectors do, and their threads are busy alike
  p.len = static_cast<uint32_t>(align_up((z->vocab + S - 1) / S, 4 * KB / es));
  p.S = (z->vocab + p.len - 1) / p.len;
  return p;
}

constexpr Plan WHOLE = {false, 0, 0};

// Alternatives: rows of up to 128 KB by one block each, longer ones in slices (rows of more than 64 slices are walked along).  us, a block of
// 1024 x 16 / slices: 2,048 rows of 200 KB, 64 alternatives 111 / 95; 2,048 of 256 KB, 20 alternatives 122 / 96; 64 of 256 KB 16 / 15.
Plan plan_top(const qsl_logits* z) {
  const uint64_t bytes = row_bytes(z);
  return bytes <= HELD_TOP_MAX || bytes > SLICES_MAX * SLICE_MAX ? WHOLE : plan_slices(z, 4 * MIN_SLICE);      // every slice's K have to be joined
}
// Statistics alone: a row need not be held.  Split where long rows are fewer than the blocks that are resident at once.  us, by a block each /
// split, bf16 with the entropy:
//   800 KB    1 row 31 / 6, 64 34 / 16, 200 37 / 32, 300 62 / 44, 400 64 / 61, 500 70 / 79, 1,000 131 / 148
//   320 KB    1 row 13 / 5, 64 15 / 10, 200 17 / 16, 300 25 / 22, 400 27 / 27, 500 29 / 32, 1,000 54 / 60
//   250 KB    1 row 11 / 6, 64 13 / 8, 100 13 / 10, 200 14 / 16; 128 KB 1 row 7 / 6, 100 8 / 8, 200 9 / 10: what splitting saves there for
//             up to 100 rows is mostly less than the second launch costs the host (4 us)
// (From about 400 rows on splitting does not pay; the border is where every row's block is resident.)
Plan plan_stats(const qsl_logits* z) { return z->rows < 2 * FEW_ROWS && row_bytes(z) > HELD_MAX ? plan_slices(z) : WHOLE; }
// Gradients: rows that a block does not hold, and long rows that are few, read twice but by all compute units (64 rows of 256 KB: 18 us
// by a block each, 13 split; 200 rows: 26 and 32; 16 rows of 128 KB: 9 and 13).
Plan plan_gradient(const qsl_logits* z) {
  const uint64_t bytes = row_bytes(z);
  return bytes > HELD_MAX || (bytes > HELD_MAX / 2 && z->rows < FEW_ROWS / 2) ? plan_slices(z) : WHOLE;
}

struct Workspace {
  uint64_t need;
  Slices sl;
  Taught w;
};
// the parts of a call's workspace at `base`
Workspace lay_out(const qsl_logits* z, const Plan& p, uint32_t keys, uint32_t entries, void* base) {
  Workspace w = {};
  if (!p.split) return w;
  char* at = static_cast<char*>(base);
  auto take = [&](uint64_t bytes) { char* r = at + w.need; w.need += align_up(bytes, 256); return r; };
  const uint64_t rows = z->rows;
  w.sl.S = p.S; w.sl.len = p.len;
  w.sl.part = reinterpret_cast<Stat4*>(take(rows * p.S * sizeof(Stat4)));
  if (keys) w.sl.key = reinterpret_cast<uint64_t*>(take(rows * p.S * keys * 8));
  if (entries) {
    w.w.row = reinterpret_cast<Stat4*>(take(rows * sizeof(Stat4)));
    w.w.index = reinterpret_cast<int32_t*>(take(rows * entries * 4));
    w.w.value = reinterpret_cast<float*>(take(rows * entries * 4));
  }
  return w;
}

// `used`: what the call's own plan lays out; a call that uses none is not asked for any, the others for what the query says
qsl_status check_workspace(const qsl_logits* z, uint32_t top, uint64_t used, const void* workspace, size_t bytes) {
  if (used == 0) return QSL_OK;
  const size_t need = qsl_logits_workspace_bytes(z, top);
  if (!workspace || !aligned(workspace, 256)) return QSL_ERR_INVALID_ARG;
  return bytes < need ? QSL_ERR_BUFFER_TOO_SMALL : QSL_OK;
}

dim3 grid_of(uint64_t blocks) {
  return dim3(static_cast<uint32_t>(std::min(blocks, GRID_X)), static_cast<uint32_t>((blocks + GRID_X - 1) / GRID_X));
}

uint64_t apply_blocks(const qsl_logits* z) { const uint64_t n = 1024 * 16 / elem_size(z->dtype); return z->rows * ((z->vocab + n - 1) / n); }

qsl_status launched() { return hipGetLastError() == hipSuccess ? QSL_OK : QSL_ERR_DEVICE; }

}  // namespace

extern "C" size_t qsl_logits_workspace_bytes(const qsl_logits* z, uint32_t top) {
  if (!logits_ok(z) || z->rows == 0 || top > std::max(QSL_TOP_MAX, QSL_TEACHER_MAX)) return 0;
  uint64_t need = std::max(lay_out(z, plan_stats(z), 0, 0, nullptr).need, lay_out(z, plan_gradient(z), 0, top, nullptr).need);
  if (top && top <= QSL_TOP_MAX) need = std::max(need, lay_out(z, plan_top(z), top, 0, nullptr).need);      // (more than that only a teacher has)
  return need;
}

extern "C" qsl_status qsl_token_logprobs(const qsl_logits* z, const int64_t* target, uint32_t top, float* logprob, float* entropy,
                                         float* lse, int32_t* top_index, float* top_logprob, float* stats, void* workspace,
                                         size_t workspace_bytes, void* hip_stream) {
  if (!logits_ok(z)) return QSL_ERR_INVALID_ARG;
  if (top > QSL_TOP_MAX || top > z->vocab) return QSL_ERR_INVALID_ARG;
  if (z->rows == 0) return QSL_OK;
  if ((top == 0) != (!top_index && !top_logprob)) return QSL_ERR_INVALID_ARG;
  if (!logprob && !entropy && !lse && !top && !stats) return QSL_ERR_INVALID_ARG;
  if (logprob && !target) return QSL_ERR_INVALID_ARG;
  if (!aligned(target, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(top_index, 4) ||
      !aligned(top_logprob, 4) || !aligned(stats, 16)) return QSL_ERR_INVALID_ARG;
  const Plan plan = top ? plan_top(z) : plan_stats(z);
  const Workspace ws = lay_out(z, plan, top, 0, workspace);
  const qsl_status st = check_workspace(z, top, ws.need, workspace, workspace_bytes);
  if (st != QSL_OK) return st;
  const uint64_t n = z->rows;
  if (!apart({array(logprob, 4 * n), array(entropy, 4 * n), array(lse, 4 * n), array(top_index, 4 * n * top), array(top_logprob, 4 * n * top),
              array(stats, 16 * n), array(workspace, ws.need)},
             {array(logprob ? target : nullptr, 8 * n), rows_at(z, z->data, z->stride)})) return QSL_ERR_INVALID_ARG;
  const ScoreArgs a = {z->data, z->stride, z->rows, z->vocab, top, z->scale, target, logprob, entropy, lse, top_index, top_logprob, stats};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Slices sl = ws.sl;
  const dim3 rows = grid_of(z->rows);
  const bool last = !stats || z->rows * row_bytes(z) > CACHE_BYTES;      // with `stats` the gradient is to follow, which finds the rows in the cache
  pick_type(z, [&](auto e) {
    typedef decltype(e) E;
    const uint32_t nvec = z->vocab / Elem<E>::N;
    pick_bool(entropy || stats, [&](auto ent) {
      if (plan.split) {
        const dim3 grid = grid_of(static_cast<uint64_t>(z->rows) * plan.S);
        const uint32_t held = (plan.len / Elem<E>::N + 255) / 256;
        if (!top) k_slice_stats<E, 0, ent()><<<grid, 256, 0, stream>>>(a, sl);
        else if (held <= 4) k_slice_stats<E, 4, ent()><<<grid, 256, 0, stream>>>(a, sl);
        else if (held <= 8) k_slice_stats<E, 8, ent()><<<grid, 256, 0, stream>>>(a, sl);
        else k_slice_stats<E, 16, ent()><<<grid, 256, 0, stream>>>(a, sl);
        k_score_join<E, ent()><<<rows, 256, 0, stream>>>(a, sl);
      } else if (top && row_bytes(z) <= HELD_TOP_MAX) {
        pick_for_top(nvec, z->rows, top, [&](auto th, auto nv) { k_score_held<E, th(), nv(), ent()><<<rows, th(), 0, stream>>>(a); });
      } else if (top) {
        k_score<false, E, 1024, ent(), true><<<rows, 1024, 0, stream>>>(a);
      } else {
        // us, 64 / 256 / 1024 threads, bf16 with the entropy: 16,384 rows of 256 vectors 12 / 36 / 68, of 320 21 / 36 / 81, of 1,024 47 / 41 / 130,
        // of 2,048 89 / 83 / 142, of 4,096 176 / 163 / 169, of 8,192 343 / 331 / 317; 64 rows of 256 vectors 3.5 / 3.8 / 4.0, of 320
        // 4.0 / 3.8 / 4.2, of 2,048 7.9 / 4.5 / 5.1, of 2,560 9.2 / 5.2 / 5.1, of 4,096 19 / 7.6 / 5.6.  (The borders are those of few rows;
        // many rows of 257 to about 900 vectors are faster by a wave each.)
        pick_bool(last, [&](auto once) {
          if (nvec <= 256) k_score<once(), E, 64, ent(), false><<<rows, 64, 0, stream>>>(a);
          else if (nvec <= 2048) k_score<once(), E, 256, ent(), false><<<rows, 256, 0, stream>>>(a);
          else k_score<once(), E, 1024, ent(), false><<<rows, 1024, 0, stream>>>(a);
        });
      }
    });
  });
  return launched();
}

extern "C" qsl_status qsl_token_logprobs_backward(const qsl_logits* z, const int64_t* target, const float* grad_logprob,
                                                  const float* grad_entropy, const float* stats, float* logprob, float* entropy,
                                                  void* dlogits, uint64_t dstride, void* workspace, size_t workspace_bytes,
                                                  void* hip_stream) {
  if (!logits_ok(z) || !gradient_ok(z, dlogits, dstride)) return QSL_ERR_INVALID_ARG;
  if (z->rows == 0) return QSL_OK;
  if ((!grad_logprob && !grad_entropy) || ((grad_logprob || logprob) && !target)) return QSL_ERR_INVALID_ARG;
  if (stats && (logprob || entropy)) return QSL_ERR_INVALID_ARG;
  if (!aligned(target, 8) || !aligned(grad_logprob, 4) || !aligned(grad_entropy, 4) || !aligned(stats, 16) || !aligned(logprob, 4) ||
      !aligned(entropy, 4)) return QSL_ERR_INVALID_ARG;
  const Plan plan = stats ? WHOLE : plan_gradient(z);
  const Workspace ws = lay_out(z, plan, 0, 0, workspace);
  const qsl_status st = check_workspace(z, 0, ws.need, workspace, workspace_bytes);
  if (st != QSL_OK) return st;
  const uint64_t n = z->rows;
  const Memory lp = array(logprob, 4 * n), H = array(entropy, 4 * n), parts = array(workspace, ws.need);
  if (!apart({lp, H, parts, rows_at(z, dlogits, dstride)}, {array(target, 8 * n), array(grad_logprob, 4 * n), array(grad_entropy, 4 * n), array(stats, 16 * n)}) ||
      !apart({lp, H, parts}, {rows_at(z, z->data, z->stride)})) return QSL_ERR_INVALID_ARG;
  const GradArgs a = {z->data, dlogits, z->stride, dstride, z->rows, z->vocab, z->scale, target, grad_logprob, grad_entropy, stats, logprob, entropy};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Slices sl = ws.sl;
  pick_type(z, [&](auto e) {
    typedef decltype(e) E;
    pick_bool(grad_entropy || entropy, [&](auto ent) {
      if (!stats && !plan.split) {
        pick_for_gradient(z->vocab / Elem<E>::N, z->rows, [&](auto th, auto nv) { k_gradient_held<E, th(), nv(), ent()><<<grid_of(z->rows), th(), 0, stream>>>(a); });
        return;
      }
      if (!stats) {
        ScoreArgs s = {};
        s.z = z->data; s.stride = z->stride; s.rows = z->rows; s.vocab = z->vocab; s.c = z->scale;
        k_slice_stats<E, 0, ent()><<<grid_of(static_cast<uint64_t>(z->rows) * plan.S), 256, 0, stream>>>(s, sl);
      }
      k_gradient_apply<E, ent()><<<grid_of(apply_blocks(z)), 256, 0, stream>>>(a, sl);
    });
  });
  return launched();
}

static qsl_status launch_distill(const qsl_logits* z, const qsl_teacher* t, const DistillArgs& a, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  const Plan plan = plan_gradient(z);
  const Workspace ws = lay_out(z, plan, 0, t->top, workspace);
  const qsl_status st = check_workspace(z, t->top, ws.need, workspace, workspace_bytes);
  if (st != QSL_OK) return st;
  const uint64_t n = z->rows, entries = 4 * n * t->top;
  const Memory loss = array(a.loss, 4 * n), stats = array(a.stats, 32 * n), parts = array(workspace, ws.need), dz = rows_at(z, a.dz, a.dstride), g = array(a.g, 4 * n);
  // a row's weight is read before its loss is written, by the threads of one block: one array may hold both
  if (!apart({loss, stats, parts, dz}, {array(t->index, entries), array(t->value, entries), array(t->lse, 4 * n), array(a.stats_in, 32 * n)}) ||
      !apart({loss, stats, parts}, {rows_at(z, z->data, z->stride)}) || !apart({stats, parts, dz}, {g}) || (a.loss != a.g && meet(loss, g))) return QSL_ERR_INVALID_ARG;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Taught w = a.dz ? ws.w : Taught{nullptr, nullptr, nullptr};
  pick_type(z, [&](auto e) {
    typedef decltype(e) E;
    pick_bool(t->lse != nullptr, [&](auto rest) {
      if (!plan.split) {
        pick_for_teacher<rest() && sizeof(E) == 2>(z->vocab / Elem<E>::N, z->rows, [&](auto th, auto nv) {
          k_distill_held<E, th(), nv(), rest()><<<grid_of(z->rows), th(), 0, stream>>>(a);
        });
        return;
      }
      if (!a.stats_in) {
        const uint32_t lds = rest() ? 4 * mask_words(std::min(plan.len, MASK_SPAN)) : 0;
        k_distill_slices<E, rest()><<<grid_of(static_cast<uint64_t>(z->rows) * plan.S), 256, lds, stream>>>(a, ws.sl);
      }
      k_distill_join<E, rest()><<<grid_of(z->rows), 256, 0, stream>>>(a, ws.sl, w);
    });
    if (plan.split && a.dz) k_distill_apply<E><<<grid_of(apply_blocks(z)), 256, 0, stream>>>(a, w);
  });
  return launched();
}

extern "C" qsl_status qsl_distill(const qsl_logits* z, const qsl_teacher* teacher, float* loss, float* stats, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  if (!logits_ok(z) || !teacher_ok(z, teacher)) return QSL_ERR_INVALID_ARG;
  if (z->rows == 0) return QSL_OK;
  if ((!loss && !stats) || !aligned(loss, 4) || !aligned(stats, 16)) return QSL_ERR_INVALID_ARG;
  const DistillArgs a = {z->data, nullptr, z->stride, 0, z->rows, z->vocab, teacher->top, z->scale, teacher->scale, teacher->index,
                         teacher->value, teacher->lse, nullptr, nullptr, loss, stats};
  return launch_distill(z, teacher, a, workspace, workspace_bytes, hip_stream);
}

extern "C" qsl_status qsl_distill_backward(const qsl_logits* z, const qsl_teacher* teacher, const float* grad_loss,
                                           const float* stats, float* loss, void* dlogits, uint64_t dstride, void* workspace,
                                           size_t workspace_bytes, void* hip_stream) {
  if (!logits_ok(z) || !teacher_ok(z, teacher) || !gradient_ok(z, dlogits, dstride)) return QSL_ERR_INVALID_ARG;
  if (z->rows == 0) return QSL_OK;
  if ((stats && loss) || !aligned(grad_loss, 4) || !aligned(stats, 16) || !aligned(loss, 4)) return QSL_ERR_INVALID_ARG;
  const DistillArgs a = {z->data, dlogits, z->stride, dstride, z->rows, z->vocab, teacher->top, z->scale, teacher->scale, teacher->index,
                         teacher->value, teacher->lse, grad_loss, stats, loss, nullptr};
  return launch_distill(z, teacher, a, workspace, workspace_bytes, hip_stream);
}
