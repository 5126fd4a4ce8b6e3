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

static_assert(TOP_MAX == QSL_TOP_MAX && TEACHER_MAX == QSL_TEACHER_MAX, "the header's limits");
static_assert(CAND_CAP >= 2 * TOP_MAX, "a full list must hold more than the alternatives");
static_assert(HASH_SIZE >= 2 * TEACHER_MAX && HASH_SIZE == 1u << 10, "teacher_entries takes the upper 10 bits of the hash");

namespace {

constexpr uint32_t MAX_ROW_BLOCKS = 1u << 20;      // blocks of a launch; further rows are taken by the same blocks

bool scale_ok(float c) { return c >= 0x1p-100f && c <= 0x1p100f; }
uint32_t elem_size(uint32_t dtype) { return dtype == QSL_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool logits_ok(const qsl_logits* z) {
  if (!z || z->dtype > QSL_F16 || z->vocab == 0 || z->vocab >= 1u << 31 || z->rows >= 1u << 31) return false;
  if (z->stride < z->vocab || z->stride >= 1ull << 40 || !scale_ok(z->scale)) return false;
  return z->rows == 0 || (z->data && aligned(z->data, elem_size(z->dtype)));
}

// dlogits are the logits, or lie apart from them
bool gradient_ok(const qsl_logits* z, const void* dz, uint64_t dstride) {
  const uint64_t es = elem_size(z->dtype);
  if (dstride < z->vocab || dstride >= 1ull << 40 || !aligned(dz, es)) return false;
  if (z->rows == 0) return true;
  if (!dz) return false;
  if (dz == z->data && (dstride == z->stride || z->rows == 1)) return true;
  const uintptr_t a = reinterpret_cast<uintptr_t>(z->data), b = reinterpret_cast<uintptr_t>(dz);
  const uint64_t la = ((z->rows - 1) * z->stride + z->vocab) * es, lb = ((z->rows - 1) * dstride + z->vocab) * es;
  return a + la <= b || b + lb <= a;
}

bool teacher_ok(const qsl_logits* z, const qsl_teacher* t) {
  if (!t || t->top == 0 || t->top > QSL_TEACHER_MAX || !scale_ok(t->scale)) return false;
  if (z->rows == 0) return true;
  return t->index && t->value && aligned(t->index, 4) && aligned(t->value, 4) && aligned(t->lse, 4);
}

bool workspace_ok(const qsl_logits* z, uint32_t top, const void* workspace, size_t bytes, qsl_status* st) {
  const size_t need = qsl_logits_workspace_bytes(z, top);
  *st = QSL_OK;
  if (need == 0) return true;
  if (!workspace || !aligned(workspace, 256)) *st = QSL_ERR_INVALID_ARG;
  else if (bytes < need) *st = QSL_ERR_BUFFER_TOO_SMALL;
  return *st == QSL_OK;
}

// f(the element type, the threads of a block) as types
template <class F>
void pick(const qsl_logits* z, F&& f) {
  auto by_threads = [&](auto e) {
    const uint32_t nvec = z->vocab / Elem<decltype(e)>::N;
    if (nvec <= 256) f(e, std::integral_constant<int, 64>());
    else if (nvec <= 2048) f(e, std::integral_constant<int, 256>());
    else f(e, std::integral_constant<int, 1024>());
  };
  if (z->dtype == QSL_F32) by_threads(float());
  else if (z->dtype == QSL_BF16) by_threads(__bf16());
  else by_threads(_Float16());
}

template <class F>
void pick_bool(bool b, F&& f) {
  if (b) f(std::true_type());
  else f(std::false_type());
}

dim3 row_grid(uint32_t rows) { return dim3(std::min(rows, MAX_ROW_BLOCKS)); }

qsl_status launched() { return hipGetLastError() == hipSuccess ? QSL_OK : QSL_ERR_DEVICE; }

uint32_t mask_bytes(uint32_t vocab) { return (std::min(vocab, MASK_SPAN) + 31) / 32 * 4; }

}  // namespace

extern "C" size_t qsl_logits_workspace_bytes(const qsl_logits* z, uint32_t top) {
  (void)z; (void)top;
  return 0;
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
  qsl_status st;
  if (!workspace_ok(z, top, workspace, workspace_bytes, &st)) return st;
  const ScoreArgs a = {z->data, z->stride, z->rows, z->vocab, top, z->scale, target, logprob, entropy, lse, top_index, top_logprob, stats};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  pick(z, [&](auto e, auto th) {
    pick_bool(entropy || stats, [&](auto ent) {
      pick_bool(top != 0, [&](auto tp) { k_score<decltype(e), th(), ent(), tp()><<<row_grid(z->rows), th(), 0, stream>>>(a); });
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
  qsl_status st;
  if (!workspace_ok(z, 0, workspace, workspace_bytes, &st)) return st;
  const GradArgs a = {z->data, dlogits, z->stride, dstride, z->rows, z->vocab, z->scale, target, grad_logprob, grad_entropy, stats, logprob, entropy};
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  pick(z, [&](auto e, auto th) {
    pick_bool(grad_entropy || entropy, [&](auto ent) {
      k_logprob_gradient<decltype(e), th(), ent()><<<row_grid(z->rows), th(), 0, stream>>>(a);
    });
  });
  return launched();
}

static qsl_status launch_distill(const qsl_logits* z, const qsl_teacher* t, const DistillArgs& a, bool grad, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  qsl_status st;
  if (!workspace_ok(z, 0, workspace, workspace_bytes, &st)) return st;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  pick(z, [&](auto e, auto th) {
    pick_bool(t->lse != nullptr, [&](auto rest) {
      pick_bool(grad, [&](auto gr) {
        const uint32_t lds = rest() && !a.stats_in ? mask_bytes(z->vocab) : 0;
        k_distill<decltype(e), th(), rest(), gr()><<<row_grid(z->rows), th(), lds, stream>>>(a);
      });
    });
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
  return launch_distill(z, teacher, a, false, workspace, workspace_bytes, hip_stream);
}

extern "C" qsl_status qsl_distill_backward(const qsl_logits* z, const qsl_teacher* teacher, const float* grad_loss,
                                           const float* stats, float* loss, void* dlogits, uint64_t dstride, void* workspace,
                                           size_t workspace_bytes, void* hip_stream) {
  if (!logits_ok(z) || !teacher_ok(z, teacher) || !gradient_ok(z, dlogits, dstride)) return QSL_ERR_INVALID_ARG;
  if (z->rows == 0) return QSL_OK;
  if ((stats && loss) || !aligned(grad_loss, 4) || !aligned(stats, 16) || !aligned(loss, 4)) return QSL_ERR_INVALID_ARG;
  const DistillArgs a = {z->data, dlogits, z->stride, dstride, z->rows, z->vocab, teacher->top, z->scale, teacher->scale, teacher->index,
                         teacher->value, teacher->lse, grad_loss, stats, loss, nullptr};
  return launch_distill(z, teacher, a, true, workspace, workspace_bytes, hip_stream);
}
