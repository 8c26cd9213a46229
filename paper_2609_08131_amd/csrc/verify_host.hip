// C-ABI entry points of the verification of drafted tokens: argument validation, workspace
// layout and launch sequence. Host-detectable errors return before anything is enqueued.
#include <math.h>

#include "verify.hpp"

using namespace jacap;

namespace {

constexpr int64_t kMaxVerifyGrid = (int64_t(1) << 24) - 1;

#define JACAP_TRY(expr)                         \
  do {                                          \
    if ((expr) != hipSuccess) return JACAP_ERR_HIP; \
  } while (0)

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct VerifySpace {
  size_t arrived, mass, parts, total;
};

jacap_status check(const jacap_verification* v, VerifyLaunch* A, VerifySpace* w) {
  if (!v || v->num_seqs < 1 || v->rows < 1 || v->vocab < 1 || v->reserved != 0) return JACAP_ERR_INVALID_ARG;
  if (v->dtype != JACAP_DTYPE_FP32 && v->dtype != JACAP_DTYPE_BF16) return JACAP_ERR_UNSUPPORTED;
  if (v->rows > kMaxVerifyRows || v->vocab > kMaxVocab) return JACAP_ERR_UNSUPPORTED;
  const float k = v->temperature > 0.0f ? (float)(1.44269504088896340736 / (double)v->temperature) : 0.0f;
  if (!(v->temperature >= 0.0f) || !isfinite(v->temperature) || !isfinite(k) ||
      (v->temperature > 0.0f && !(k > 0.0f)))
    return JACAP_ERR_INVALID_ARG;
  if (v->l_stride_seq < 0 || v->l_stride_row < 0 || v->q_stride_seq < 0 || v->q_stride_row < 0 ||
      !aligned(v->parents, 4))
    return JACAP_ERR_INVALID_ARG;
  *A = VerifyLaunch{};
  A->B = v->num_seqs;
  A->S = v->rows;
  A->V = v->vocab;
  A->dtype = v->dtype;
  A->k = k;
  A->lss = v->l_stride_seq;
  A->lsr = v->l_stride_row;
  A->qss = v->q_stride_seq;
  A->qsr = v->q_stride_row;
  A->parents = v->parents;
  A->row_slices = verify_slices(v->vocab, v->dtype, kRowVecs);
  A->slices = verify_slices(v->vocab, v->dtype, kVerifyVecs);
  const int64_t rows = (int64_t)A->B * A->S;
  if (rows > kMaxVerifyGrid || rows * A->row_slices > kMaxVerifyGrid ||
      (int64_t)A->B * A->slices > kMaxVerifyGrid) return JACAP_ERR_UNSUPPORTED;
  size_t o = 256;
  w->arrived = o;
  o = align256(o + 4 * (size_t)A->B);
  w->mass = o;
  o = align256(o + 8 * (size_t)A->B * A->slices);
  w->parts = o;
  o = align256(o + sizeof(RowPart) * (size_t)rows * A->row_slices);
  w->total = o;
  return JACAP_OK;
}

}  // namespace

extern "C" {

jacap_status jacap_verify_workspace_size(const jacap_verification* ver, size_t* bytes) {
  if (!bytes) return JACAP_ERR_INVALID_ARG;
  VerifyLaunch A;
  VerifySpace w;
  const jacap_status s = check(ver, &A, &w);
  if (s != JACAP_OK) return s;
  *bytes = w.total;
  return JACAP_OK;
}

jacap_status jacap_verify(const jacap_verification* ver, const void* logits, const int32_t* tokens,
                          const float* uniform, const float* draft, int32_t* path, int32_t* count,
                          int32_t* next, float* row_weight, void* ws, size_t ws_bytes,
                          void* stream) {
  VerifyLaunch A;
  VerifySpace w;
  const jacap_status s = check(ver, &A, &w);
  if (s != JACAP_OK) return s;
  if (!ws || !aligned(ws, 256)) return JACAP_ERR_INVALID_ARG;
  if (ws_bytes < w.total) return JACAP_ERR_WORKSPACE;
  const bool greedy = A.k == 0.0f;
  if (!logits || !aligned(logits, A.dtype == JACAP_DTYPE_BF16 ? 2 : 4) || (!tokens && A.S > 1) ||
      !aligned(tokens, 4) || (!uniform && !greedy) || !aligned(uniform, 4) || !aligned(draft, 4) || !path ||
      !aligned(path, 4) || !count || !aligned(count, 4) || !next || !aligned(next, 4) || !aligned(row_weight, 4))
    return JACAP_ERR_INVALID_ARG;
  char* base = static_cast<char*>(ws);
  A.logits = logits;
  A.tokens = tokens;
  A.uniform = uniform;
  A.draft = greedy ? nullptr : draft;
  A.path = path;
  A.count = count;
  A.next = next;
  A.row_weight = row_weight;
  A.status = ws_ptr<uint32_t>(base, 0);
  A.arrived = ws_ptr<uint32_t>(base, w.arrived);
  A.mass = ws_ptr<double>(base, w.mass);
  A.parts = ws_ptr<RowPart>(base, w.parts);
  A.stream = static_cast<hipStream_t>(stream);
  {
    TimedPhase tp(A.stream, JACAP_PHASE_VERIFY_ROWS);
    JACAP_TRY(launch_verify_rows(A));
  }
  TimedPhase tp(A.stream, JACAP_PHASE_VERIFY);
  JACAP_TRY(launch_verify(A));
  return JACAP_OK;
}

}  // extern "C"
