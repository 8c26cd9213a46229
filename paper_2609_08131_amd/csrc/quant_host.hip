// C-ABI entry points of the 8-bit cache: argument validation, workspace layout and launch
// sequences. Host-detectable errors return before anything is enqueued.
#include <algorithm>

#include "quant.hpp"

using namespace jacap;

namespace {

#define JACAP_TRY(expr)                         \
  do {                                          \
    if ((expr) != hipSuccess) return JACAP_ERR_HIP; \
  } while (0)

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool array_ok(const void* p) { return p && aligned(p, 16); }
bool token_array_ok(const void* p, const jacap_batch* b, uintptr_t align = 16) {
  return p ? aligned(p, align) : b->total_tokens == 0;
}
bool optional_ok(const void* p, uintptr_t align) { return !p || aligned(p, align); }

// The cache's description; `own`: the batch's strides are another cache's (jacap_quantize),
// else they are not read and `b` gets the codes'.
jacap_status check_quant(const jacap_config* cfg, const jacap_batch* batch, const jacap_quant* quant, bool own,
                         jacap_batch* b, QuantArgs* q) {
  if (!cfg || !batch || !quant || quant->reserved != 0) return JACAP_ERR_INVALID_ARG;
  if (quant->block != 16 && quant->block != 32 && quant->block != 64 && quant->block != 128)
    return JACAP_ERR_UNSUPPORTED;
  if (batch->total_tokens % quant->block != 0) return JACAP_ERR_INVALID_ARG;
  const int64_t st[] = {quant->k_stride_layer, quant->k_stride_head, quant->k_stride_token,
                        quant->v_stride_layer, quant->v_stride_head, quant->v_stride_token};
  for (int64_t x : st)
    if (x < 0 || x % 16 != 0) return JACAP_ERR_INVALID_ARG;
  if (quant->k_stride_token < cfg->head_dim || quant->v_stride_token < cfg->head_dim) return JACAP_ERR_INVALID_ARG;
  if (quant->k_stride_token > kMaxTokenStride || quant->v_stride_token > kMaxTokenStride)
    return JACAP_ERR_UNSUPPORTED;
  *b = *batch;
  if (!own) {
    b->k_stride_layer = quant->k_stride_layer;
    b->k_stride_head = quant->k_stride_head;
    b->k_stride_token = quant->k_stride_token;
    b->v_stride_layer = quant->v_stride_layer;
    b->v_stride_head = quant->v_stride_head;
    b->v_stride_token = quant->v_stride_token;
  }
  *q = QuantArgs{};
  while (1 << q->shift < quant->block) ++q->shift;
  q->ksl = quant->k_stride_layer;
  q->ksh = quant->k_stride_head;
  q->kst = quant->k_stride_token;
  q->vsl = quant->v_stride_layer;
  q->vsh = quant->v_stride_head;
  q->vst = quant->v_stride_token;
  return JACAP_OK;
}

void point_at(QuantArgs* q, const void* kq, const void* vq, const float* scales) {
  q->k = static_cast<const uint8_t*>(kq);
  q->v = static_cast<const uint8_t*>(vq);
  q->scales = reinterpret_cast<const float2*>(scales);
}

// jacap_attend_quant's descriptors and workspace.
jacap_status prepare_attend(const jacap_config* cfg, const jacap_batch* batch, const jacap_attention* attn,
                            const jacap_quant* quant, void* stream, QuantLaunch* A, AttendSpace* w) {
  jacap_batch b;
  jacap_status s = check_quant(cfg, batch, quant, false, &b, &A->q);
  if (s != JACAP_OK) return s;
  s = check_attend(cfg, &b, attn, stream, &A->attn);
  if (s != JACAP_OK) return s;
  A->attn.at.row_mask = quant->block - 1;
  // (the sums of more rows than keep their logits need no workspace here)
  AttnLaunch L = A->attn;
  if (L.at.R > kKeepRows) L.at.accumulate = 0;
  WeightsSpace sum;
  s = layout_attend(L, cfg->dtype == JACAP_DTYPE_BF16, w, &sum);
  if (s != JACAP_OK) return s;
  // Short caches: a launch less, while a unit is but a few steps of its waves (a token over one
  // sequence of 512 tokens, 8 KV heads, replayed from a graph: 15.6 us, 17.9 by spans; over 16
  // of them 16.7 and 23.2; over one of 1024 18.7 and 17.9).
  w->whole = w->rw == 0 && A->attn.base.geo.maxn <= kWholeTokens;
  const int64_t blocks = A->attn.base.geo.maxn / kThreads + 1;
  return (int64_t)A->attn.base.geo.U * blocks <= kMaxGrid ? JACAP_OK : JACAP_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

jacap_status jacap_quantize(const jacap_config* cfg, const jacap_batch* batch,
                            const jacap_attention* attn, const jacap_quant* quant, const void* k,
                            const void* v, const float* acc, void* kq, void* vq, float* scales,
                            void* stream) {
  QuantLaunch A;
  jacap_batch b;
  jacap_status s = check_quant(cfg, batch, quant, true, &b, &A.q);
  if (s != JACAP_OK) return s;
  s = check_attention(cfg, &b, attn, stream, &A.attn);
  if (s != JACAP_OK) return s;
  Geo& g = A.attn.base.geo;
  A.attn.at.row_mask = quant->block - 1;
  if ((int64_t)g.U * (g.maxn / 128 + 1) > kMaxGrid) return JACAP_ERR_UNSUPPORTED;
  if (!token_array_ok(k, batch) || !token_array_ok(v, batch) || !optional_ok(acc, 4) ||
      !token_array_ok(kq, batch) || !token_array_ok(vq, batch) || !token_array_ok(scales, batch, 8))
    return JACAP_ERR_INVALID_ARG;
  TimedPhase tp(A.attn.base.stream, JACAP_PHASE_QUANTIZE);
  JACAP_TRY(launch_quantize(A, k, v, acc, kq, vq, scales));
  return JACAP_OK;
}

jacap_status jacap_append_quant(const jacap_config* cfg, const jacap_batch* batch,
                                const jacap_attention* attn, const jacap_quant* quant,
                                const void* kd, const void* vd, const int32_t* start,
                                const int32_t* count, const int32_t* rows, const int32_t* slots,
                                int32_t slot_cap, void* kq, void* vq, float* scales, float* acc,
                                const float* acc_draft, int32_t* start_out, uint32_t* status,
                                void* stream) {
  QuantLaunch A;
  jacap_batch b;
  jacap_status s = check_quant(cfg, batch, quant, false, &b, &A.q);
  if (s != JACAP_OK) return s;
  s = check_attend(cfg, &b, attn, stream, &A.attn);
  if (s != JACAP_OK) return s;
  Geo& g = A.attn.base.geo;
  A.attn.at.row_mask = quant->block - 1;
  g.live = nullptr;  // the whole of a sequence's rows may be written
  if (g.U > kMaxGrid) return JACAP_ERR_UNSUPPORTED;
  if (!array_ok(kd) || !array_ok(vd) || (!start && !slots) || !optional_ok(start, 4) || !optional_ok(count, 4) ||
      !optional_ok(rows, 4) || !optional_ok(slots, 4) || slot_cap < 0 || !token_array_ok(kq, batch) ||
      !token_array_ok(vq, batch) || !token_array_ok(scales, batch, 8) || !optional_ok(acc, 4) ||
      !optional_ok(acc_draft, 4) || !optional_ok(start_out, 4) || !optional_ok(status, 4))
    return JACAP_ERR_INVALID_ARG;
  const AppendArgs p{start, count, rows, slots, slot_cap, acc, acc_draft, start_out, status};
  TimedPhase tp(A.attn.base.stream, JACAP_PHASE_APPEND);
  JACAP_TRY(launch_append(A, p, kd, vd, kq, vq, scales));
  return JACAP_OK;
}

jacap_status jacap_attend_quant_workspace_size(const jacap_config* cfg, const jacap_batch* batch,
                                               const jacap_attention* attn, const jacap_quant* quant,
                                               size_t* bytes) {
  if (!bytes) return JACAP_ERR_INVALID_ARG;
  QuantLaunch A;
  AttendSpace w;
  const jacap_status s = prepare_attend(cfg, batch, attn, quant, nullptr, &A, &w);
  if (s != JACAP_OK) return s;
  *bytes = w.total;
  return JACAP_OK;
}

jacap_status jacap_attend_quant(const jacap_config* cfg, const jacap_batch* batch,
                                const jacap_attention* attn, const jacap_quant* quant,
                                const void* q, const void* kq, const void* vq, const float* scales,
                                const void* kd, const void* vd, void* out, float* lse, float* acc,
                                float* acc_draft, void* ws, size_t ws_bytes, void* stream) {
  QuantLaunch A;
  AttendSpace w;
  const jacap_status s = prepare_attend(cfg, batch, attn, quant, stream, &A, &w);
  if (s != JACAP_OK) return s;
  AttnLaunch& L = A.attn;
  if (!ws || !aligned(ws, 256)) return JACAP_ERR_INVALID_ARG;
  if (ws_bytes < w.total) return JACAP_ERR_WORKSPACE;
  L.base.wsp = static_cast<char*>(ws);
  if (!array_ok(q) || !token_array_ok(kq, batch) || !token_array_ok(vq, batch) ||
      !token_array_ok(scales, batch, 8) || !array_ok(kd) || !array_ok(vd) || !array_ok(out) ||
      !optional_ok(lse, 4) || !optional_ok(acc, 4) || !optional_ok(acc_draft, 4))
    return JACAP_ERR_INVALID_ARG;
  if (attn->accumulate && !acc && batch->total_tokens > 0) return JACAP_ERR_INVALID_ARG;
  point_at(&A.q, kq, vq, scales);
  const bool sums = attn->accumulate && !w.keep;  // a pass of its own, from the rows' lse
  float* ls = lse ? lse : attn->accumulate ? ws_ptr<float>(L.base.wsp, w.lse) : nullptr;
  {
    TimedPhase tp(L.base.stream, JACAP_PHASE_ATTEND);
    JACAP_TRY(launch_attend_quant(A, w, q, kd, vd, out, ls, acc));
  }
  if (w.whole ? w.keep : attend_joins(L, w)) {
    TimedPhase tp(L.base.stream, JACAP_PHASE_ATTEND_JOIN);
    JACAP_TRY(launch_attend_join_groups(L, w, kQuantGroup, out, ls, acc, acc_draft));
  }
  if (sums) {
    TimedPhase tp(L.base.stream, JACAP_PHASE_ATTN_SUM);
    L.at.causal = 0;
    if (acc_draft) JACAP_TRY(launch_draft_sum(L, q, kd, ls, acc_draft));
    if (batch->total_tokens > 0) JACAP_TRY(launch_quant_sum(A, q, ls, acc, nullptr));
  }
  return JACAP_OK;
}

jacap_status jacap_attn_weights_quant(const jacap_config* cfg, const jacap_batch* batch,
                                      const jacap_attention* attn, const jacap_quant* quant,
                                      const void* q, const void* kq, const float* scales,
                                      const float* lse_in, float* acc, uint32_t* status,
                                      void* stream) {
  QuantLaunch A;
  jacap_batch b;
  jacap_status s = check_quant(cfg, batch, quant, false, &b, &A.q);
  if (s != JACAP_OK) return s;
  s = check_attention(cfg, &b, attn, stream, &A.attn);
  if (s != JACAP_OK) return s;
  Geo& g = A.attn.base.geo;
  A.attn.at.row_mask = quant->block - 1;
  if (attn->causal || cfg->window > kMaxDraft || (int64_t)g.U * (g.maxn / kThreads + 1) > kMaxGrid)
    return JACAP_ERR_UNSUPPORTED;
  if (!array_ok(q) || !token_array_ok(kq, batch) || !token_array_ok(scales, batch, 8) || !lse_in ||
      !aligned(lse_in, 4) || !token_array_ok(acc, batch, 4) || !optional_ok(status, 4))
    return JACAP_ERR_INVALID_ARG;
  point_at(&A.q, kq, kq, scales);
  TimedPhase tp(A.attn.base.stream, JACAP_PHASE_ATTN_SUM);
  JACAP_TRY(launch_quant_sum(A, q, lse_in, acc, status));
  return JACAP_OK;
}

}  // extern "C"
