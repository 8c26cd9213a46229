// C-ABI entry points of the attention over the cache and of the eviction by
// accumulated weight: argument validation, workspace layouts and launch
// sequences. Host-detectable errors return before anything is enqueued.
#include <math.h>

#include <algorithm>

#include "attention.hpp"

using namespace jacap;

namespace {

#define JACAP_TRY(expr)                         \
  do {                                          \
    if ((expr) != hipSuccess) return JACAP_ERR_HIP; \
  } while (0)

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Required arrays, and those that may be null where a batch holds no tokens.
bool array_ok(const void* p) { return p && aligned(p, 16); }
bool token_array_ok(const void* p, const jacap_batch* b, uintptr_t align = 16) {
  return p ? aligned(p, align) : b->total_tokens == 0;
}
bool optional_ok(const void* p, uintptr_t align) { return !p || aligned(p, align); }

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// The descriptor and what every call shares. ws = null: no workspace is checked.
jacap_status check(const jacap_config* cfg, const jacap_batch* batch, const jacap_attention* at,
                   void* stream, AttnLaunch* A) {
  if (!batch || !at) return JACAP_ERR_INVALID_ARG;
  // No sequence is longer than all of them, whatever length the caller declares: what is cut
  // and counted below (in 32 bits, up to a chunk past the end) follows the shorter.
  jacap_batch b = *batch;
  if (b.total_tokens > kMaxTokens) return JACAP_ERR_UNSUPPORTED;
  b.max_seq_len = (int32_t)std::min<int64_t>(b.max_seq_len, std::max<int64_t>(b.total_tokens, 0));
  const jacap_status s = prepare_launch(cfg, &b, nullptr, 0, stream, &A->base);
  if (s != JACAP_OK) return s;
  if (!(at->scale > 0.0f) || !isfinite(at->scale * kLog2e)) return JACAP_ERR_INVALID_ARG;
  if (!(at->decay >= 0.0f && at->decay <= 1.0f)) return JACAP_ERR_INVALID_ARG;
  if ((at->accumulate | 1) != 1 || (at->causal | 1) != 1) return JACAP_ERR_INVALID_ARG;
  if (!optional_ok(at->live_lens, 4) || !optional_ok(at->row_weight, 4) || !optional_ok(at->tree, 8))
    return JACAP_ERR_INVALID_ARG;
  const int64_t R = (int64_t)A->base.geo.G * cfg->window;
  if (R > INT32_MAX / 2) return JACAP_ERR_UNSUPPORTED;
  A->base.geo.live = at->live_lens;
  Attn& a = A->at;
  a = Attn{};
  a.c = (float)((double)at->scale * 1.44269504088896340736);
  a.decay = at->decay;
  a.accumulate = at->accumulate;
  a.causal = at->causal;
  a.R = (int)R;
  a.row_weight = at->row_weight;
  a.tree = reinterpret_cast<const uint32_t*>(at->tree);
  a.tree_words = (cfg->window + 63) / 64 * 2;
  return JACAP_OK;
}

jacap_status check_attend(const jacap_config* cfg, const jacap_batch* batch,
                          const jacap_attention* at, void* stream, AttnLaunch* A) {
  const jacap_status s = check(cfg, batch, at, stream, A);
  if (s != JACAP_OK) return s;
  if (cfg->window > kMaxDraft) return JACAP_ERR_UNSUPPORTED;
  const int64_t st[] = {at->dk_stride_seq, at->dk_stride_layer, at->dk_stride_head,
                        at->dk_stride_row, at->dv_stride_seq, at->dv_stride_layer,
                        at->dv_stride_head, at->dv_stride_row, at->o_stride_seq,
                        at->o_stride_layer, at->o_stride_head, at->o_stride_pos};
  for (int64_t x : st)
    if (x < 0 || x % 8 != 0) return JACAP_ERR_INVALID_ARG;
  const int d = cfg->head_dim;
  if (at->dk_stride_row < d || at->dv_stride_row < d || at->o_stride_pos < d)
    return JACAP_ERR_INVALID_ARG;
  if (at->dk_stride_row > kMaxTokenStride || at->dv_stride_row > kMaxTokenStride)
    return JACAP_ERR_UNSUPPORTED;
  Attn& a = A->at;
  a.dks = at->dk_stride_seq; a.dkl = at->dk_stride_layer; a.dkh = at->dk_stride_head; a.dkr = at->dk_stride_row;
  a.dvs = at->dv_stride_seq; a.dvl = at->dv_stride_layer; a.dvh = at->dv_stride_head; a.dvr = at->dv_stride_row;
  a.os = at->o_stride_seq; a.ol = at->o_stride_layer; a.oh = at->o_stride_head; a.op = at->o_stride_pos;
  return JACAP_OK;
}

// How the passes over rows and tokens of the weights are cut; `o` the
// workspace's size so far. The chunks of the log-sums are one round of the chip (fp32
// rows, 32768 tokens: 92 us, 102 with chunks of half the size; five sequences of 100 to
// 30000 tokens 120 and 141, equal long ones the same); small batches take fewer rows a
// workgroup and half a round of longer chunks, as the rows' loads and the join of the
// chunks weigh more (128 rows of 8192 tokens 21.2 us, 23.7 otherwise; of 16384 29.9 and 35.3;
// of 32768 42.9 and 45.9; 64 rows of 8192 tokens 17.1 and 16.9). The rows of the sums stay
// in LDS, a stretch of tokens passing them (256 rows, 4 layers of 131072 tokens: 718 us
// with the log-sums, 865 with the rows staged for every 256 tokens; 100 rows, 2 layers of
// 65536: 111 and 141; 256 rows of 1000 tokens 26.7 and 25.6, from the split of their rows);
// more than fit there are staged, in parts while the grid is small.
void layout_sum(const Geo& g, const Attn& at, bool bf16, WeightsSpace* w, size_t* o) {
  const int64_t LHT = (int64_t)g.L * g.H * g.T;
  const int tiles = (at.R + 15) / 16;
  w->mt = !bf16 ? kRowTilesFp32 : tiles <= 2 ? 2 : tiles <= 4 ? 4 : kRowTilesBf16;
  auto cut = [&](int blocks) {
    w->row_blocks = (tiles + w->mt - 1) / w->mt;
    return (LHT * w->row_blocks / blocks + 63) / 64 * 64;
  };
  int64_t per_block = cut(kRowsBlocks);
  if (per_block < kRowsSmall) {
    w->mt = std::min(w->mt, 4);
    per_block = cut(kRowsBlocks / 2);
  }
  w->chunk = (int)std::max<int64_t>(kRowsChunkMin, std::min<int64_t>(per_block, kRowsChunk));
  w->chunks = std::max(1, (g.maxn + w->chunk - 1) / w->chunk);
  w->tiles = bf16 ? kSumTilesBf16 : kSumTilesFp32;
  const int tokens = 64 * w->tiles;
  w->blocks = (g.maxn + tokens - 1) / tokens;
  w->held = 0;
  w->row_splits = 1;
  if (at.R <= held_rows(g.D * (bf16 ? 2 : 4))) {
    const int64_t per = (LHT / kHeldBlocks + tokens - 1) / tokens * tokens;
    w->held = (int)std::min<int64_t>(std::max<int64_t>(per, tokens), 1 << 20);
    w->blocks = (g.maxn + w->held - 1) / w->held;
  } else {
    const int64_t grid = std::max<int64_t>(1, LHT / tokens);
    w->row_splits =
        (int)std::max<int64_t>(1, std::min<int64_t>(kSumBlocks / grid, at.R / kSumRowsMin));
  }
  w->part = *o;
  if (w->row_splits > 1) *o = align256(*o + 4 * (size_t)w->row_splits * LHT);
}

bool sum_grid_ok(const Geo& g, const WeightsSpace& w) {
  return (int64_t)g.U * w.row_blocks * w.chunks <= kMaxGrid &&
         (int64_t)g.U * std::max(1, w.blocks) * w.row_splits <= kMaxGrid;
}

jacap_status layout_weights(const AttnLaunch& A, bool bf16, WeightsSpace* w) {
  const Geo& g = A.base.geo;
  const int64_t UR = (int64_t)g.U * A.at.R;
  if (UR / 16 > kMaxGrid) return JACAP_ERR_UNSUPPORTED;
  size_t o = 256;
  layout_sum(g, A.at, bf16, w, &o);
  w->lse = o;
  o = align256(o + 4 * (size_t)UR);
  w->ml = o;
  if (w->chunks > 1) o = align256(o + 8 * (size_t)UR * w->chunks);
  w->total = o;
  return sum_grid_ok(g, *w) ? JACAP_OK : JACAP_ERR_UNSUPPORTED;
}

// sum: the accumulation's own cut, for accumulating from more rows than keep
// their logits.
jacap_status layout_attend(const AttnLaunch& A, bool bf16, AttendSpace* w, WeightsSpace* sum) {
  const Geo& g = A.base.geo;
  const int64_t UR = (int64_t)g.U * A.at.R, LHT = (int64_t)g.L * g.H * g.T;
  if (UR > kMaxGrid) return JACAP_ERR_UNSUPPORTED;
  size_t o = 256;
  w->mt = A.at.R <= 16 ? 1 : 2;
  w->rw = !bf16 || A.at.R <= kWideRows ? 0 : A.at.R <= 64 ? 2 : A.at.R <= 128 ? 4 : 8;
  const int rows = w->rw ? 32 * w->rw : 16 * w->mt;
  w->row_blocks = (A.at.R + rows - 1) / rows;
  w->spans = w->places = 0;
  w->chunk = w->splits = 1;
  int64_t pieces;
  if (w->rw) {
    // one round of a workgroup per compute unit, in whole stages of 128 tokens
    const int64_t per = (LHT * w->row_blocks + kWideBlocks - 1) / kWideBlocks;
    w->chunk = (int)std::min<int64_t>(std::max<int64_t>((per + 127) / 128 * 128, kWideChunkMin),
                                      1 << 20);
    w->splits = std::max(1, (g.maxn + w->chunk - 1) / w->chunk);
    // Bounded by the tokens: with a place for each chunk of the longest in every sequence,
    // 64 sequences of which one has 131072 tokens would take 2 GB (252 rows, 8 KV heads;
    // 100 MB so).
    w->places = w->splits > 1 ? (int)(g.T / w->chunk) + g.B : 0;
    pieces = (int64_t)g.L * g.H * w->places * A.at.R;
  } else {
    // no more spans than there can be work for
    const int64_t most = (LHT / kSpanMin + (int64_t)g.U * (1 + kUnitGroups)) * w->row_blocks;
    w->spans = (int)std::min<int64_t>(kSpans, most);
    pieces = 2 * (int64_t)w->spans * rows;
  }
  w->keep = A.at.accumulate && A.at.R <= kKeepRows;
  w->before = o;
  o = align256(o + 4 * ((size_t)g.B + 1));
  w->lse = o;
  o = align256(o + 4 * (size_t)UR);
  w->ml = o;
  o = align256(o + 8 * (size_t)pieces);
  w->part = o;
  o = align256(o + 4 * (size_t)pieces * g.D);
  w->z = o;
  if (w->keep) o = align256(o + 4 * (size_t)g.L * g.H * (g.T / 16 + g.B + 1) * 16 * A.at.R);
  w->zd = o;
  if (w->keep) o = align256(o + 4 * (size_t)UR * g.w);
  *sum = WeightsSpace{};
  if (A.at.accumulate && !w->keep) layout_sum(g, A.at, bf16, sum, &o);
  w->total = o;
  const int64_t token_blocks = g.maxn / kJoinTokens + 1;
  // 32-bit counts of groups (of at least 64 tokens) and of pieces
  const int64_t groups =
      (int64_t)g.L * g.H * w->row_blocks * (g.T / 64 + (int64_t)g.B * (1 + kUnitGroups));
  if (((int64_t)g.U * w->splits + 8) * w->row_blocks > kMaxGrid || UR + g.U * token_blocks > kMaxGrid ||
      groups > kMaxGroups || pieces > INT32_MAX || !sum_grid_ok(g, *sum))
    return JACAP_ERR_UNSUPPORTED;
  return JACAP_OK;
}

bool is_bf16(const jacap_config* c) { return c->dtype == JACAP_DTYPE_BF16; }

jacap_status take_workspace(void* ws, size_t ws_bytes, size_t need, Launch* L) {
  if (!ws || !aligned(ws, 256)) return JACAP_ERR_INVALID_ARG;
  if (ws_bytes < need) return JACAP_ERR_WORKSPACE;
  L->wsp = static_cast<char*>(ws);
  return JACAP_OK;
}

// jacap_evict_weighted(_slots): the kept positions are staged at byte 256.
size_t kept_bytes(const jacap_config* c, const Geo& g) {
  return align256(256 + 4 * (size_t)g.U * std::max(c->budget_k, 1));
}

}  // namespace

extern "C" {

jacap_status jacap_attend_workspace_size(const jacap_config* cfg, const jacap_batch* batch,
                                         const jacap_attention* attn, size_t* bytes) {
  if (!bytes) return JACAP_ERR_INVALID_ARG;
  AttnLaunch A;
  jacap_status s = check_attend(cfg, batch, attn, nullptr, &A);
  if (s != JACAP_OK) return s;
  AttendSpace w;
  WeightsSpace sum;
  s = layout_attend(A, is_bf16(cfg), &w, &sum);
  if (s != JACAP_OK) return s;
  *bytes = w.total;
  return JACAP_OK;
}

jacap_status jacap_attend(const jacap_config* cfg, const jacap_batch* batch,
                          const jacap_attention* attn, const void* q, const void* k,
                          const void* v, const void* kd, const void* vd, void* out, float* lse,
                          float* acc, float* acc_draft, void* ws, size_t ws_bytes, void* stream) {
  AttnLaunch A;
  jacap_status s = check_attend(cfg, batch, attn, stream, &A);
  if (s != JACAP_OK) return s;
  AttendSpace w;
  WeightsSpace sum;
  s = layout_attend(A, is_bf16(cfg), &w, &sum);
  if (s != JACAP_OK) return s;
  s = take_workspace(ws, ws_bytes, w.total, &A.base);
  if (s != JACAP_OK) return s;
  if (!array_ok(q) || !token_array_ok(k, batch) || !token_array_ok(v, batch) || !array_ok(kd) ||
      !array_ok(vd) || !array_ok(out) || !optional_ok(lse, 4) || !optional_ok(acc, 4) ||
      !optional_ok(acc_draft, 4))
    return JACAP_ERR_INVALID_ARG;
  if (attn->accumulate && !acc && batch->total_tokens > 0) return JACAP_ERR_INVALID_ARG;
  const bool sums = attn->accumulate && !w.keep;  // a pass of its own, from the rows' lse
  float* ls = lse ? lse : attn->accumulate ? ws_ptr<float>(A.base.wsp, w.lse) : nullptr;
  {
    TimedPhase tp(A.base.stream, JACAP_PHASE_ATTEND);
    JACAP_TRY(launch_attend(A, w, q, k, v, kd, vd, out, ls, acc));
  }
  if (attend_joins(A, w)) {
    TimedPhase tp(A.base.stream, JACAP_PHASE_ATTEND_JOIN);
    JACAP_TRY(launch_attend_join(A, w, out, ls, acc, acc_draft));
  }
  if (sums) {
    TimedPhase tp(A.base.stream, JACAP_PHASE_ATTN_SUM);
    A.at.causal = 0;
    if (acc_draft) JACAP_TRY(launch_draft_sum(A, q, kd, ls, acc_draft));
    if (batch->total_tokens > 0) JACAP_TRY(launch_attn_sum(A, sum, q, k, ls, acc, nullptr));
  }
  return JACAP_OK;
}

jacap_status jacap_attn_weights_workspace_size(const jacap_config* cfg, const jacap_batch* batch,
                                               const jacap_attention* attn, size_t* bytes) {
  if (!bytes) return JACAP_ERR_INVALID_ARG;
  AttnLaunch A;
  jacap_status s = check(cfg, batch, attn, nullptr, &A);
  if (s != JACAP_OK) return s;
  WeightsSpace w;
  s = layout_weights(A, is_bf16(cfg), &w);
  if (s != JACAP_OK) return s;
  *bytes = w.total;
  return JACAP_OK;
}

jacap_status jacap_attn_weights(const jacap_config* cfg, const jacap_batch* batch,
                                const jacap_attention* attn, const void* q, const void* k,
                                const float* lse_in, float* lse_out, float* acc, void* ws,
                                size_t ws_bytes, void* stream) {
  AttnLaunch A;
  jacap_status s = check(cfg, batch, attn, stream, &A);
  if (s != JACAP_OK) return s;
  WeightsSpace w;
  s = layout_weights(A, is_bf16(cfg), &w);
  if (s != JACAP_OK) return s;
  s = take_workspace(ws, ws_bytes, w.total, &A.base);
  if (s != JACAP_OK) return s;
  if (!array_ok(q) || !token_array_ok(k, batch) || !token_array_ok(acc, batch, 4) ||
      !optional_ok(lse_in, 4) || !optional_ok(lse_out, 4) || (lse_in && lse_out))
    return JACAP_ERR_INVALID_ARG;
  const float* ls = lse_in;
  if (!lse_in) {
    float* to = lse_out ? lse_out : ws_ptr<float>(A.base.wsp, w.lse);
    TimedPhase tp(A.base.stream, JACAP_PHASE_ATTN_LSE);
    JACAP_TRY(launch_attn_lse(A, w, q, k, acc, to));
    ls = to;
  }
  TimedPhase tp(A.base.stream, JACAP_PHASE_ATTN_SUM);
  JACAP_TRY(launch_attn_sum(A, w, q, k, ls, acc, ws_ptr<uint32_t>(A.base.wsp, 0)));
  return JACAP_OK;
}

jacap_status jacap_evict_weighted_workspace_size(const jacap_config* cfg, const jacap_batch* batch,
                                                 const jacap_attention* attn, size_t* bytes) {
  if (!bytes) return JACAP_ERR_INVALID_ARG;
  AttnLaunch A;
  const jacap_status s = check(cfg, batch, attn, nullptr, &A);
  if (s != JACAP_OK) return s;
  *bytes = kept_bytes(cfg, A.base.geo);
  return JACAP_OK;
}

jacap_status jacap_evict_weighted(const jacap_config* cfg, const jacap_batch* batch,
                                  const jacap_attention* attn, const float* acc, const void* k,
                                  const void* v, int32_t* idx, void* k_out, void* v_out,
                                  float* acc_out, void* stream) {
  AttnLaunch A;
  const jacap_status s = check(cfg, batch, attn, stream, &A);
  if (s != JACAP_OK) return s;
  if (attn->a_stride_seq < 0 || attn->a_stride_layer < 0 || attn->a_stride_head < 0)
    return JACAP_ERR_INVALID_ARG;
  if (cfg->budget_k == 0) return JACAP_OK;
  if (!array_ok(idx) || !token_array_ok(acc, batch, 4) || !acc_out || !aligned(acc_out, 4) ||
      !token_array_ok(k, batch) || !token_array_ok(v, batch) || !token_array_ok(k_out, batch) ||
      !token_array_ok(v_out, batch))
    return JACAP_ERR_INVALID_ARG;
  const Launch& L = A.base;
  {
    TimedPhase tp(L.stream, JACAP_PHASE_SELECT);
    JACAP_TRY(launch_select(L, acc, idx));
  }
  TimedPhase tp(L.stream, JACAP_PHASE_COMPACT);
  JACAP_TRY(launch_compact_weighted(L, idx, k, v, k_out, v_out, acc, acc_out, attn->a_stride_seq,
                                    attn->a_stride_layer, attn->a_stride_head));
  return JACAP_OK;
}

jacap_status jacap_evict_weighted_slots(const jacap_config* cfg, const jacap_batch* batch,
                                        const jacap_attention* attn, float* acc, int32_t* slots,
                                        int32_t slot_cap, void* ws, size_t ws_bytes,
                                        void* stream) {
  AttnLaunch A;
  jacap_status s = check(cfg, batch, attn, stream, &A);
  if (s != JACAP_OK) return s;
  s = take_workspace(ws, ws_bytes, kept_bytes(cfg, A.base.geo), &A.base);
  if (s != JACAP_OK) return s;
  if (!array_ok(slots) || !token_array_ok(acc, batch, 4) || slot_cap < 0 ||
      slot_cap < batch->max_seq_len - cfg->budget_k)
    return JACAP_ERR_INVALID_ARG;
  Launch& L = A.base;
  L.ws.kept = 256;
  TimedPhase tp(L.stream, JACAP_PHASE_SELECT);
  JACAP_TRY(launch_select_empty(L, acc, slots, slot_cap));
  return JACAP_OK;
}

}  // extern "C"
