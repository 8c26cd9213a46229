// Drives the host layer of the attention over the cache and of the eviction by
// accumulated weight (attention_host.hip), built with AddressSanitizer and
// UndefinedBehaviorSanitizer, against the stand-ins of attention_stubs.cpp: no GPU
// is touched, and no data pointer is read. Exits non-zero on the first
// unexpected result.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

#include "attention_stubs.hpp"
#include "stub_log.hpp"

static int failures = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      fprintf(stderr, "FAILED at line %d: %s\n", __LINE__, #cond);         \
      ++failures;                                                          \
    }                                                                      \
  } while (0)

// Distinct, suitably aligned stand-ins for device pointers (never dereferenced).
static void* fake(uintptr_t slot) { return reinterpret_cast<void*>((slot + 1) << 20); }

struct Shape {
  int L, H, G, d, rows, B;
  int64_t total, longest;   // cached rows, and the length the caller declares
  int dtype;
};

struct Problem {
  jacap_config c;
  jacap_batch b;
  jacap_attention a;
};

static Problem make(const Shape& s) {
  Problem p;
  memset(&p, 0, sizeof(p));
  p.c.num_layers = s.L;
  p.c.num_kv_heads = s.H;
  p.c.num_q_heads = s.H * s.G;
  p.c.head_dim = s.d;
  p.c.window = s.rows;
  p.c.temperature = 1.0f;
  p.c.dtype = s.dtype;
  p.b.num_seqs = s.B;
  p.b.max_seq_len = (int32_t)s.longest;
  p.b.total_tokens = s.total;
  p.b.seq_offsets = (const int32_t*)fake(50);
  p.b.k_stride_token = p.b.v_stride_token = s.d;
  p.b.k_stride_head = p.b.v_stride_head = s.total * s.d;
  p.b.k_stride_layer = p.b.v_stride_layer = s.total * s.d * s.H;
  p.b.q_stride_pos = p.b.out_stride_row = s.d;
  p.b.q_stride_head = (int64_t)s.rows * s.d;
  p.b.q_stride_layer = p.b.q_stride_head * s.H * s.G;
  p.b.q_stride_seq = p.b.q_stride_layer * s.L;
  p.a.scale = 0.125f;
  p.a.decay = 1.0f;
  p.a.dk_stride_row = p.a.dv_stride_row = p.a.o_stride_pos = s.d;
  p.a.o_stride_head = p.b.q_stride_head;
  p.a.o_stride_layer = p.b.q_stride_layer;
  p.a.o_stride_seq = p.b.q_stride_seq;
  return p;
}

static jacap_status attend(const Problem& p, size_t ws) {
  return jacap_attend(&p.c, &p.b, &p.a, fake(1), fake(2), fake(3), fake(4), fake(5), fake(6), (float*)fake(7),
                      (float*)fake(8), (float*)fake(9), fake(1000), ws, nullptr);
}
static jacap_status weights(const Problem& p, size_t ws) {
  return jacap_attn_weights(&p.c, &p.b, &p.a, fake(1), fake(2), nullptr, (float*)fake(7), (float*)fake(8),
                            fake(1000), ws, nullptr);
}

// The cut of the sums covers the longest sequence, in grids that a launch takes.
static void check_sum(const jacap::WeightsSpace& w, int64_t n, int64_t units) {
  const int64_t tokens = w.held ? w.held : 64 * w.tiles;
  EXPECT(tokens > 0 && (int64_t)w.blocks * tokens >= n);
  EXPECT(w.row_splits >= 1 && units * std::max(1, w.blocks) * w.row_splits < (1 << 24));
}

static void run(const Shape& s) {
  const int64_t n = std::min(s.longest, s.total), U = (int64_t)s.B * s.L * s.H, R = (int64_t)s.G * s.rows;
  for (int accumulate = 0; accumulate < 2; ++accumulate) {
    Problem p = make(s);
    p.a.accumulate = accumulate;
    size_t ws = 0;
    const jacap_status st = jacap_attend_workspace_size(&p.c, &p.b, &p.a, &ws);
    EXPECT(st == (s.rows <= 512 ? JACAP_OK : JACAP_ERR_UNSUPPORTED));
    if (st != JACAP_OK) break;
    EXPECT(ws > 0 && ws % 256 == 0);
    stub::reset_attention();
    EXPECT(attend(p, ws - 1) == JACAP_ERR_WORKSPACE && stub::attention_calls[stub::kAttend] == 0);
    EXPECT(attend(p, ws) == JACAP_OK && stub::attention_calls[stub::kAttend] == 1);
    const jacap::AttendSpace& w = stub::attend;
    EXPECT(stub::attention.base.geo.maxn == n);
    const size_t pieces = w.rw ? (size_t)((int64_t)s.L * s.H * w.places * R) : (size_t)2 * w.spans * 16 * w.mt;
    EXPECT(w.before >= 4 && w.lse >= w.before + 4 * (size_t)(s.B + 1) && w.ml >= w.lse + 4 * (size_t)(U * R));
    EXPECT(w.part >= w.ml + 8 * pieces && w.z >= w.part + 4 * pieces * s.d && w.total <= ws);
    if (w.keep)
      EXPECT(w.zd >= w.z + 64 * (size_t)s.L * s.H * (size_t)(s.total / 16 + s.B + 1) * R &&
             w.total >= w.zd + 4 * (size_t)(U * R * s.rows));
    if (w.rw) {
      EXPECT((int64_t)w.chunk * w.splits >= n && 32 * w.rw * w.row_blocks >= R);
      // room for the chunks of any sequences, whatever their lengths; no more than they need
      EXPECT(w.splits == 1 || w.places >= s.total / w.chunk + s.B);
      EXPECT(w.ml + 4096 + (size_t)(s.total / w.chunk + s.B) * s.L * s.H * R * (8 + 4 * s.d) >= w.z);
    }
    if (!w.rw) EXPECT(w.spans >= 1 && 16 * w.mt * w.row_blocks >= R);
    const bool sums = accumulate && !w.keep;
    EXPECT(stub::attention_calls[stub::kDraftSum] == sums);
    EXPECT(stub::attention_calls[stub::kSum] == (sums && s.total > 0));
    if (sums && s.total > 0) check_sum(stub::sum, n, U);
  }
  Problem p = make(s);
  p.a.causal = 1;
  size_t ws = 0;
  EXPECT(jacap_attn_weights_workspace_size(&p.c, &p.b, &p.a, &ws) == JACAP_OK);
  stub::reset_attention();
  EXPECT(weights(p, ws - 1) == JACAP_ERR_WORKSPACE && stub::attention_calls[stub::kLse] == 0);
  EXPECT(weights(p, ws) == JACAP_OK);
  EXPECT(stub::attention_calls[stub::kLse] == 1 && stub::attention_calls[stub::kSum] == 1);
  const jacap::WeightsSpace& w = stub::lse;
  EXPECT((int64_t)w.chunk * w.chunks >= n && 16 * (int64_t)w.mt * w.row_blocks >= R);
  EXPECT(w.ml >= w.lse + 4 * (size_t)(U * R) && w.total <= ws);
  EXPECT(w.chunks == 1 || w.total >= w.ml + 8 * (size_t)(U * R) * w.chunks);
  EXPECT(w.row_splits == 1 || w.lse >= w.part + 4 * (size_t)w.row_splits * s.L * s.H * s.total);
  check_sum(stub::sum, n, U);

  // the evictions
  for (int budget : {0, 1, 300}) {
    p.c.budget_k = budget;
    p.b.out_stride_head = (int64_t)budget * s.d;
    stub::reset();
    stub::reset_attention();
    EXPECT(jacap_evict_weighted(&p.c, &p.b, &p.a, (float*)fake(1), fake(2), fake(3), (int32_t*)fake(4), fake(5),
                                fake(6), (float*)fake(7), nullptr) == JACAP_OK);
    EXPECT(stub::attention_calls[stub::kCompactWeighted] == (budget > 0) && stub::calls[stub::kSelect] == (budget > 0));
    EXPECT(jacap_evict_weighted_workspace_size(&p.c, &p.b, &p.a, &ws) == JACAP_OK);
    EXPECT(ws >= 256 + 4 * (size_t)U * budget);
    const int32_t cap = (int32_t)std::max<int64_t>(0, s.longest - budget);
    EXPECT(jacap_evict_weighted_slots(&p.c, &p.b, &p.a, (float*)fake(1), (int32_t*)fake(2), cap, fake(1000), ws,
                                      nullptr) == JACAP_OK);
    EXPECT(jacap_evict_weighted_slots(&p.c, &p.b, &p.a, (float*)fake(1), (int32_t*)fake(2), cap, fake(1000), ws - 1,
                                      nullptr) == JACAP_ERR_WORKSPACE);
    EXPECT(jacap_evict_weighted_slots(&p.c, &p.b, &p.a, (float*)fake(1), (int32_t*)fake(2), cap - 1, fake(1000), ws,
                                      nullptr) == JACAP_ERR_INVALID_ARG);
  }
}

static void run_invalid() {
  const Shape base = {2, 2, 2, 128, 8, 2, 4000, 3000, JACAP_DTYPE_BF16};
  auto one = [&](jacap_status want, const Problem& p, int line) {
    stub::reset_attention();
    size_t ws = 0;
    const jacap_status a = jacap_attend_workspace_size(&p.c, &p.b, &p.a, &ws), b = attend(p, (size_t)1 << 40);
    if (a != want || b != want) {
      fprintf(stderr, "line %d: want %d got %d / %d\n", line, want, a, b);
      ++failures;
    }
    for (int i = 0; i < stub::kNumAttention && want != JACAP_OK; ++i) EXPECT(stub::attention_calls[i] == 0);
  };
#define CASE(want, mutate) do { Problem p = make(base); mutate; one(want, p, __LINE__); } while (0)
  CASE(JACAP_OK, (void)0);
  CASE(JACAP_ERR_INVALID_ARG, p.a.scale = 0.0f);
  CASE(JACAP_ERR_INVALID_ARG, p.a.scale = 3e38f);               // infinite in powers of two
  CASE(JACAP_ERR_INVALID_ARG, p.a.scale = __builtin_nanf(""));
  CASE(JACAP_ERR_INVALID_ARG, p.a.decay = -0.5f);
  CASE(JACAP_ERR_INVALID_ARG, p.a.decay = __builtin_nanf(""));
  CASE(JACAP_ERR_INVALID_ARG, p.a.accumulate = 2);
  CASE(JACAP_ERR_INVALID_ARG, p.a.causal = -1);
  CASE(JACAP_ERR_INVALID_ARG, p.a.live_lens = (const int32_t*)((char*)fake(3) + 2));
  CASE(JACAP_ERR_INVALID_ARG, p.a.tree = (const uint64_t*)((char*)fake(3) + 4));
  CASE(JACAP_ERR_INVALID_ARG, p.a.dk_stride_row = 120);
  CASE(JACAP_ERR_INVALID_ARG, p.a.dv_stride_head = -8);
  CASE(JACAP_ERR_INVALID_ARG, p.a.o_stride_seq = 4);
  CASE(JACAP_ERR_UNSUPPORTED, p.a.dv_stride_row = ((int64_t)1 << 24) + 8);
  CASE(JACAP_ERR_UNSUPPORTED, p.c.window = 513);
  CASE(JACAP_ERR_INVALID_ARG, p.b.max_seq_len = -1);
  CASE(JACAP_ERR_INVALID_ARG, p.b.total_tokens = -1);
  CASE(JACAP_ERR_UNSUPPORTED, p.b.total_tokens = INT32_MAX);    // positions past the last step's end
  CASE(JACAP_ERR_UNSUPPORTED, p.b.total_tokens = (int64_t)INT32_MAX + 1);
  CASE(JACAP_ERR_UNSUPPORTED, (p.c.num_q_heads = 1 << 30, p.c.num_kv_heads = 1, p.c.window = 512));
  CASE(JACAP_ERR_UNSUPPORTED, (p.c.num_q_heads = 1 << 21, p.c.num_kv_heads = 1, p.c.window = 512,
                               p.b.total_tokens = 2000000000, p.b.max_seq_len = INT32_MAX));
  // many rows: the counts of the weights alone
  Problem p = make(base);
  size_t ws = 0;
  p.c.num_kv_heads = 1;
  p.c.window = INT32_MAX;
  EXPECT(jacap_attn_weights_workspace_size(&p.c, &p.b, &p.a, &ws) == JACAP_ERR_UNSUPPORTED);
  p.c.window = 1 << 29;
  p.c.num_q_heads = 1;
  p.b.total_tokens = 2000000000;
  p.b.max_seq_len = INT32_MAX;
  EXPECT(jacap_attn_weights_workspace_size(&p.c, &p.b, &p.a, &ws) == JACAP_ERR_UNSUPPORTED);
  EXPECT(jacap_attend_workspace_size(&p.c, &p.b, nullptr, &ws) == JACAP_ERR_INVALID_ARG);
  EXPECT(jacap_attend_workspace_size(&p.c, nullptr, &p.a, &ws) == JACAP_ERR_INVALID_ARG);
  EXPECT(jacap_attend_workspace_size(nullptr, &p.b, &p.a, &ws) == JACAP_ERR_INVALID_ARG);
  EXPECT(jacap_attend_workspace_size(&p.c, &p.b, &p.a, nullptr) == JACAP_ERR_INVALID_ARG);
}

int main() {
  const int bf = JACAP_DTYPE_BF16, fp = JACAP_DTYPE_FP32;
  const Shape shapes[] = {
      // L, H, G, d, rows, sequences, tokens, declared length
      {1, 8, 4, 128, 1, 1, 512, 512, bf},
      {1, 8, 4, 128, 1, 16, 300000, 32768, bf},
      {8, 8, 4, 128, 1, 1, 131072, 131072, bf},
      {1, 8, 4, 128, 63, 4, 62000, 16578, bf},
      {1, 8, 4, 128, 63, 64, 140000, 131072, bf},     // one long sequence among short ones
      {1, 4, 2, 64, 7, 8, 9779, 8193, fp},
      {2, 3, 7, 64, 512, 3, 1000, 900, fp},
      {4, 8, 4, 128, 64, 1, 131072, 131072, bf},
      {1, 8, 4, 128, 8192, 1, 8192, 8192, bf},
      {1, 1, 4, 64, 131072, 1, 140000, 140000, bf},
      {1, 1, 1, 64, 1, 1, 0, 0, bf},
      {1, 1, 1, 64, 40, 3, 0, 0, bf},
      {32, 8, 8, 128, 512, 2, 100, 70, bf},
      // lengths declared far beyond the tokens there are
      {1, 8, 4, 128, 1, 4, 5000, INT32_MAX, bf},
      {1, 8, 4, 128, 63, 4, 5000, INT32_MAX, bf},
      {1, 2, 4, 64, 300, 4, 5000, INT32_MAX - 1000, fp},
      {1, 1, 1, 64, 1, 1, 2000000000, INT32_MAX, bf},  // the most tokens
      {1, 1, 1, 64, 64, 1, 2000000000, 2000000000, bf},
  };
  for (const Shape& s : shapes) {
    const int before = failures;
    run(s);
    if (failures > before)
      fprintf(stderr, "  in shape L%d H%d G%d d%d rows %d seqs %d tokens %lld longest %lld\n", s.L, s.H, s.G, s.d,
              s.rows, s.B, (long long)s.total, (long long)s.longest);
  }
  run_invalid();
  if (failures) {
    fprintf(stderr, "%d failure(s)\n", failures);
    return 1;
  }
  printf("attention host layer ok under the sanitizers\n");
  return 0;
}
