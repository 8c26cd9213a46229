// Drives the host layers of the 8-bit cache (quant_host.hip) and of the verification of
// drafted tokens (verify_host.hip), built with AddressSanitizer and
// UndefinedBehaviorSanitizer, against stand-ins for their launchers (below, and those of
// attention_stubs.cpp): no GPU is touched, and no data pointer is read. Exits non-zero on
// the first unexpected result.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

#include "quant.hpp"
#include "verify.hpp"

static int quantized, appended, attended, joined, summed, rows_launched, verified;
static jacap::QuantLaunch quant_seen;
static jacap::AttendSpace space_seen;
static jacap::AppendArgs append_seen;
static jacap::VerifyLaunch verify_seen;

namespace jacap {
hipError_t launch_quantize(const QuantLaunch& A, const void*, const void*, const float*, void*, void*, float*) {
  quant_seen = A;
  ++quantized;
  return hipSuccess;
}
hipError_t launch_append(const QuantLaunch& A, const AppendArgs& p, const void*, const void*, void*, void*, float*) {
  quant_seen = A;
  append_seen = p;
  ++appended;
  return hipSuccess;
}
hipError_t launch_attend_quant(const QuantLaunch& A, const AttendSpace& w, const void*, const void*, const void*,
                               void*, float*, const float*) {
  quant_seen = A;
  space_seen = w;
  ++attended;
  return hipSuccess;
}
int attend_quant_group(const AttnLaunch&, const AttendSpace&) { return 128; }
hipError_t launch_attend_join_groups(const AttnLaunch&, const AttendSpace&, int, void*, float*, float*, float*) {
  ++joined;
  return hipSuccess;
}
hipError_t launch_quant_sum(const QuantLaunch& A, const void*, const float*, float*, uint32_t*) {
  quant_seen = A;
  ++summed;
  return hipSuccess;
}
hipError_t launch_verify_rows(const VerifyLaunch& A) {
  verify_seen = A;
  ++rows_launched;
  return hipSuccess;
}
hipError_t launch_verify(const VerifyLaunch&) {
  ++verified;
  return hipSuccess;
}
}  // namespace jacap

static int failures = 0;
#define EXPECT(cond)                                                       \
  do {                                                                     \
    if (!(cond)) {                                                         \
      fprintf(stderr, "FAILED at line %d: %s\n", __LINE__, #cond);         \
      ++failures;                                                          \
    }                                                                      \
  } while (0)

static void* fake(uintptr_t slot) { return reinterpret_cast<void*>((slot + 1) << 20); }

struct Shape {
  int L, H, G, d, rows, B;
  int64_t total, longest;
  int block, dtype;
};

static void run(const Shape& s) {
  jacap_config c;
  jacap_batch b;
  jacap_attention a;
  jacap_quant q;
  memset(&c, 0, sizeof(c));
  memset(&b, 0, sizeof(b));
  memset(&a, 0, sizeof(a));
  memset(&q, 0, sizeof(q));
  c.num_layers = s.L;
  c.num_kv_heads = s.H;
  c.num_q_heads = s.H * s.G;
  c.head_dim = s.d;
  c.window = s.rows;
  c.temperature = 1.0f;
  c.dtype = s.dtype;
  b.num_seqs = s.B;
  b.max_seq_len = (int32_t)s.longest;
  b.total_tokens = s.total;
  b.seq_offsets = (const int32_t*)fake(50);
  b.k_stride_token = b.v_stride_token = s.d;
  b.q_stride_pos = b.out_stride_row = s.d;
  q.block = s.block;
  q.k_stride_token = q.v_stride_token = s.d;
  q.k_stride_head = q.v_stride_head = s.total * s.d;
  q.k_stride_layer = q.v_stride_layer = s.total * s.d * s.H;
  a.scale = 0.125f;
  a.decay = 1.0f;
  a.dk_stride_row = a.dv_stride_row = a.o_stride_pos = s.d;
  const int64_t n = std::min(s.longest, s.total), R = (int64_t)s.G * s.rows, U = (int64_t)s.B * s.L * s.H;
  for (int accumulate = 0; accumulate < 2; ++accumulate) {
    a.accumulate = accumulate;
    size_t ws = 0;
    EXPECT(jacap_attend_quant_workspace_size(&c, &b, &a, &q, &ws) == JACAP_OK && ws > 0 && ws % 256 == 0);
    auto call = [&](size_t bytes) {
      return jacap_attend_quant(&c, &b, &a, &q, fake(1), fake(2), fake(3), (float*)fake(4), fake(5), fake(6), fake(7),
                                (float*)fake(8), (float*)fake(9), (float*)fake(10), fake(1000), bytes, nullptr);
    };
    attended = joined = summed = 0;
    EXPECT(call(ws - 1) == JACAP_ERR_WORKSPACE && attended == 0);
    EXPECT(call(ws) == JACAP_OK && attended == 1);
    const jacap::AttendSpace& w = space_seen;
    EXPECT(w.total <= ws && quant_seen.attn.base.geo.maxn == n && quant_seen.attn.at.row_mask == s.block - 1);
    EXPECT(1 << quant_seen.q.shift == s.block && quant_seen.attn.base.geo.kst == s.d);
    const size_t pieces = w.rw ? (size_t)((int64_t)s.L * s.H * w.places * R) : (size_t)2 * w.spans * 16 * w.mt;
    EXPECT(w.part >= w.ml + 8 * pieces && w.z >= w.part + 4 * pieces * s.d);
    if (w.rw) {
      EXPECT((int64_t)w.chunk * w.splits >= n && w.chunk % 128 == 0 && 32 * w.rw * w.row_blocks >= R);
      EXPECT(w.splits == 1 || w.places >= s.total / w.chunk + s.B);
    } else {
      EXPECT(w.spans >= 1 && 16 * w.mt * w.row_blocks >= R);
    }
    if (w.keep) EXPECT(w.zd >= w.z + 64 * (size_t)s.L * s.H * (size_t)(s.total / 16 + s.B + 1) * R);
    EXPECT(summed == (accumulate && !w.keep && s.total > 0));
    EXPECT(joined == (w.whole ? w.keep : w.rw == 0 || w.splits > 1));
    EXPECT(!w.whole || (n <= 512 && w.rw == 0));
  }
  a.accumulate = 0;
  quantized = appended = summed = 0;
  EXPECT(jacap_quantize(&c, &b, &a, &q, fake(1), fake(2), (float*)fake(3), fake(4), fake(5), (float*)fake(6),
                        nullptr) == JACAP_OK && quantized == 1);
  EXPECT(quant_seen.attn.base.geo.kst == s.d && quant_seen.q.kst == s.d);
  a.live_lens = (const int32_t*)fake(60);
  EXPECT(jacap_append_quant(&c, &b, &a, &q, fake(1), fake(2), (int32_t*)fake(3), nullptr, nullptr, nullptr, 0, fake(4),
                            fake(5), (float*)fake(6), nullptr, nullptr, nullptr, nullptr, nullptr) == JACAP_OK);
  EXPECT(appended == 1 && quant_seen.attn.base.geo.live == nullptr && append_seen.slots == nullptr);
  EXPECT(jacap_attn_weights_quant(&c, &b, &a, &q, fake(1), fake(2), (float*)fake(3), (float*)fake(4), (float*)fake(5),
                                  nullptr, nullptr) == JACAP_OK && summed == 1);
  EXPECT(U > 0);
}

static void verify(int B, int S, int V, int dtype) {
  jacap_verification v;
  memset(&v, 0, sizeof(v));
  v.num_seqs = B;
  v.rows = S;
  v.vocab = V;
  v.dtype = dtype;
  v.temperature = 0.8f;
  v.l_stride_row = V;
  v.l_stride_seq = (int64_t)S * V;
  size_t ws = 0;
  EXPECT(jacap_verify_workspace_size(&v, &ws) == JACAP_OK && ws > 0);
  auto call = [&](size_t bytes) {
    return jacap_verify(&v, fake(1), (int32_t*)fake(2), (float*)fake(3), nullptr, (int32_t*)fake(4), (int32_t*)fake(5),
                        (int32_t*)fake(6), nullptr, fake(1000), bytes, nullptr);
  };
  rows_launched = verified = 0;
  EXPECT(call(ws - 1) == JACAP_ERR_WORKSPACE && rows_launched == 0);
  EXPECT(call(ws) == JACAP_OK && rows_launched == 1 && verified == 1);
  const char* base = static_cast<const char*>(fake(1000));
  const jacap::VerifyLaunch& A = verify_seen;
  const int per = dtype == JACAP_DTYPE_BF16 ? 8 : 4;
  // every piece of a row, wherever it begins inside one, is in a slice
  for (int off = 0; off < per; ++off) {
    const int64_t pieces = ((int64_t)off + V + per - 1) / per;
    EXPECT((int64_t)A.row_slices * jacap::kVerifyThreads * jacap::kRowVecs >= pieces);
    EXPECT((int64_t)A.slices * jacap::kVerifyThreads * jacap::kVerifyVecs >= pieces);
  }
  EXPECT((const char*)A.arrived >= base + 4 && (const char*)A.mass >= (const char*)(A.arrived + B));
  EXPECT((const char*)A.parts >= (const char*)(A.mass + (size_t)B * A.slices));
  EXPECT((const char*)(A.parts + (size_t)B * S * A.row_slices) <= base + ws);
}

int main() {
  const Shape shapes[] = {
      {1, 1, 1, 64, 1, 1, 64, 64, 16, 1},           {1, 8, 4, 128, 1, 1, 131072, 131072, 32, 1},
      {1, 8, 4, 128, 63, 4, 61824, 16512, 64, 1},   {4, 4, 2, 64, 31, 5, 12800, 4096, 128, 0},
      {32, 8, 4, 128, 1, 16, 65536, 8192, 32, 1},   {2, 2, 8, 128, 512, 3, 3840, INT32_MAX, 16, 1},
      {1, 2, 7, 64, 16, 900, 921600, 20000, 32, 0}, {1, 1, 4, 128, 40, 2, 0, 0, 32, 1},
      {1, 1, 1, 128, 33, 1, (1 << 30), (1 << 30), 128, 1},
  };
  for (const Shape& s : shapes)
    if (s.total > 0 || s.longest == 0) run(s);
  const int vocabularies[] = {1, 3, 8, 100, 8191, 8192, 8193, 32000, 128256, 1 << 24};
  for (int V : vocabularies)
    for (int dtype = 0; dtype < 2; ++dtype) verify(V > 1000000 ? 1 : 3, 5, V, dtype);
  verify(64, 512, 32000, 1);
  if (failures) return 1;
  printf("host layers of the 8-bit cache and the verification ok under the sanitizers\n");
  return 0;
}
