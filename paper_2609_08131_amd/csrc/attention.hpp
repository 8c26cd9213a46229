// Definitions shared by the attention kernels and their host code: attention
// of new or drafted tokens over the cache (k_attend.hip) and accumulated
// attention weights (k_attn_weights.hip).
//
// Both use one MFMA arrangement. Logits are formed transposed, S^T = K Q^T, in
// 16 x 16 tiles (16 tokens of the cache by 16 query rows): lane (m = lane % 16,
// q = lane / 16) supplies 16-byte pieces of token m's row for A and of query
// row m for B, and receives the logits of query row m for tokens 4 q .. 4 q + 3.
// Piece a of a row is its bytes 64 a + 16 q .. + 15: four lanes read 64
// contiguous bytes per load, and A and B agree on the order of the channels
// in the contraction, which is all that matters.
#pragma once

#include "jacap_internal.hpp"

namespace jacap {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kMaxDraft = 512;        // rows per query head jacap_attend takes
// Rows per KV head (G S) up to which jacap_attend keeps its logits (4 bytes a row and
// token written, then read) to accumulate from; more rows, and their keys are
// read again (256 bytes a token at d = 128, bf16) and multiplied again.
constexpr int kKeepRows = 16;
constexpr int kSpans = 512;           // workgroups the attention of few rows is cut into, of
constexpr int kSpanMin = 256;         // ... at least this many tokens
constexpr int kUnitGroups = 4;        // what beginning and ending a unit costs, in groups of 4 steps
constexpr int64_t kMaxGroups = INT32_MAX / 2;  // groups of a batch
constexpr int kWideChunkMin = 256;    // tokens per workgroup of many rows, at least
constexpr int kWideRows = 32;         // more rows than these share K and V through LDS (bf16),
constexpr int kWideBlocks = 256;      // a workgroup per compute unit
constexpr int kJoinFew = 16;           // pieces of a row that one group of threads joins in turn
constexpr int kJoinRows = 1024;        // rows of a batch up to which a workgroup joins one
constexpr int kJoinTokens = 1024;     // tokens per workgroup accumulating from kept logits
// The log-sums, rows in registers: 16-row tiles per workgroup, at most, tokens,
// and workgroups (two per compute unit); with fewer than kRowsSmall tokens each, the
// batch is small.
constexpr int kRowTilesBf16 = 8, kRowTilesFp32 = 2;
constexpr int kRowsChunk = 16384, kRowsChunkMin = 256, kRowsBlocks = 512, kRowsSmall = 1024;
// The accumulation: 16-token tiles per wave (their keys in registers). The rows of a
// unit, up to 64 KiB of them, stay in LDS for one of kHeldBlocks stretches of the tokens;
// more are staged, and cut into parts of at least kSumRowsMin while the grid is
// below kSumBlocks workgroups.
constexpr int kSumTilesBf16 = 4, kSumTilesFp32 = 2;
constexpr int held_rows(int row_bytes) { return row_bytes <= 256 ? 256 : 128; }
constexpr int kHeldBlocks = 512;
constexpr int kSumRowsMin = 128, kSumBlocks = 1024;
constexpr int64_t kMaxTokens = INT32_MAX - (int64_t(1) << 21);  // cached rows of a (layer, KV head)
constexpr int64_t kMaxGrid = (int64_t(1) << 24) - 1;  // workgroups of 256 threads in one launch

// Device view of jacap_attention (and the launch's chunking).
struct Attn {
  float c;         // scale * log2(e): logits in powers of two
  float decay;
  int accumulate, causal;
  int R;           // rows per KV head: G * window, row r = head r / window, position r % window
  const float* row_weight;
  const uint32_t* tree;  // 32-bit words, little end first
  int tree_words;        // ... per row
  int64_t dks, dkl, dkh, dkr, dvs, dvl, dvh, dvr, os, ol, oh, op;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

// How rows of D elements of type T lie in the fragments.
template <typename T, int D>
struct Row {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kBytes = D * sizeof(T);
  static constexpr int kPieces = kBytes / 64;           // 16-byte pieces per lane of a K or Q row
  static constexpr int kTiles = kBf16 ? 2 : 1;          // 16-token tiles per step: what one MFMA
                                                        // of P V contracts (32 bf16; 4 x 4 fp32)
  static constexpr int kStep = 16 * kTiles;
  static constexpr int kVBytes = kBytes / 16 < 16 ? kBytes / 16 : 16;  // V bytes per load and lane
  static constexpr int kVec = kVBytes / (int)sizeof(T);  // channels per load
  static constexpr int kVLoads = kBytes / 16 / kVBytes;  // loads per V row and lane
  static constexpr int kVWords = kVBytes / 4;
  static constexpr int kBlocks = kVLoads * kVec;         // 16-channel blocks of the output
};

// The largest of four logits as an MFMA leaves them. The middle of a, b and +inf is the
// larger of a and b (of a NaN and a number, the number). fmaxf would first quiet each
// operand that comes out of an MFMA, one instruction each, and so would this if the compiler
// knew the infinity. The maximum itself is not written as assembly: the wait states between
// an MFMA and a vector instruction that reads its result are the compiler's to insert,
// and it does so for the instructions that it knows only.
__device__ __forceinline__ float max4(const f32x4& z) {
  float inf = INFINITY;
  asm("" : "+s"(inf));
  const float a = __builtin_amdgcn_fmed3f(z[0], z[1], inf);
  return __builtin_amdgcn_fmed3f(__builtin_amdgcn_fmed3f(a, z[2], inf), z[3], inf);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 16 bytes to byte offset `off` of a buffer range; nothing past its end.
__device__ __forceinline__ void buffer_store16(__amdgpu_buffer_rsrc_t r, int32_t off, f32x4 x) {
  typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4v, x), r, off, 0, 0);
}

// The 16 x 16 logits tile of 16 tokens and 16 query rows.
template <typename T, int D>
__device__ __forceinline__ f32x4 logits(const uint4 (&k)[Row<T, D>::kPieces],
                                        const uint4 (&q)[Row<T, D>::kPieces]) {
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int a = 0; a < Row<T, D>::kPieces; ++a) {
    if constexpr (Row<T, D>::kBf16) {
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, k[a]),
                                                  __builtin_bit_cast(bf8, q[a]), z, 0, 0, 0);
    } else {
      const f32x4 kk = __builtin_bit_cast(f32x4, k[a]), qq = __builtin_bit_cast(f32x4, q[a]);
#pragma unroll
      for (int w = 0; w < 4; ++w) z = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[w], qq[w], z, 0, 0, 0);
    }
  }
  return z;
}

// Query row r of a unit's rows (pieces of lane group qg), zeros where it is not
// used; r < R in any case. No branch: one on the lane's row would take the
// unit's addresses out of the scalar registers.
template <typename T, int D>
__device__ __forceinline__ void load_row(const Geo& g, const T* qu, int r, bool used, int qg,
                                         uint4 (&f)[Row<T, D>::kPieces]) {
  const int head = r / g.w, p = r - head * g.w;
  const char* src = reinterpret_cast<const char*>(qu + head * g.qsh + p * g.qsp) + 16 * qg;
#pragma unroll
  for (int a = 0; a < Row<T, D>::kPieces; ++a) {
    const uint4 x = *reinterpret_cast<const uint4*>(src + 64 * a);
    f[a] = used ? x : uint4{0, 0, 0, 0};
  }
}

// First query row of a unit's G heads.
template <typename T>
__device__ __forceinline__ const T* unit_queries(const Geo& g, const Unit& un, const T* q) {
  return q + un.b * g.qss + un.l * g.qsl + (int64_t)un.h * g.G * g.qsh;
}

// The status word: bad offsets or lengths of any sequence. Called by every
// thread of one workgroup.
__device__ __forceinline__ void write_status(const Geo& g, uint32_t* status) {
  int bad = 0;
  for (int b = threadIdx.x; b < g.B; b += kThreads) {
    const int32_t a = g.seq_off[b], e = g.seq_off[b + 1];
    const bool ok = offsets_ok(g, a, e);
    bad |= !ok || !live_ok(g, b, e - a);
  }
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) *status = bad ? (uint32_t)JACAP_FLAG_BAD_OFFSETS : 0u;
}

// A softmax's part holds the maximum its weights refer to (in powers of two) and
// their sum. Before its first logit the maximum is the lowest finite number, so
// that neither -inf - (-inf) nor a test for it arises: exp2(-inf - ref) and
// exp2(ref - larger) are 0. It is raised only when a logit exceeds it by more
// than kLazyMax, so most steps rescale nothing; the weights stay below 2^8, far
// inside fp32 and bf16.
// A logit of +inf raises it to kTop only, so that its own weight is infinite, not NaN: the sum
// and its logarithm are then +inf, as the formula has them.
constexpr float kNoMax = -3.402823466e+38f, kTop = -kNoMax;
constexpr float kLazyMax = 8.0f;

// ---------------------------------------------------------------------------
// Workspaces (byte offsets; the status word at 0) and launchers
// ---------------------------------------------------------------------------
struct AttendSpace {
  int mt;              // 16-row tiles per workgroup,
  int spans;           // ... and workgroups; or
  int rw;              // waves of 32 rows that share the cache through LDS (0: none do),
  int chunk, splits;   // ... with tokens per workgroup, chunks of the longest sequence
  int places;          // ... and pieces of a row of a (layer, KV head), at most
  int row_blocks;
  size_t before;       // int32 [B + 1]             groups of tokens before each sequence
  size_t ml;           // float2 [pieces]           (maximum, sum) of a row's piece
  size_t part;         // float  [pieces][D]        its unnormalised output; the pieces:
                       // [2 spans][16 mt], or [L][H][places R], a sequence's [R][its pieces]
  size_t lse;          // float  [U][R]
  size_t z;            // float  [L][H][tiles][R][16] kept logits (accumulating from few rows)
  size_t zd;           // float  [U][R][S]          ... and the drafted tokens'
  size_t total;
  bool keep;           // logits are kept
};

struct WeightsSpace {
  int chunk, chunks, mt, row_blocks;  // the log-sums: rows in registers
  int tiles;           // the sums: 16-token tiles per wave, keys in registers
  int held;            // rows that stay in LDS: tokens per workgroup (else 0)
  int blocks;          // token blocks of the longest sequence
  int row_splits;      // parts the rows of the sums are cut into
  size_t ml;           // float2 [U][R][chunks]
  size_t lse;          // float [U][R]
  size_t part;         // float [row_splits][L][H][T]
  size_t total;
};

struct AttnLaunch {
  Launch base;
  Attn at;
};

hipError_t launch_attend(const AttnLaunch& A, const AttendSpace& w, const void* q, const void* k,
                         const void* v, const void* kd, const void* vd, void* out, float* lse,
                         const float* acc);
bool attend_joins(const AttnLaunch& A, const AttendSpace& w);
hipError_t launch_attend_join(const AttnLaunch& A, const AttendSpace& w, void* out, float* lse,
                              float* acc, float* acc_draft);
hipError_t launch_attn_lse(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                           const float* acc, float* lse);
// Adds the rows' weights, given their log-sums, to acc; status may be null.
hipError_t launch_attn_sum(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                           const float* lse, float* acc, uint32_t* status);
// The weights the drafted tokens received (after jacap_attend of many rows).
hipError_t launch_draft_sum(const AttnLaunch& A, const void* q, const void* kd, const float* lse,
                            float* acc_draft);

}  // namespace jacap
