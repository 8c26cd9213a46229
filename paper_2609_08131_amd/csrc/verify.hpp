// Definitions shared by the kernels and the host code of the verification of
// drafted tokens (k_verify.hip, verify_host.hip).
#pragma once

#include "jacap_internal.hpp"

namespace jacap {

constexpr int kVerifyThreads = 256;
constexpr int kRowVecs = 8;         // 16-byte pieces of a row per thread: of the rows' sums,
constexpr int kVerifyVecs = 4;      // ... and of the draw
constexpr int kMaxVerifyRows = 512;
constexpr int kMaxVocab = 1 << 24;

// What a slice of a row's logits leaves: its largest (and, greedy, the first place of it),
// and the sum of exp((z - largest) / temperature).
struct RowPart {
  float top;
  int32_t at;
  double sum;
};

struct VerifyLaunch {
  int B, S, V, dtype;
  float k;             // log2(e) / temperature; 0: greedy
  int64_t lss, lsr, qss, qsr;
  const int32_t* parents;
  const void* logits;
  const int32_t* tokens;
  const float *uniform, *draft;
  int32_t *path, *count, *next;
  float* row_weight;
  // workspace
  uint32_t* status;
  uint32_t* arrived;   // [B] slices of the draw that are summed
  double* mass;        // [B][slices]
  RowPart* parts;      // [B][S][row_slices]
  int row_slices;      // of a row's sums,
  int slices;          // ... and of the draw
  hipStream_t stream;
};

// Slices of a row of V logits: pieces of 16 bytes, one more where a row begins inside one.
inline int verify_slices(int V, int dtype, int vecs) {
  const int per = dtype == JACAP_DTYPE_BF16 ? 8 : 4;
  const int pieces = (V + 2 * (per - 1)) / per, slice = kVerifyThreads * vecs;
  return (pieces + slice - 1) / slice;
}

hipError_t launch_verify_rows(const VerifyLaunch& A);
hipError_t launch_verify(const VerifyLaunch& A);

}  // namespace jacap
