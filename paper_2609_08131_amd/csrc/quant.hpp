// Definitions shared by the kernels and host code of the 8-bit cache: e4m3 codes
// with a power-of-two scale for each block of tokens of a (layer, KV head).
//
// code * scale is exact in bf16, and gfx950 converts two codes an instruction with the
// scale's exponent added, so the values enter the bf16 matrix products as they are read.
// A K row's 16-byte piece a of lane group q (bytes 64 a + 16 q .. + 15: four lanes read 64
// contiguous bytes) makes two of a product's operands, 8 channels each; query rows are
// loaded in the same order.
#pragma once

#include "attention.hpp"

namespace jacap {

constexpr int kScaleMin = -100, kScaleMax = 119;  // exponents of a scale
constexpr float kCodeMax = 448.0f;
constexpr int kMaxAppend = kMaxDraft;             // tokens of a sequence that one call appends

// The cache as the kernels see it; its strides are in Geo (ksl .. vst, in bytes) but where
// the wide cache's are there (jacap_quantize: the members here).
struct QuantArgs {
  const uint8_t *k, *v;
  const float2* scales;  // [L][H][T >> shift]: K's, V's
  int shift;             // log2 of the tokens per scale
  int64_t ksl, ksh, kst, vsl, vsh, vst;
};

// Two codes of a word (the low or the high ones) times the scale, as packed bf16.
template <bool HIGH>
__device__ __forceinline__ uint32_t widen2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH));
}
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b, float scale) {
  return uint4{widen2<false>(a, scale), widen2<true>(a, scale), widen2<false>(b, scale), widen2<true>(b, scale)};
}

// A unit's scales for its n tokens (0 past them), 8 bytes a block.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scale_range(const QuantArgs& a, const Geo& g, const Unit& un,
                                                              int n) {
  const int64_t at = ((int64_t)un.l * g.H + un.h) * (g.T >> a.shift) + (un.t0 >> a.shift);
  return buffer_range(a.scales + at, (n + (1 << a.shift) - 1) >> a.shift << 3);
}

// Byte of a bf16 row, less 32 q, at which lane group q's operand x begins: its channels are
// 64 (x / 2) + 16 q + 8 (x % 2) .. + 7.
__host__ __device__ constexpr int quant_piece(int x) { return 128 * (x / 2) + 16 * (x % 2); }

// load_row in that order.
template <int D>
__device__ __forceinline__ void load_quant_row(const Geo& g, const __bf16* qu, int r, bool used, int qg,
                                               uint4 (&f)[D / 32]) {
  const int head = r / g.w, p = r - head * g.w;
  const char* src = reinterpret_cast<const char*>(qu + head * g.qsh + p * g.qsp) + 32 * qg;
#pragma unroll
  for (int a = 0; a < D / 32; ++a) {
    const uint4 x = *reinterpret_cast<const uint4*>(src + quant_piece(a));
    f[a] = used ? x : uint4{0, 0, 0, 0};
  }
}

struct QuantLaunch {
  AttnLaunch attn;
  QuantArgs q;
};

hipError_t launch_quantize(const QuantLaunch& A, const void* k, const void* v, const float* acc, void* kq,
                           void* vq, float* scales);
struct AppendArgs {
  const int32_t *start, *count, *rows, *slots;  // any null but one of start and slots
  int slot_cap;
  float* acc;
  const float* acc_draft;
  int32_t* start_out;
  uint32_t* status;
};
hipError_t launch_append(const QuantLaunch& A, const AppendArgs& p, const void* kd, const void* vd, void* kq,
                         void* vq, float* scales);
hipError_t launch_attend_quant(const QuantLaunch& A, const AttendSpace& w, const void* q, const void* kd,
                               const void* vd, void* out, float* lse, const float* acc);
constexpr int kQuantGroup = 128;  // tokens of a group of its spans
// Adds the rows' weights, given their log-sums, to acc; status may be null.
hipError_t launch_quant_sum(const QuantLaunch& A, const void* q, const float* lse, float* acc, uint32_t* status);

}  // namespace jacap
