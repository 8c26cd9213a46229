// jacap_quantize and jacap_append_quant: K and V written as e4m3 codes with a
// power-of-two scale for each block of tokens of a (layer, KV head).
//
//   a = the block's largest finite |x|,  scale = 2^e, e the least with a <= 448 2^e,
//   code = nearest e4m3 value of x / scale (ties to even)
//
// 448 = 1.75 x 2^8 and a = f 2^x, 1 <= f < 2, give e = x - 8, or x - 7 where f > 1.75: the
// exponent's and the mantissa's bits. x / scale is exact, the conversion the one rounding.
// Long calls are bound by their reads and writes: four bf16 sequences of 1023 to 16384 tokens, 32
// layers of 8 KV heads of 128, 6.0 GB in 1.17 ms, 5.1 TB/s, as fast as a large copy. Short ones
// by a launch and a chain of loads: 8192 tokens of one layer 14 us, 16 tokens of 32 layers 7.
#include "quant.hpp"

namespace jacap {

namespace {

constexpr int kQuantTokens = 128;  // per workgroup: the largest block
constexpr int kFewAppend = 4;      // tokens of a call up to which one wave takes a unit
constexpr uint32_t kInfBits = 0x7F800000u;

// The exponent for a block whose largest finite magnitude has these bits (fp32).
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleMin), kScaleMax);
}
__device__ __forceinline__ float scale_value(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// How rows of D elements lie over a wave: 16 bytes a lane.
template <typename T, int D>
struct Spread {
  static constexpr int kLanes = D * (int)sizeof(T) / 16;  // per row
  static constexpr int kRows = 64 / kLanes;               // per load
  static constexpr int kElems = 16 / (int)sizeof(T);      // codes per lane
};

// Element i of 16 bytes, as fp32 bits.
template <typename T>
__device__ __forceinline__ uint32_t elem_bits(const uint4& x, int i) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  if constexpr (sizeof(T) == 4) return w[i];
  return (i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16;
}

// The largest magnitude of 16 bytes (fp32 bits), and of the finite ones only.
template <typename T>
__device__ __forceinline__ uint32_t most_of(const uint4& x) {
  if constexpr (sizeof(T) == 4) {
    return max(max(x.x & 0x7FFFFFFFu, x.y & 0x7FFFFFFFu), max(x.z & 0x7FFFFFFFu, x.w & 0x7FFFFFFFu));
  } else {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    auto pair = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu); };
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(pair(x.x), pair(x.y)),
                                              __builtin_elementwise_max(pair(x.z), pair(x.w)));
    return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
  }
}
template <typename T>
__device__ __forceinline__ uint32_t most_finite_of(const uint4& x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
    const uint32_t b = elem_bits<T>(x, i) & 0x7FFFFFFFu;
    m = max(m, b < kInfBits ? b : 0u);
  }
  return m;
}

// Four values in units of the scale (inv = 1 / scale) as four codes.
template <bool ODD>
__device__ __forceinline__ uint32_t codes4(const float (&x)[4], float inv) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = __builtin_amdgcn_fmed3f(x[i] * inv, -kCodeMax, kCodeMax);
    if (ODD) y[i] = fabsf(x[i]) < INFINITY ? y[i] : NAN;
  }
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}

// 16 bytes of a row to codes at dst. ODD: some value may not be finite.
template <typename T, bool ODD>
__device__ __forceinline__ void store_codes(uint8_t* dst, const uint4& x, float inv) {
  float f[16 / sizeof(T)];
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(T); ++i) f[i] = __uint_as_float(elem_bits<T>(x, i));
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<uint32_t*>(dst) = codes4<ODD>(f, inv);
  } else {
    const float a[4] = {f[0], f[1], f[2], f[3]}, b[4] = {f[4], f[5], f[6], f[7]};
    *reinterpret_cast<uint2*>(dst) = uint2{codes4<ODD>(a, inv), codes4<ODD>(b, inv)};
  }
}

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}

}  // namespace

// A workgroup takes 128 tokens of a unit, K and V, and each wave 32 of them, held in
// registers between the maximum and the conversion: the cache is read once. Blocks of more
// than 32 tokens share their maxima through LDS.
template <typename T, int D, bool HIDES>
__global__ __launch_bounds__(kThreads) void quantize_kernel(Geo g, Attn at, QuantArgs qa, const T* k, const T* v,
                                                            const float* acc, uint8_t* kq, uint8_t* vq,
                                                            float2* scales, int chunks) {
  using S = Spread<T, D>;
  constexpr int NL = 32 / S::kRows;  // loads of 32 tokens
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int u = blockIdx.x / chunks, chunk = blockIdx.x - u * chunks;
  const Unit un = attention_unit(g, at, u);
  // Its rows, whether or not they hold tokens. A sequence whose length is not one of its rows' is
  // left as it is: its scales would be those of no token, and what its codes stand for lost.
  int rows = whole_blocks(g, at, un.b) ? __builtin_amdgcn_readfirstlane(decode_unit(g, u).n) : 0;
  if (!live_ok(g, un.b, rows)) rows = 0;
  const int c0 = chunk * kQuantTokens;
  if (c0 >= rows) return;
  __shared__ uint32_t most[2][8];
  float2* sc = scales + ((int64_t)un.l * g.H + un.h) * (g.T >> qa.shift) + ((un.t0 + c0) >> qa.shift);
  const int blocks = min(kQuantTokens, rows - c0) >> qa.shift;
  if (c0 >= un.n) {
    if (tid < blocks) sc[tid] = float2{scale_value(kScaleMin), scale_value(kScaleMin)};
    return;
  }
  const int r0 = c0 + 32 * wave, left = min(32, un.n - r0);  // the wave's tokens
  const int lr = lane / S::kLanes, piece = lane % S::kLanes;
  uint4 x[2][NL];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const T* base = (i ? v + un.l * g.vsl + un.h * g.vsh : k + un.l * g.ksl + un.h * g.ksh) +
                    (un.t0 + r0) * (i ? g.vst : g.kst);
    const int32_t st = (int32_t)((i ? g.vst : g.kst) * sizeof(T));
    const auto range = buffer_range(base, rows_bytes(left, st, D * (int)sizeof(T)));
#pragma unroll
    for (int j = 0; j < NL; ++j) x[i][j] = buffer_load16(range, (j * S::kRows + lr) * st + 16 * piece);
  }
  uint32_t takes = 0;  // bit j: row j kRows + lr is a token
#pragma unroll
  for (int j = 0; j < NL; ++j) takes |= (j * S::kRows + lr < left ? 1u : 0u) << j;
  if constexpr (HIDES) {
    const auto range = buffer_range(acc + token_row(g, un) + r0, 4 * max(0, left));
#pragma unroll
    for (int j = 0; j < NL; ++j)
      if (buffer_load_f32(range, 4 * (j * S::kRows + lr)) < 0.0f) takes &= ~(1u << j);
  }
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t m = 0;
#pragma unroll
      for (int j = half * NL / 2; j < (half + 1) * NL / 2; ++j)
        m = max(m, takes >> j & 1 ? most_of<T>(x[i][j]) : 0u);
      m = wave_max_bits(m);
      if (m >= kInfBits) {
        odd = true;
        m = 0;
#pragma unroll
        for (int j = half * NL / 2; j < (half + 1) * NL / 2; ++j)
          m = max(m, takes >> j & 1 ? most_finite_of<T>(x[i][j]) : 0u);
        m = wave_max_bits(m);
      }
      if (lane == 0) most[i][2 * wave + half] = m;
    }
  __syncthreads();
  const int per = 1 << qa.shift >> 4;  // 16-token parts of a block
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint8_t* dst = (i ? vq + un.l * qa.vsl + un.h * qa.vsh + (un.t0 + r0) * qa.vst
                      : kq + un.l * qa.ksl + un.h * qa.ksh + (un.t0 + r0) * qa.kst) +
                   piece * S::kElems;
    const int64_t st = i ? qa.vst : qa.kst;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t m = 0;
      for (int y = 0; y < per; ++y) m = max(m, most[i][((2 * wave + half) & ~(per - 1)) + y]);
      const float inv = scale_value(-scale_exponent(m));
#pragma unroll
      for (int j = half * NL / 2; j < (half + 1) * NL / 2; ++j)
        if (takes >> j & 1) {
          uint8_t* at = dst + (j * S::kRows + lr) * st;
          if (odd) store_codes<T, true>(at, x[i][j], inv);
          else store_codes<T, false>(at, x[i][j], inv);
        }
    }
  }
  if (tid < blocks) {
    uint32_t a = 0, b = 0;
    for (int y = 0; y < per; ++y) {
      a = max(a, most[0][tid * per + y]);
      b = max(b, most[1][tid * per + y]);
    }
    sc[tid] = float2{scale_value(scale_exponent(a)), scale_value(scale_exponent(b))};
  }
}

// A workgroup takes the new tokens of a unit: where each goes, the exponent its K and V
// need, the blocks' new exponents (of the block's first token here: the largest of those
// that go to it and its own), the codes of blocks whose scale has grown rounded again, and
// the tokens' codes.
// Up to kFewAppend tokens by one wave, so that more units are in flight (4096 units of one
// token: 14.8 us by four waves, 7.0 so); the chain of loads (the tokens' places, their rows and scales) is what
// such a call takes.
template <typename T, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void append_kernel(Geo g, Attn at, QuantArgs qa, AppendArgs p,
                                                         const T* kd, const T* vd, uint8_t* kq,
                                                         uint8_t* vq, float2* scales) {
  using S = Spread<T, D>;
  constexpr int GROUPS = THREADS / S::kLanes;  // groups of lanes that take a row each
  constexpr int MOST = THREADS == 64 ? kFewAppend : kMaxAppend;
  constexpr int PER = (MOST + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, S_ = g.w;
  const Unit un = decode_unit(g, blockIdx.x);
  const int rows = whole_blocks(g, at, un.b) ? un.n : 0;
  __shared__ int pos[MOST];                      // -1: not written
  __shared__ int16_t src[MOST];
  __shared__ int16_t need[2][MOST];              // exponents: the row's, then its block's new one
  __shared__ int16_t fell[2][MOST];              // how far the block's codes fall (its first token)
  const int m = p.count ? min(max(p.count[un.b], 0), S_) : S_;
  const int64_t start = p.start ? p.start[un.b] : 0;
  if (p.start_out && p.start_out != p.start && un.l == 0 && un.h == 0 && tid == 0)
    p.start_out[un.b] = (int32_t)start + m;
  if (m == 0) return;
  bool bad = false;
  float2* const sc = scales + ((int64_t)un.l * g.H + un.h) * (g.T >> qa.shift) + (un.t0 >> qa.shift);
  float2 held[PER];  // the scales of the tokens' blocks
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int j = tid + x * THREADS;
    if (j >= m) continue;
    const int64_t place = start + j;
    int64_t to = place;
    if (p.slots) to = place >= 0 && place < p.slot_cap ? p.slots[(int64_t)blockIdx.x * p.slot_cap + place] : -1;
    const int r = p.rows ? p.rows[un.b * (int64_t)S_ + j] : j;
    const bool ok = to >= 0 && to < rows && (uint32_t)r < (uint32_t)S_;
    bad |= !ok;
    if (ok) held[x] = sc[to >> qa.shift];
    pos[j] = ok ? (int)to : -1;
    src[j] = (int16_t)(ok ? r : 0);
  }
  if (p.status && bad) atomicOr(p.status, (uint32_t)JACAP_FLAG_BAD_OFFSETS);
  __syncthreads();
  const T* const base[2] = {kd + un.b * at.dks + un.l * at.dkl + un.h * at.dkh,
                            vd + un.b * at.dvs + un.l * at.dvl + un.h * at.dvh};
  const int64_t stride[2] = {at.dkr, at.dvr};
  const int grp = tid / S::kLanes, piece = tid % S::kLanes;
  auto load = [&](int job) {  // K's and V's rows of the tokens in turn
    const int i = job & 1, j = job >> 1;
    return *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(
               base[i] + (int64_t)src[j] * stride[i]) + 16 * piece);
  };
  uint4 first = {};
  for (int j0 = 0; j0 < 2 * m; j0 += GROUPS) {
    const int job = min(j0 + grp, 2 * m - 1);
    const uint4 x = load(job);
    if (j0 == 0) first = x;
    uint32_t most = most_finite_of<T>(x);
#pragma unroll
    for (int o = S::kLanes / 2; o > 0; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
    if (piece == 0) need[job & 1][job >> 1] = (int16_t)scale_exponent(most);
  }
  __syncthreads();
  // Of two tokens for one position the later is written.
  if (p.slots && m > 1) {
    uint32_t again = 0;
    for (int x = 0, j = tid; x < PER && j < m; ++x, j += THREADS)
      for (int y = j + 1; y < m; ++y)
        if (pos[y] == pos[j]) again |= 1u << x;
    __syncthreads();
    for (int x = 0, j = tid; x < PER && j < m; ++x, j += THREADS)
      if (again >> x & 1) pos[j] = -1;
    __syncthreads();
  }
  {
    // (read by all before any is written: the rows' own exponents are in `need` until then)
    int16_t e[2][PER], old[2][PER];
    bool lead[PER];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int j = tid + x * THREADS;
      if (j >= m || pos[j] < 0) continue;
      const int block = pos[j] >> qa.shift;
      const float2 s = held[x];
      lead[x] = true;
      for (int i = 0; i < 2; ++i)
        e[i][x] = old[i][x] = (int16_t)((int)(__float_as_uint(i ? s.y : s.x) >> 23 & 0xFF) - 127);
      for (int y = 0; y < m; ++y) {
        if (pos[y] < 0 || pos[y] >> qa.shift != block) continue;
        if (y < j) lead[x] = false;
        for (int i = 0; i < 2; ++i) e[i][x] = max(e[i][x], need[i][y]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int j = tid + x * THREADS;
      if (j >= m || pos[j] < 0) {
        if (j < m) fell[0][j] = fell[1][j] = 0;
        continue;
      }
      for (int i = 0; i < 2; ++i) {
        need[i][j] = e[i][x];
        fell[i][j] = (int16_t)(lead[x] ? e[i][x] - old[i][x] : 0);
      }
      if (lead[x] && (e[0][x] > old[0][x] || e[1][x] > old[1][x]))
        sc[pos[j] >> qa.shift] = float2{scale_value(e[0][x]), scale_value(e[1][x])};
    }
  }
  __syncthreads();
  uint8_t* const out[2] = {kq + un.l * qa.ksl + un.h * qa.ksh + un.t0 * qa.kst,
                           vq + un.l * qa.vsl + un.h * qa.vsh + un.t0 * qa.vst};
  const int64_t ost[2] = {qa.kst, qa.vst};
  bool grown = false;
  for (int j = 0; j < m; ++j) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int f = fell[i][j];
      if (f == 0) continue;
      grown = true;
      // codes 2^-f times as large (past 2^-126 all are 0)
      const float down = scale_value(max(-f, -126));
      uint8_t* const blk = out[i] + (int64_t)(pos[j] >> qa.shift << qa.shift) * ost[i];
      constexpr int PIECES = D / 16;
      for (int y = tid; y < PIECES << qa.shift; y += THREADS) {
        uint4* const to = reinterpret_cast<uint4*>(blk + (int64_t)(y / PIECES) * ost[i] + y % PIECES * 16);
        const uint4 x = *to;
        auto fall = [&](uint32_t w) {
          typedef float f32x2 __attribute__((ext_vector_type(2)));
          const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
          const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * down, a[1] * down, 0, false);
          return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * down, b[1] * down, lo, true);
        };
        *to = uint4{fall(x.x), fall(x.y), fall(x.z), fall(x.w)};
      }
    }
  }
  if (grown) __syncthreads();  // (the same in every thread) rows written below lie in such blocks
  for (int j0 = 0; j0 < 2 * m; j0 += GROUPS) {
    const int job = j0 + grp, i = job & 1, j = job >> 1;
    if (job >= 2 * m || pos[j] < 0) continue;
    const uint4 x = j0 == 0 ? first : load(job);
    store_codes<T, true>(out[i] + (int64_t)pos[j] * ost[i] + piece * S::kElems, x, scale_value(-need[i][j]));
    if (p.acc && i == 0 && piece == 0)
      p.acc[token_row(g, un) + pos[j]] = p.acc_draft ? p.acc_draft[(int64_t)blockIdx.x * S_ + src[j]] : 0.0f;
  }
}

// Where the next token goes, after the tokens where it replaces start, which they have read.
__global__ __launch_bounds__(kThreads) void append_start_kernel(Geo g, AppendArgs p) {
  const int b = blockIdx.x * kThreads + threadIdx.x;
  if (b >= g.B) return;
  const int m = p.count ? min(max(p.count[b], 0), g.w) : g.w;
  p.start_out[b] = (p.start ? p.start[b] : 0) + m;
}

template <typename T, int D>
static hipError_t quantize_typed(const QuantLaunch& A, const void* k, const void* v, const float* acc, void* kq,
                                 void* vq, float* scales) {
  const Geo& g = A.attn.base.geo;
  const int chunks = (g.maxn + kQuantTokens - 1) / kQuantTokens;
  if (chunks == 0) return hipSuccess;
  auto go = [&](auto kern) {
    kern<<<(unsigned)(g.U * (int64_t)chunks), kThreads, 0, A.attn.base.stream>>>(
        g, A.attn.at, A.q, (const T*)k, (const T*)v, acc, (uint8_t*)kq, (uint8_t*)vq, (float2*)scales, chunks);
  };
  if (acc) go(quantize_kernel<T, D, true>);
  else go(quantize_kernel<T, D, false>);
  return hipGetLastError();
}

hipError_t launch_quantize(const QuantLaunch& A, const void* k, const void* v, const float* acc, void* kq,
                           void* vq, float* scales) {
  const bool wide = A.attn.base.geo.D == 128;
  if (A.attn.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? quantize_typed<__bf16, 128>(A, k, v, acc, kq, vq, scales)
                : quantize_typed<__bf16, 64>(A, k, v, acc, kq, vq, scales);
  return wide ? quantize_typed<float, 128>(A, k, v, acc, kq, vq, scales)
              : quantize_typed<float, 64>(A, k, v, acc, kq, vq, scales);
}

template <typename T, int D>
static hipError_t append_typed(const QuantLaunch& A, const AppendArgs& p, const void* kd, const void* vd,
                               void* kq, void* vq, float* scales) {
  const Geo& g = A.attn.base.geo;
  auto go = [&](auto kern, int threads) {
    kern<<<(unsigned)g.U, threads, 0, A.attn.base.stream>>>(g, A.attn.at, A.q, p, (const T*)kd, (const T*)vd,
                                                            (uint8_t*)kq, (uint8_t*)vq, (float2*)scales);
  };
  if (g.w <= kFewAppend) go(append_kernel<T, D, 64>, 64);
  else go(append_kernel<T, D, kThreads>, kThreads);
  return hipGetLastError();
}

hipError_t launch_append(const QuantLaunch& A, const AppendArgs& p, const void* kd, const void* vd, void* kq,
                         void* vq, float* scales) {
  const Geo& g = A.attn.base.geo;
  const bool wide = g.D == 128;
  hipError_t e;
  if (A.attn.base.cfg->dtype == JACAP_DTYPE_BF16)
    e = wide ? append_typed<__bf16, 128>(A, p, kd, vd, kq, vq, scales)
             : append_typed<__bf16, 64>(A, p, kd, vd, kq, vq, scales);
  else
    e = wide ? append_typed<float, 128>(A, p, kd, vd, kq, vq, scales)
             : append_typed<float, 64>(A, p, kd, vd, kq, vq, scales);
  if (e != hipSuccess || !p.start_out || p.start_out != p.start) return e;
  append_start_kernel<<<(g.B + kThreads - 1) / kThreads, kThreads, 0, A.attn.base.stream>>>(g, p);
  return hipGetLastError();
}

}  // namespace jacap
