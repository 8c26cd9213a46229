// jacap_attend_quant and jacap_attn_weights_quant: attention over a cache of e4m3 codes
// with a power-of-two scale for each block of tokens, and the weights that rows of known
// lse gave its tokens.
//
//   z_ri = scale q_r . k_i,  lse_r = log sum exp(z_r.),  out_r = sum exp(z_r. - lse_r) v
//   acc_i <- decay acc_i + sum_r rw_r exp(z_ri - lse_r)
//
// The arrangement is attend_kernel's (transposed logits, O^T = V^T P^T with the logits'
// lanes as they stand, spans of equal work), the cache's values made on the way into the
// products: a 16-byte piece of a K row is two operands, and of V, whose operands are one
// channel of four tokens, the bytes of two tokens are paired by a permute before two of
// them are converted an instruction. A step is 32 tokens, attend_kernel's (see kStepTiles).
// Code times scale is exact in bf16, so fp32 queries and
// weights need not be multiplied in fp32: each is the sum of three bf16 terms (8 bits of
// its 24 each), three products of a sixteenth of the time of one fp32 product's (252 fp32
// rows, four sequences of 12001 to 16450: 359 us; attend_kernel over a wide cache 642).
//
// Long caches are bound by their read: a token over 131072, four layers of 8 KV heads, 1.08 GB:
// 162 us, 6.6 TB/s; eight sequences of 31 to 131072, 439 MB, 74 us without accumulation (5.9
// TB/s), 76 where empty slots are hidden, 95 where the logits are kept too (27 MB written).
// 512 tokens, 1 MB, take 10 us, which no read bounds.
#include "attend_shared.hpp"

namespace jacap {

namespace {

// x = a + b + c in bf16, exactly but for fp32's smallest; a NaN or infinity is a alone.
struct Split {
  __bf16 a, b, c;
};
__device__ __forceinline__ Split split3(float x) {
  Split s;
  s.a = (__bf16)x;
  const float r = x - (float)s.a;
  const bool ok = fabsf(x) < INFINITY && fabsf((float)s.a) < INFINITY;
  s.b = (__bf16)(ok ? r : 0.0f);
  s.c = (__bf16)(ok ? r - (float)s.b : 0.0f);
  return s;
}

template <typename T>
constexpr int kTerms = sizeof(T) == 2 ? 1 : 3;

// Query row r in the order of the codes' operands, each channel as its terms.
template <typename T, int D>
__device__ __forceinline__ void load_query(const Geo& g, const T* qu, int r, bool used, int qg,
                                           uint4 (&f)[kTerms<T>][D / 32]) {
  if constexpr (sizeof(T) == 2) {
    load_quant_row<D>(g, qu, r, used, qg, f[0]);
  } else {
    const int head = r / g.w, p = r - head * g.w;
    const float* src = qu + head * g.qsh + p * g.qsp + 16 * qg;
#pragma unroll
    for (int a = 0; a < D / 32; ++a) {
      bf8 t[3];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(src + quant_piece(a) / 2 + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Split s = split3(used ? x[e] : 0.0f);
          t[0][4 * h + e] = s.a;
          t[1][4 * h + e] = s.b;
          t[2][4 * h + e] = s.c;
        }
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) f[i][a] = __builtin_bit_cast(uint4, t[i]);
    }
  }
}

// The 16 x 16 logits of 16 tokens (this lane: pieces of token m's codes) and 16 rows. The
// smaller terms first: their sums are added to the larger ones', not lost in them one by one.
template <int TERMS, int D>
__device__ __forceinline__ f32x4 quant_logits(const uint4 (&k)[D / 64], float scale,
                                              const uint4 (&q)[TERMS][D / 32]) {
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
  uint4 op[D / 32];
#pragma unroll
  for (int a = 0; a < D / 64; ++a) {
    op[2 * a] = widen8(k[a].x, k[a].y, scale);
    op[2 * a + 1] = widen8(k[a].z, k[a].w, scale);
  }
#pragma unroll
  for (int i = TERMS - 1; i >= 0; --i)
#pragma unroll
    for (int a = 0; a < D / 32; ++a)
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, op[a]), __builtin_bit_cast(bf8, q[i][a]),
                                                  z, 0, 0, 0);
  return z;
}

template <typename T>
struct QuantParams {
  Geo g;
  Attn at;
  AttendArgs<T> p;
  QuantArgs qa;
  int row_blocks;
  int whole;  // a workgroup per unit and row block
};

// 16-token tiles of a step (a token over 131072, four layers: 162 us with 2 tiles, 176 with 4).
constexpr int kStepTiles = 2;

}  // namespace

template <typename T, int D, int MT, Mode MODE>
__global__ __launch_bounds__(kThreads, 2) void attend_quant_kernel(QuantParams<T> params) {
  using W = Row<T, D>;
  constexpr int NT = kStepTiles, STEP = 16 * NT, GROUP = kQuantGroup, TERMS = kTerms<T>;
  static_assert(GROUP == 4 * STEP);
  constexpr int CH = D / 16, VW = D / 64;  // channels of V per lane and token, words of codes
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per_seq = params.g.L * params.g.H * params.row_blocks;  // units and row blocks of one
  __shared__ float sm[4][16 * MT], sl[4][16 * MT];
  __shared__ __align__(16) float red[4][16][D + 4];
  // The sequences' rows, 64 sequences at a time in the lanes; the first ones are kept.
  const int B = params.g.B;
  auto rows64 = [&](int b0) { return b0 + lane < B ? sequence_rows(params.g, params.at, b0 + lane) : int2{0, -1}; };
  auto groups64 = [&](const int2& x) { return x.y < 0 ? 0 : real_groups(x.y, GROUP) + kUnitGroups; };
  int2 held = rows64(0);
  int held_b = 0;
  int64_t seq_groups = 0;
  int b = 0, before = 0;  // the sequence of the span's first group, and the groups before it
  int at_group, end_group, quantum = 1, total = 0;
  if (params.whole) {
    // as if the sequence were the first one
    b = blockIdx.x / per_seq;
    held = rows64(held_b = b & ~63);
    const int c = real_groups(__builtin_amdgcn_readlane(held.y, b - held_b), GROUP);
    at_group = (blockIdx.x - b * per_seq) * (c + kUnitGroups);
    end_group = at_group + c;
  } else {
  for (int b0 = 0; b0 < B; b0 += 64)
    seq_groups += (uint32_t)__builtin_amdgcn_readlane(wave_scan(groups64(b0 == 0 ? held : rows64(b0))), 63);
  // (more than the host allowed for: offsets that go back and forth, flagged; no work)
  total = seq_groups * per_seq <= kMaxGroups ? (int)(seq_groups * per_seq) : 0;
  quantum = span_quantum(total, gridDim.x, GROUP);
  at_group = blockIdx.x * quantum;
  end_group = min(total, at_group + quantum);
  // (the groups before it are of one unit each)
  for (int b0 = 0; b0 < B; b0 += 64) {
    if (b0 > 0) held = rows64(held_b = b0);
    const int c = groups64(held), incl = before + wave_scan(c);
    const uint64_t past = __ballot(incl * per_seq > at_group);
    if (past) {
      const int j = __builtin_ctzll(past);
      b = b0 + j;
      before = __builtin_amdgcn_readlane(incl - c, j);
      break;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  }
  while (at_group < end_group) {
  // The parameters are read again for each unit, as attend_kernel reads them.
  auto args = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args));
  const QuantParams<T>& again = *(const QuantParams<T>*)args;
  const Geo& g = again.g;
  const Attn& at = again.at;
  const AttendArgs<T>& p = again.p;
  const QuantArgs& qa = again.qa;
  const int row_blocks = again.row_blocks, S = g.w, R = at.R, shift = qa.shift;
  int n, c;  // the sequence's length and groups
  for (;;) {
    if (b >= held_b + 64) held = rows64(held_b = b);
    n = __builtin_amdgcn_readlane(held.y, b - held_b);
    c = real_groups(n, GROUP);
    if (at_group < (before + c + kUnitGroups) * per_seq) break;
    before += c + kUnitGroups;
    ++b;
  }
  const int run = c + kUnitGroups, in_seq = at_group - before * per_seq;
  const int vu = in_seq / run, from = in_seq - vu * run, len = min(run - from, end_group - at_group);
  const int first_group = at_group;
  at_group += len;
  if (from >= c) continue;
  const int lh = row_blocks == 1 ? vu : vu / row_blocks, rb = vu - lh * row_blocks;
  const int u = b * g.L * g.H + lh;
  const Unit un = {b, lh / g.H, lh % g.H, 0, __builtin_amdgcn_readlane(held.x, b - held_b), n};
  const bool drafts = from + len >= c, whole = from == 0 && drafts;
  const int t0 = from * GROUP, t1 = min(n, (from + len) * GROUP);
  const int64_t piece = 2 * (int64_t)blockIdx.x + (first_group != (int)blockIdx.x * quantum);

  // The query rows (lane: row m of each tile).
  uint4 qf[MT][TERMS][D / 32];
  int row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    row[i] = (rb * MT + i) * 16 + m;
    load_query<T, D>(g, unit_queries(g, un, p.q), min(row[i], R - 1), row[i] < R, qg, qf[i]);
  }
  f32x4 o[MT][CH];
  float ref[MT], l[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    ref[i] = kNoMax;
    l[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < CH; ++j) o[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const uint8_t* kb = qa.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
  const uint8_t* vb = qa.v + un.l * g.vsl + un.h * g.vsh + un.t0 * g.vst;
  constexpr bool HIDES = MODE != kPlain;
  const float* accb = p.acc + token_row(g, un);  // read only where the call hides
  const auto sc_range = scale_range(qa, g, un, n);

  uint4 kf[NT][D / 64];
  uint32_t vr[NT][4][VW];
  constexpr int kVPolicy = MT == 1 ? kPolicyStream : kPolicyShared;
  // Codes of the rows [r0, t1), at most a step of them (zeros past the end).
  auto load_k = [&](int r0) {
    const int32_t bytes = (int32_t)g.kst;
    const auto rs = buffer_range(kb + r0 * g.kst, rows_bytes(min(STEP, t1 - r0), bytes, D));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int a = 0; a < D / 64; ++a) kf[t][a] = buffer_load16(rs, (16 * t + m) * bytes + 64 * a + 16 * qg);
  };
  auto load_v = [&](int r0) {
    const int32_t bytes = (int32_t)g.vst;
    const auto rs = buffer_range(vb + r0 * g.vst, rows_bytes(min(STEP, t1 - r0), bytes, D));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int off = (16 * t + 4 * qg + i) * bytes + CH * m;
        if constexpr (VW == 2) {
          const auto x = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, kVPolicy);
          vr[t][i][0] = x[0];
          vr[t][i][1] = x[1];
        } else {
          vr[t][i][0] = __builtin_amdgcn_raw_buffer_load_b32(rs, off, 0, kVPolicy);
        }
      }
  };
  // Scales of the step's tiles: tile lane % NT's K and V (0 past the end).
  auto load_scales = [&](int r0) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b64(sc_range, (r0 + 16 * (lane & (NT - 1))) >> shift << 3, 0, 0);
    return float2{__uint_as_float(x[0]), __uint_as_float(x[1])};
  };
  auto uniform_lane = [](float x, int i) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i));
  };
  // The accumulator entry of token r0 + lane % STEP (0 past the chunk's end): a ballot of
  // their signs is the step's hidden tokens.
  const auto acc_range = buffer_range(accb + t0, 4 * max(0, t1 - t0));
  auto load_acc = [&](int r0) { return buffer_load_f32(acc_range, 4 * (r0 - t0 + (lane & (STEP - 1)))); };
  const auto keep_range = buffer_range(p.z + keep_at(g, un, R, t0 / 16), (t1 - t0 + 15) / 16 * R * 64);
  // (rows past R: past the range's end at any step, by an addition where a choice of the
  // offset would be a branch around each store)
  const int keep_at_lane = row[0] < R ? row[0] * 64 + qg * 16 : INT32_MAX / 2;

  // The softmax's step over N tiles of logits: raises the maxima where it has to, leaves
  // the weights in z and adds them to the sums.
  auto soft = [&](auto tiles, f32x4 (&z)[MT][decltype(tiles)::value]) {
    constexpr int N = decltype(tiles)::value;
    float top[MT], over = -INFINITY;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      top[i] = z[i][0][0];
#pragma unroll
      for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) top[i] = fmaxf(top[i], z[i][t][e]);
      over = fmaxf(over, __builtin_fmaf(top[i], at.c, -ref[i]));
    }
    if (__ballot(over > kLazyMax) != 0) {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        float now = top[i] * at.c;
        now = fmaxf(now, __shfl_xor(now, 16));
        now = fmaxf(now, __shfl_xor(now, 32));
        now = fminf(fmaxf(now, ref[i]), kTop);
        const float f = exp2_fast(ref[i] - now);
        ref[i] = now;
        l[i] *= f;
#pragma unroll
        for (int j = 0; j < CH; ++j) o[i][j] *= f;
      }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float sum[N];
#pragma unroll
      for (int t = 0; t < N; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[i][t][e] = exp2_fast(__builtin_fmaf(z[i][t][e], at.c, -ref[i]));
        sum[t] = (z[i][t][0] + z[i][t][1]) + (z[i][t][2] + z[i][t][3]);
      }
#pragma unroll
      for (int x = 1; x < N; x *= 2)
#pragma unroll
        for (int t = 0; t + x < N; t += 2 * x) sum[t] += sum[t + x];
      l[i] += sum[0];
    }
  };
  // The weights of two tiles as operands, term by term.
  auto operands = [&](const f32x4& a, const f32x4& b, bf8 (&pb)[TERMS]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = e < 4 ? a[e & 3] : b[e & 3];
      if constexpr (TERMS == 1) {
        pb[0][e] = (__bf16)x;
      } else {
        const Split s = split3(x);
        pb[0][e] = s.a;
        pb[1][e] = s.b;
        pb[2][e] = s.c;
      }
    }
  };

  // A step over the codes held, of which bit j of vis says that rows may see token j.
  auto step = [&](uint32_t vis, int r0, float2 sc, auto fetch_k, auto fetch_v) {
    f32x4 z[MT][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float scale = uniform_lane(sc.x, t);
#pragma unroll
      for (int i = 0; i < MT; ++i) z[i][t] = quant_logits<TERMS, D>(kf[t], scale, qf[i]);
    }
    fetch_k();
    if (vis != ~0u) {
      // What no row sees takes no part, whatever it holds: its weight is 0 and so is its V,
      // since 0 times a NaN would not be.
      const uint32_t mine = vis >> (4 * qg);  // bit 16 t + e: token 16 t + 4 q + e
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool see = mine >> (16 * t + e) & 1;
#pragma unroll
          for (int x = 0; x < VW; ++x) vr[t][e][x] = see ? vr[t][e][x] : 0u;
#pragma unroll
          for (int i = 0; i < MT; ++i) z[i][t][e] = see ? z[i][t][e] : -INFINITY;
        }
    }
    f32x4 keep[MODE == kKeeps ? NT : 1];
    if constexpr (MODE == kKeeps) {
      // in powers of two, for the accumulation
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) keep[t][e] = z[0][t][e] * at.c;
    }
    soft(std::integral_constant<int, NT>{}, z);
#pragma unroll
    for (int t = 0; t < NT; t += 2) {
      const float s0 = uniform_lane(sc.y, t), s1 = uniform_lane(sc.y, t + 1);
      bf8 pb[MT][TERMS];
#pragma unroll
      for (int i = 0; i < MT; ++i) operands(z[i][t], z[i][t + 1], pb[i]);
#pragma unroll
      for (int w = 0; w < VW; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // channels 4 w + 2 h and the next, of tokens 0, 1 and 2, 3 of both tiles
          const uint32_t sel = h ? 0x07030602u : 0x05010400u;
          const uint32_t x0 = __builtin_amdgcn_perm(vr[t][1][w], vr[t][0][w], sel);
          const uint32_t x1 = __builtin_amdgcn_perm(vr[t][3][w], vr[t][2][w], sel);
          const uint32_t y0 = __builtin_amdgcn_perm(vr[t + 1][1][w], vr[t + 1][0][w], sel);
          const uint32_t y1 = __builtin_amdgcn_perm(vr[t + 1][3][w], vr[t + 1][2][w], sel);
          const uint4 a = {widen2<false>(x0, s0), widen2<false>(x1, s0), widen2<false>(y0, s1), widen2<false>(y1, s1)};
          const uint4 b = {widen2<true>(x0, s0), widen2<true>(x1, s0), widen2<true>(y0, s1), widen2<true>(y1, s1)};
          const int j = 4 * w + 2 * h;
#pragma unroll
          for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int s = TERMS - 1; s >= 0; --s) {
              o[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), pb[i][s], o[i][j], 0, 0, 0);
              o[i][j + 1] =
                  __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, b), pb[i][s], o[i][j + 1], 0, 0, 0);
            }
        }
    }
    fetch_v();
    if constexpr (MODE == kKeeps) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
        buffer_store16(keep_range, keep_at_lane + ((r0 - t0) / 16 + t) * R * 64, keep[t]);
    }
  };

  // A step over drafted tokens d0 .., each row seeing those of its mask only: their rows are in
  // T, and so are the products (fp32: 16 tokens, by the fp32 matrix instruction).
  auto draft_step = [&](int d0) {
    constexpr int DT = W::kTiles;
    const int rows = min(W::kStep, S - d0);
    const uint32_t vis = rows == 32 ? ~0u : (1u << rows) - 1, mine = vis >> (4 * qg);
    const T* kdb = p.kd + un.b * at.dks + un.l * at.dkl + un.h * at.dkh;
    const T* vdb = p.vd + un.b * at.dvs + un.l * at.dvl + un.h * at.dvh;
    const int32_t kbytes = (int32_t)(at.dkr * sizeof(T)), vbytes = (int32_t)(at.dvr * sizeof(T));
    const auto kr = buffer_range(kdb + d0 * at.dkr, rows_bytes(rows, kbytes, W::kBytes));
    const auto vrg = buffer_range(vdb + d0 * at.dvr, rows_bytes(rows, vbytes, W::kBytes));
    constexpr int WORDS = CH * (int)sizeof(T) / 4;  // of V per lane and token
    uint32_t vv[DT][4][WORDS];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        buffer_load_words<WORDS>(vrg, (16 * t + 4 * qg + e) * vbytes + m * CH * (int)sizeof(T), vv[t][e]);
    uint32_t mask[MT];
    f32x4 z[MT][DT];
#pragma unroll
    for (int i = 0; i < MT; ++i) mask[i] = row[i] < R ? draft_mask(at, un.b, row[i] % S, S, d0) : 0u;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      uint4 kk[W::kPieces];
#pragma unroll
      for (int a = 0; a < W::kPieces; ++a)
        kk[a] = buffer_load16(kr, (16 * t + m) * kbytes + (sizeof(T) == 2 ? 32 * qg + quant_piece(a) : 64 * a + 16 * qg));
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (sizeof(T) == 2) {
          z[i][t] = logits<T, D>(kk, qf[i][0]);
        } else {
          uint4 qq[W::kPieces];
          load_row<T, D>(g, unit_queries(g, un, p.q), min(row[i], R - 1), row[i] < R, qg, qq);
          z[i][t] = logits<T, D>(kk, qq);
        }
      }
    }
    // A drafted token that some rows see and others do not is added apart, row by row, if
    // its V holds a value that is not finite: a weight of 0 would not hide it.
    uint64_t bad[DT][4];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bool odd = false;
#pragma unroll
        for (int x = 0; x < WORDS; ++x) {
          const uint32_t y = vv[t][e][x];
          odd |= (y & 0x7F800000u) == 0x7F800000u;
          if (sizeof(T) == 2) odd |= (y & 0x7F80u) == 0x7F80u;
        }
        const bool in = mine >> (16 * t + e) & 1;
        bad[t][e] = __ballot(odd && in);
        const bool zero = !in || (bad[t][e] >> (16 * qg) & 0xFFFF) != 0;
#pragma unroll
        for (int x = 0; x < WORDS; ++x) vv[t][e][x] = zero ? 0u : vv[t][e][x];
#pragma unroll
        for (int i = 0; i < MT; ++i)
          z[i][t][e] = in && (mask[i] >> (16 * t + 4 * qg + e) & 1) ? z[i][t][e] : -INFINITY;
      }
    if constexpr (MODE == kKeeps) {
      float* dst = p.zd + ((int64_t)u * R + min(row[0], R - 1)) * S + d0;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (row[0] < R && d0 + 16 * t + 4 * qg + e < S) dst[16 * t + 4 * qg + e] = z[0][t][e] * at.c;
    }
    soft(std::integral_constant<int, DT>{}, z);
    if constexpr (sizeof(T) == 2) {
      bf8 pb[MT][TERMS];
#pragma unroll
      for (int i = 0; i < MT; ++i) operands(z[i][0], z[i][DT - 1], pb[i]);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
        uint4 a;
        a.x = __builtin_amdgcn_perm(vv[0][1][j / 2], vv[0][0][j / 2], sel);
        a.y = __builtin_amdgcn_perm(vv[0][3][j / 2], vv[0][2][j / 2], sel);
        a.z = __builtin_amdgcn_perm(vv[DT - 1][1][j / 2], vv[DT - 1][0][j / 2], sel);
        a.w = __builtin_amdgcn_perm(vv[DT - 1][3][j / 2], vv[DT - 1][2][j / 2], sel);
#pragma unroll
        for (int i = 0; i < MT; ++i)
          o[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), pb[i][0], o[i][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < MT; ++i)
            o[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vv[0][e][j % WORDS]), z[i][0][e], o[i][j], 0,
                                                           0, 0);
    }
    for (int t = 0; t < DT; ++t)
      for (int e = 0; e < 4; ++e) {
        if (bad[t][e] == 0) continue;
        for (int x = 0; x < 4; ++x) {
          if ((bad[t][e] >> (16 * x) & 0xFFFF) == 0) continue;
          const int j = 16 * t + 4 * x + e;
          const T* src = vdb + (d0 + j) * at.dvr;
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            float w = 0.0f;  // selected, not indexed: the weights stay in registers
#pragma unroll
            for (int t2 = 0; t2 < DT; ++t2)
#pragma unroll
              for (int e2 = 0; e2 < 4; ++e2) w = t2 == t && e2 == e ? z[i][t2][e2] : w;
            w = __shfl(w, 16 * x + m);
            if (!(mask[i] >> j & 1)) continue;
#pragma unroll
            for (int jj = 0; jj < CH; ++jj)
#pragma unroll
              for (int e2 = 0; e2 < 4; ++e2) o[i][jj][e2] += w * (float)src[(4 * qg + e2) * CH + jj];
          }
        }
      }
  };

  // The span's steps in turn over the waves, behind the drafted tokens'. The next step's K is
  // requested as soon as this one's has been multiplied, V likewise, into the same
  // registers: a step's loads are in flight all the time, the first one's during the
  // drafted tokens' steps.
  const int dsteps = drafts ? (S + W::kStep - 1) / W::kStep : 0;
  int r0 = t0 + ((wave - dsteps) & 3) * STEP;  // the wave's first step of the chunk
  // (requested in the order of the loop's steps: the waits before the loop and in it are for
  // the same number of later loads)
  load_k(r0);
  float2 sc = load_scales(r0);
  float a = 0.0f;
  if constexpr (HIDES) a = load_acc(r0);
  load_v(r0);
  for (int s = wave; s < dsteps; s += 4) draft_step(s * W::kStep);
  for (; r0 < t1; r0 += 4 * STEP) {
    const int next = r0 + 4 * STEP, rows = min(STEP, t1 - r0);
    uint32_t vis = rows == 32 ? ~0u : (1u << rows) - 1;
    if constexpr (HIDES) vis &= ~(uint32_t)__ballot(a < 0.0f);
    float2 then;
    step(vis, r0, sc,
         [&] {
           load_k(next);
           then = load_scales(next);
           if constexpr (HIDES) a = load_acc(next);
         },
         [&] { load_v(next); });
    sc = then;
  }

  // Join the waves: rows' maxima and sums first, then the output tile by tile.
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    l[i] += __shfl_xor(l[i], 16);
    l[i] += __shfl_xor(l[i], 32);
    if (qg == 0) {
      sm[wave][16 * i + m] = ref[i];
      sl[wave][16 * i + m] = l[i];
    }
  }
  __syncthreads();
  const int jr = tid >> 4, jc = (tid & 15) * CH;  // the joined tile's row and channels of a thread
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    float top = sm[0][16 * i + m];
    for (int x = 1; x < 4; ++x) top = fmaxf(top, sm[x][16 * i + m]);
    const float f = exp2_fast(ref[i] - top);
    if (i > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < CH; j += 4) {
        const f32x4 x = {o[i][j][e] * f, o[i][j + 1][e] * f, o[i][j + 2][e] * f, o[i][j + 3][e] * f};
        *reinterpret_cast<f32x4*>(&red[wave][m][(4 * qg + e) * CH + j]) = x;
      }
    __syncthreads();
    const int r = (rb * MT + i) * 16 + jr;
    float jt = sm[0][16 * i + jr];
    for (int x = 1; x < 4; ++x) jt = fmaxf(jt, sm[x][16 * i + jr]);
    float sum = 0.0f, val[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) val[c] = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      sum += sl[x][16 * i + jr] * exp2_fast(sm[x][16 * i + jr] - jt);
#pragma unroll
      for (int c = 0; c < CH; ++c) val[c] += red[x][jr][jc + c];
    }
    if (r < R) {
      if (whole) {
        const int head = r / S, pos = r - head * S;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        T* dst = p.out + un.b * at.os + un.l * at.ol + (int64_t)(un.h * g.G + head) * at.oh + pos * at.op + jc;
#pragma unroll
        for (int c = 0; c < CH; ++c) dst[c] = (T)(val[c] * inv);
        if (p.lse && (tid & 15) == 0)
          p.lse[(((int64_t)un.b * g.L + un.l) * g.Hq + un.h * g.G + head) * S + pos] =
              sum == 0.0f ? -INFINITY : (jt + __log2f(sum)) * kLn2;
      } else {
        const int64_t pr = piece * (16 * MT) + 16 * i + jr;
        if ((tid & 15) == 0) p.ml[pr] = float2{jt, sum};
        float* dst = p.part + pr * D + jc;
#pragma unroll
        for (int c = 0; c < CH; ++c) dst[c] = val[c];
      }
    }
  }
  __syncthreads();  // the joined tiles are read before the next unit's are written
  }
  if (blockIdx.x == gridDim.x - 1) {  // (its span is the shortest, if it has one)
    // for the join: the groups before each sequence
    if (wave == 0) {
      int sum = 0;
      for (int b0 = 0; b0 < B; b0 += 64) {
        const int incl = sum + wave_scan(groups64(rows64(b0)));
        if (b0 + lane < B) params.p.before[b0 + lane + 1] = total > 0 ? incl : 0;
        sum = __builtin_amdgcn_readlane(incl, 63);
      }
      if (lane == 0) params.p.before[0] = 0;
    }
    write_status(params.g, params.at, params.p.status);
  }
}

// ---------------------------------------------------------------------------
// The weights that rows of known lse gave the cached tokens. A workgroup lists the rows that
// count (those of weight 0, mostly a verified tree's rejected ones, are left out before any
// product) and holds the first of them as operands in LDS; then a stretch of a unit's
// tokens passes them, 64 a wave at a time. A lane's sums are of its own row and 4 tokens a tile,
// the 16 rows' joined at the end; each token's sum is one wave's, in the rows' order.
// The codes of a wave's next 64 tokens are requested when this round's products have been
// issued, into the same registers, so that only the joining of the rows' sums hides their
// latency: read and products mostly take turns (63 rows over 131072 tokens, 143 MB: 39 us, of
// which the read would take 20). In short stretches the list of rows and their operands, before
// the first product, weigh as much: the accepted rows of four trees over 12001 to 16450
// tokens, 67 MB of codes and accumulators, 18 to 21 us, of which the read would take 9.
// ---------------------------------------------------------------------------
constexpr int kSumList = 1024;          // rows listed at a time
constexpr int kSumLds = 40 * 1024;      // of operands: three workgroups to a compute unit
constexpr int kSumTokens = 256;         // of a workgroup at a time
constexpr int kQuantSumBlocks = 768;    // workgroups that the stretches are cut for

template <typename T>
struct QuantSumArgs {
  const T* q;
  const float* lse;
  float* acc;
  uint32_t* status;
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 3) void quant_sum_kernel(Geo g, Attn at, QuantArgs qa, QuantSumArgs<T> p,
                                                                int blocks, int stretch) {
  constexpr int TERMS = kTerms<T>, NT = 4, TOKENS = 16 * NT, OPS = D / 32;
  constexpr int HELD = kSumLds / (TERMS * OPS * 1024);  // 16-row tiles in LDS
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blockIdx.x == 0 && p.status) write_status(g, at, p.status);
  const int u = blockIdx.x / blocks, blk = blockIdx.x - u * blocks;
  const Unit un = attention_unit(g, at, u);
  const int s0 = blk * stretch, s1 = min(un.n, s0 + stretch);
  if (s0 >= s1) return;
  const int S = g.w, R = at.R;
  __shared__ __align__(16) uint4 ops[HELD * TERMS * OPS * 64];
  __shared__ int list[kSumList];                  // rows of weight not 0, lse not -inf
  __shared__ float2 row[kSumList];                // their lse (in powers of two), weight
  __shared__ int counts[4];
  const uint8_t* kb = qa.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
  const auto sr = scale_range(qa, g, un, un.n);
  const int64_t tr = token_row(g, un);
  uint4 kf[NT][D / 64];
  float old, scale;  // of lane's token; of tile lane % NT
  auto load = [&](int r0) {
    const int32_t bytes = (int32_t)g.kst;
    const auto rs = buffer_range(kb + r0 * g.kst, rows_bytes(min(TOKENS, s1 - r0), bytes, D));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int a = 0; a < D / 64; ++a) kf[t][a] = buffer_load16(rs, (16 * t + m) * bytes + 64 * a + 16 * qg);
    scale = buffer_load_f32(sr, (r0 + 16 * (lane & (NT - 1))) >> qa.shift << 3);
    old = buffer_load_f32(buffer_range(p.acc + tr + r0, 4 * max(0, min(TOKENS, s1 - r0))), 4 * lane);
  };
  int r0 = s0 + wave * TOKENS;
  load(r0);

  const T* qu = unit_queries(g, un, p.q);
  const float* lse = p.lse + (int64_t)u * R;
  int n = 0;  // rows listed
  auto make_list = [&](int first) {
    n = 0;
    __syncthreads();
    const int end = min(R, first + kSumList);
    for (int x = first; x < end; x += kThreads) {
      const int r = x + tid;
      float w = 0.0f, ls = 0.0f;
      if (r < end) {
        ls = lse[r];
        w = at.row_weight ? at.row_weight[(int64_t)un.b * S + r % S] : 1.0f;
      }
      const bool takes = w != 0.0f && ls != -INFINITY;
      const uint64_t mask = __ballot(takes);
      if (lane == 0) counts[wave] = __builtin_popcountll(mask);
      __syncthreads();
      int to = n;
      for (int y = 0; y < 4; ++y) {
        if (y < wave) to += counts[y];
        n += counts[y];
      }
      if (takes) {
        to += __builtin_popcountll(mask & ((1ull << lane) - 1));
        list[to] = r;
        row[to] = float2{ls * kLog2e, w};
      }
      __syncthreads();
    }
    // the last tile's padding: queries of 0 and the weight 0
    if (tid < 16 && n + tid < kSumList) row[n + tid] = float2{0.0f, 0.0f};
    for (int x = wave; x < HELD && 16 * x < n; x += 4) {
      uint4 f[TERMS][OPS];
      load_query<T, D>(g, qu, list[min(16 * x + m, n - 1)], 16 * x + m < n, qg, f);
#pragma unroll
      for (int i = 0; i < TERMS; ++i)
#pragma unroll
        for (int a = 0; a < OPS; ++a) ops[((x * TERMS + i) * OPS + a) * 64 + lane] = f[i][a];
    }
    __syncthreads();
  };
  for (int b0 = s0; b0 < s1; b0 += kSumTokens, r0 += kSumTokens) {
    float sum[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[t][e] = 0.0f;
    for (int first = 0; first < R; first += kSumList) {
      if (b0 == s0 || R > kSumList) make_list(first);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (r0 + 16 * t >= s1) continue;
        uint4 op[OPS];
        const float sc = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), t));
#pragma unroll
        for (int a = 0; a < D / 64; ++a) {
          op[2 * a] = widen8(kf[t][a].x, kf[t][a].y, sc);
          op[2 * a + 1] = widen8(kf[t][a].z, kf[t][a].w, sc);
        }
        for (int x = 0; 16 * x < n; ++x) {
          uint4 q[TERMS][OPS];
          if (x < HELD) {
#pragma unroll
            for (int i = 0; i < TERMS; ++i)
#pragma unroll
              for (int a = 0; a < OPS; ++a) q[i][a] = ops[((x * TERMS + i) * OPS + a) * 64 + lane];
          } else {
            load_query<T, D>(g, qu, list[min(16 * x + m, n - 1)], 16 * x + m < n, qg, q);
          }
          const float2 rw = row[16 * x + m];
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = TERMS - 1; i >= 0; --i)
#pragma unroll
            for (int a = 0; a < OPS; ++a)
              z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, op[a]),
                                                          __builtin_bit_cast(bf8, q[i][a]), z, 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sum[t][e] = __builtin_fmaf(rw.y, exp2_fast(__builtin_fmaf(z[e], at.c, -rw.x)), sum[t][e]);
        }
      }
    }
    const float was = old;
    const int left = s1 - r0;
    if (b0 + kSumTokens < s1) load(r0 + kSumTokens);
    // the rows' sums of each token, in every lane of its group of 16
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum[t][e] += dpp_f32<kDppQuadXor1>(sum[t][e]);
        sum[t][e] += dpp_f32<kDppQuadXor2>(sum[t][e]);
        sum[t][e] += dpp_f32<kDppHalfMirror>(sum[t][e]);
        sum[t][e] += dpp_f32<kDppMirror>(sum[t][e]);
      }
    // lane j takes token j: tile j / 16, lane group j / 4 % 4, entry j % 4
    float mine = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int e = lane & 3;
      const float x = e == 0 ? sum[t][0] : e == 1 ? sum[t][1] : e == 2 ? sum[t][2] : sum[t][3];
      const float y = __shfl(x, 16 * (lane >> 2 & 3) + e);
      mine = t == lane >> 4 ? y : mine;
    }
    if (lane < left && !(was < 0.0f))
      p.acc[tr + r0 + lane] = at.decay > 0.0f ? __builtin_fmaf(at.decay, was, mine) : mine;
  }
}

template <typename T, int D>
static hipError_t attend_quant_typed(const QuantLaunch& Q, const AttendSpace& w, const void* q, const void* kd,
                                     const void* vd, void* out, float* lse, const float* acc) {
  const AttnLaunch& A = Q.attn;
  const Geo& g = A.base.geo;
  char* ws = A.base.wsp;
  AttendArgs<T> p{(const T*)q, nullptr, nullptr, (const T*)kd, (const T*)vd, (T*)out, lse,
                  acc, ws_ptr<float2>(ws, w.ml), ws_ptr<float>(ws, w.part),
                  w.keep ? ws_ptr<float>(ws, w.z) : nullptr,
                  w.keep ? ws_ptr<float>(ws, w.zd) : nullptr, ws_ptr<uint32_t>(ws, 0),
                  ws_ptr<int32_t>(ws, w.before)};
  auto go = [&](auto kern) {
    const unsigned grid = w.whole ? (unsigned)(g.U * w.row_blocks) : w.spans;
    kern<<<grid, kThreads, 0, A.base.stream>>>(QuantParams<T>{g, A.at, p, Q.q, w.row_blocks, w.whole});
  };
  if constexpr (sizeof(T) == 2) {
    if (w.rw > 0) {
      const int64_t pairs = (int64_t)g.U * w.splits;
      const int64_t grid = w.row_blocks > 1 ? (pairs + 7) / 8 * 8 * w.row_blocks : pairs;
      auto wide = [&](auto kern, int lds) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        kern<<<(unsigned)grid, kWideThreads, lds, A.base.stream>>>(g, A.at, p, Q.q, w.chunk, w.splits,
                                                                   w.row_blocks, w.places);
        return hipGetLastError();
      };
      auto pick = [&](auto rw) {
        constexpr int RW = decltype(rw)::value;
        return acc ? wide(attend_wide_kernel<D, RW, true, true>, Wide<D, RW, true>::kLds)
                   : wide(attend_wide_kernel<D, RW, false, true>, Wide<D, RW, true>::kLds);
      };
      if (w.rw == 2) return pick(std::integral_constant<int, 2>{});
      if (w.rw == 4) return pick(std::integral_constant<int, 4>{});
      return pick(std::integral_constant<int, 8>{});
    }
  }
  if (w.keep) go(attend_quant_kernel<T, D, 1, kKeeps>);
  else if (w.mt == 1 && acc) go(attend_quant_kernel<T, D, 1, kHides>);
  else if (w.mt == 1) go(attend_quant_kernel<T, D, 1, kPlain>);
  else if (acc) go(attend_quant_kernel<T, D, 2, kHides>);
  else go(attend_quant_kernel<T, D, 2, kPlain>);
  return hipGetLastError();
}

hipError_t launch_attend_quant(const QuantLaunch& A, const AttendSpace& w, const void* q, const void* kd,
                               const void* vd, void* out, float* lse, const float* acc) {
  const bool wide = A.attn.base.geo.D == 128;
  if (A.attn.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? attend_quant_typed<__bf16, 128>(A, w, q, kd, vd, out, lse, acc)
                : attend_quant_typed<__bf16, 64>(A, w, q, kd, vd, out, lse, acc);
  return wide ? attend_quant_typed<float, 128>(A, w, q, kd, vd, out, lse, acc)
              : attend_quant_typed<float, 64>(A, w, q, kd, vd, out, lse, acc);
}

// Tokens of a workgroup of the sums: an equal part for each of kQuantSumBlocks or more, in whole
// rounds of its waves, so that all are in flight at once (the accepted rows of four trees over
// 16384 tokens: 20.7 us, 23.7 with parts rounded down and a second, small round of
// workgroups; 63 rows over 131072 39 and 47); one round where the rows are listed again for each.
static int quant_sum_stretch(const AttnLaunch& A) {
  const Geo& g = A.base.geo;
  if (A.at.R > kSumList) return kSumTokens;
  const int64_t per = ((int64_t)g.L * g.H * g.T / kQuantSumBlocks + kSumTokens) / kSumTokens * kSumTokens;
  return (int)std::min<int64_t>(std::max<int64_t>(per, kSumTokens), 1 << 20);
}

template <typename T, int D>
static hipError_t quant_sum_typed(const QuantLaunch& A, const void* q, const float* lse, float* acc,
                                  uint32_t* status) {
  const Geo& g = A.attn.base.geo;
  const int stretch = quant_sum_stretch(A.attn);
  const int blocks = std::max(1, (g.maxn + stretch - 1) / stretch);
  quant_sum_kernel<T, D><<<(unsigned)((int64_t)g.U * blocks), kThreads, 0, A.attn.base.stream>>>(
      g, A.attn.at, A.q, QuantSumArgs<T>{(const T*)q, lse, acc, status}, blocks, stretch);
  return hipGetLastError();
}

hipError_t launch_quant_sum(const QuantLaunch& A, const void* q, const float* lse, float* acc, uint32_t* status) {
  const bool wide = A.attn.base.geo.D == 128;
  if (A.attn.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? quant_sum_typed<__bf16, 128>(A, q, lse, acc, status)
                : quant_sum_typed<__bf16, 64>(A, q, lse, acc, status);
  return wide ? quant_sum_typed<float, 128>(A, q, lse, acc, status)
              : quant_sum_typed<float, 64>(A, q, lse, acc, status);
}

}  // namespace jacap
