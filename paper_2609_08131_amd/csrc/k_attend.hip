// jacap_attend: attention of the query rows of a decoding step (one new token
// or a tree of drafted tokens) over the cache and the drafted tokens.
//
//   z_ri = scale q_r . k_i,  lse_r = log sum exp(z_r.),  out_r = sum exp(z_r. - lse_r) v
//
// One pass over K and V with the running maximum and sum of a softmax. A
// workgroup takes 16 MT of the R = G S rows of a unit and a stretch of its
// tokens; its four waves take the stretch's steps in turn, each with a softmax
// of its own, and no barrier before the stretch's end, where they are joined
// in LDS. The stretches of long sequences are joined by a second kernel.
//
// P V without a transpose in LDS: the second product is also formed
// transposed, O^T = V^T P^T, and a lane's logits (query row m, tokens 4 q ..
// 4 q + 3 of each tile) are its operand of P^T as they stand, with the tokens
// in that order. The operand of V^T then is channel m of a 16-channel block
// for the same tokens, 4 q .. 4 q + 3. A lane reads kVec consecutive channels
// kVec m .. of those tokens (whole rows per 16 lanes) and calls channel
// kVec m + j row m of block j: for bf16 a byte permute per pair of values, and
// nothing at all for fp32. The result leaves each lane with 4 kVec
// consecutive channels of its own query row.
//
// Few rows are bound by the reads of K and V (one token, d = 128, 8 heads: 8 layers of
// 131072 6.9 TB/s; one of 131072 5.6 and 16 sequences of 4096 to 32768 5.2 TB/s with
// their logits kept), many by the products and the softmax's vector work in turn, which two
// waves a SIMD overlap little (252 rows, four sequences of 12001 to 16450: 84 us; MFMA busy
// 32% of the cycles, vector instructions 32%, both at once 7%).
#include "attend_shared.hpp"

namespace jacap {

// The tokens of a group: four steps.
template <typename T, int D>
constexpr int kGroup = 4 * Row<T, D>::kStep;

// 29 to 58 scalar registers (addresses and strides of the unit, read once per unit or
// step) spill to lanes of vector registers; of two fp32 tiles at d = 128, 11 vector
// registers to scratch (252 fp32 rows, four sequences of 12001 to 16450: 642 us, the
// products alone 411).
template <typename T, int D, int MT, Mode MODE>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendParams<T> params) {
  using W = Row<T, D>;
  constexpr int NT = W::kTiles, NP = W::kPieces, NL = W::kVLoads, VW = W::kVWords;
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int GROUP = kGroup<T, D>;
  const int per_seq = params.g.L * params.g.H * params.row_blocks;  // units and row blocks of one
  __shared__ float sm[4][16 * MT], sl[4][16 * MT];
  __shared__ __align__(16) float red[4][16][D + 4];
  {
    // The parameters' cache lines, requested together: the loop reads them piece by
    // piece, each piece's first read a miss of its own (8 units of 8192 tokens: 12 us, 11 so).
    auto line = [](int i) { return ((const uint32_t*)__builtin_amdgcn_kernarg_segment_ptr())[16 * i]; };
    static_assert(sizeof(AttendParams<T>) > 6 * 64 && sizeof(AttendParams<T>) <= 7 * 64, "lines");
    asm volatile("" ::"s"(line(0)), "s"(line(1)), "s"(line(2)), "s"(line(3)), "s"(line(4)), "s"(line(5)),
                 "s"(line(6)));
  }
  // The sequences' rows, 64 sequences at a time in the lanes; the first ones are kept.
  const int B = params.g.B;
  auto rows64 = [&](int b0) { return b0 + lane < B ? sequence_rows(params.g, params.at, b0 + lane) : int2{0, -1}; };
  auto groups64 = [&](const int2& x) { return x.y < 0 ? 0 : real_groups(x.y, GROUP) + kUnitGroups; };
  int2 held = rows64(0);
  int held_b = 0;
  int64_t seq_groups = 0;
  for (int b0 = 0; b0 < B; b0 += 64)
    seq_groups += (uint32_t)__builtin_amdgcn_readlane(wave_scan(groups64(b0 == 0 ? held : rows64(b0))), 63);
  // (more than the host allowed for: offsets that go back and forth, flagged; no work)
  const int total = seq_groups * per_seq <= kMaxGroups ? (int)(seq_groups * per_seq) : 0;
  const int quantum = span_quantum(total, gridDim.x, GROUP);
  int at_group = blockIdx.x * quantum;
  const int end_group = min(total, at_group + quantum);
  // the sequence of the span's first group, and the groups before it (of one unit each)
  int b = 0, before = 0;
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
  while (at_group < end_group) {
  // The parameters are read again for each unit: kept in registers over the loop,
  // they would not fit (200 scalar registers spilled to vector lanes).
  auto args = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args));
  const AttendParams<T>& again = *(const AttendParams<T>*)args;
  const Geo& g = again.g;
  const Attn& at = again.at;
  const AttendArgs<T>& p = again.p;
  const int row_blocks = again.row_blocks, S = g.w, R = at.R;
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
  uint4 qf[MT][NP];
  int row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    row[i] = (rb * MT + i) * 16 + m;
    load_row<T, D>(g, unit_queries(g, un, p.q), min(row[i], R - 1), row[i] < R, qg, qf[i]);
  }

  f32x4 o[MT][W::kBlocks];
  float ref[MT], l[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    ref[i] = kNoMax;
    l[i] = 0.0f;
#pragma unroll
    for (int b = 0; b < W::kBlocks; ++b) o[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const T* kb = p.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
  const T* vb = p.v + un.l * g.vsl + un.h * g.vsh + un.t0 * g.vst;
  constexpr bool HIDES = MODE != kPlain;
  const float* accb = p.acc + token_row(g, un);  // read only where the call hides

  uint4 kf[NT][NP];
  uint32_t vr[NT][4][NL][VW];
  // V is read in whole lines, once where the rows are one block: streamed past the
  // caches (a token over 8 layers of 131072: 6.2 TB/s without the hint, 6.9 with it).
  // K's loads take half lines and keep the default policy.
  constexpr int kVPolicy = MT == 1 ? kPolicyStream : kPolicyShared;
  // Rows [r0, end) of a K or V row range, at most a step of them (zeros past the end).
  auto load_k = [&](const T* base, int64_t stride, int r0, int end) {
    const int32_t bytes = (int32_t)(stride * sizeof(T));
    const auto rs = buffer_range(base + r0 * stride,
                                 rows_bytes(min(W::kStep, end - r0), bytes, W::kBytes));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int a = 0; a < NP; ++a) kf[t][a] = buffer_load16(rs, (16 * t + m) * bytes + 64 * a + 16 * qg);
  };
  auto load_v = [&](const T* base, int64_t stride, int r0, int end) {
    const int32_t bytes = (int32_t)(stride * sizeof(T));
    const auto rs = buffer_range(base + r0 * stride,
                                 rows_bytes(min(W::kStep, end - r0), bytes, W::kBytes));
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < NL; ++b)
          buffer_load_words<VW, kVPolicy>(rs, (16 * t + 4 * qg + i) * bytes + (16 * b + m) * W::kVBytes,
                                          vr[t][i][b]);
  };
  // The accumulator entry of token r0 + lane % kStep (0 past the chunk's end): one load
  // per step; a ballot of their signs is the step's hidden tokens.
  const auto acc_range = buffer_range(accb + t0, 4 * max(0, t1 - t0));
  auto load_acc = [&](int r0) {
    return buffer_load_f32(acc_range, 4 * (r0 - t0 + (lane & (W::kStep - 1))));
  };
  // The chunk's kept logits: its own tiles (its last step may have no second one, whose
  // room would be another's).
  const auto keep_range = buffer_range(p.z + keep_at(g, un, R, t0 / 16), (t1 - t0 + 15) / 16 * R * 64);

  // One step over the K and V rows held. vis: bit j, token j of the step is one that rows
  // may see; DRAFT: each row sees those of its mask only. `fetch_k` and
  // `fetch_v` are called where the registers of K and V have been read.
  auto step = [&](auto draft, uint32_t vis, const uint32_t (&mask)[MT], int r0, auto fetch_k,
                  auto fetch_v) {
    constexpr bool DRAFT = decltype(draft)::value;
    constexpr uint32_t ALL = W::kStep == 32 ? ~0u : (1u << (W::kStep & 31)) - 1;
    const bool masked = DRAFT || vis != ALL;
    f32x4 z[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) z[i][t] = logits<T, D>(kf[t], qf[i]);
    fetch_k();
    const uint32_t mine = vis >> (4 * qg);  // bit 16 t + e: token 16 t + 4 q + e
    uint64_t bad[NT][4] = {};               // drafted tokens with a non-finite value, by lane
    if (masked) {
      // What no row sees takes no part, whatever it holds: its weight is 0 and so is
      // its V, since 0 times a NaN or infinity would not be.
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          bool zero = !(mine >> (16 * t + e) & 1);
          if constexpr (DRAFT) {
            // ... and a drafted token that some rows see and others do not is added
            // apart, row by row, if it holds such a value.
            bool odd = false;
#pragma unroll
            for (int b = 0; b < NL; ++b)
#pragma unroll
              for (int x = 0; x < VW; ++x) {
                const uint32_t y = vr[t][e][b][x];
                odd |= (y & 0x7F800000u) == 0x7F800000u;
                if (W::kBf16) odd |= (y & 0x7F80u) == 0x7F80u;
              }
            bad[t][e] = __ballot(odd && !zero);
            zero |= (bad[t][e] >> (16 * qg) & 0xFFFF) != 0;
          }
#pragma unroll
          for (int b = 0; b < NL; ++b)
#pragma unroll
            for (int x = 0; x < VW; ++x) vr[t][e][b][x] = zero ? 0u : vr[t][e][b][x];
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            bool see = mine >> (16 * t + e) & 1;
            if constexpr (DRAFT) see = see && (mask[i] >> (16 * t + 4 * qg + e) & 1);
            z[i][t][e] = see ? z[i][t][e] : -INFINITY;
          }
        }
    }
    if constexpr (MODE == kKeeps) {
      // in powers of two, for the accumulation
      if constexpr (DRAFT) {
        float* dst = p.zd + ((int64_t)u * R + min(row[0], R - 1)) * S + r0;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (row[0] < R && r0 + 16 * t + 4 * qg + e < S) dst[16 * t + 4 * qg + e] = z[0][t][e] * at.c;
      } else {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = z[0][t][e] * at.c;
          buffer_store16(keep_range,
                         row[0] < R ? (((r0 - t0) / 16 + t) * R + row[0]) * 64 + qg * 16 : INT32_MAX - 15, x);
        }
      }
    }
    float top[MT], over = -INFINITY;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      top[i] = z[i][0][0];
#pragma unroll
      for (int t = 0; t < NT; ++t)
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
        for (int b = 0; b < W::kBlocks; ++b) o[i][b] *= f;
      }
    }
    // (a step's weights are added to each other first: one by one, the small ones would
    // be lost beside the sum)
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float sum[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[i][t][e] = exp2_fast(__builtin_fmaf(z[i][t][e], at.c, -ref[i]));
        sum[t] = (z[i][t][0] + z[i][t][1]) + (z[i][t][2] + z[i][t][3]);
      }
      l[i] += NT == 2 ? sum[0] + sum[NT - 1] : sum[0];
    }
    if constexpr (W::kBf16) {
      bf8 pb[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pb[i][e] = (__bf16)z[i][0][e];
          pb[i][4 + e] = (__bf16)z[i][NT - 1][e];
        }
#pragma unroll
      for (int j = 0; j < W::kVec; ++j) {
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
        uint4 a;
        a.x = __builtin_amdgcn_perm(vr[0][1][0][j / 2], vr[0][0][0][j / 2], sel);
        a.y = __builtin_amdgcn_perm(vr[0][3][0][j / 2], vr[0][2][0][j / 2], sel);
        a.z = __builtin_amdgcn_perm(vr[NT - 1][1][0][j / 2], vr[NT - 1][0][0][j / 2], sel);
        a.w = __builtin_amdgcn_perm(vr[NT - 1][3][0][j / 2], vr[NT - 1][2][0][j / 2], sel);
#pragma unroll
        for (int i = 0; i < MT; ++i)
          o[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), pb[i], o[i][j],
                                                            0, 0, 0);
      }
    } else {
#pragma unroll
      for (int b = 0; b < NL; ++b)
#pragma unroll
        for (int j = 0; j < W::kVec; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < MT; ++i)
              o[i][b * W::kVec + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  __uint_as_float(vr[0][e][b][j]), z[i][0][e], o[i][b * W::kVec + j], 0, 0, 0);
    }
    fetch_v();
    if constexpr (DRAFT) {
      for (int t = 0; t < NT; ++t)
        for (int e = 0; e < 4; ++e) {
          if (bad[t][e] == 0) continue;
          for (int x = 0; x < 4; ++x) {
            if ((bad[t][e] >> (16 * x) & 0xFFFF) == 0) continue;
            const int j = 16 * t + 4 * x + e;
            const T* src = p.vd + un.b * at.dvs + un.l * at.dvl + un.h * at.dvh + (r0 + j) * at.dvr;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              float w = 0.0f;  // selected, not indexed: the weights stay in registers
#pragma unroll
              for (int t2 = 0; t2 < NT; ++t2)
#pragma unroll
                for (int e2 = 0; e2 < 4; ++e2) w = t2 == t && e2 == e ? z[i][t2][e2] : w;
              w = __shfl(w, 16 * x + m);
              if (!(mask[i] >> j & 1)) continue;
#pragma unroll
              for (int b = 0; b < NL; ++b)
#pragma unroll
                for (int jj = 0; jj < W::kVec; ++jj)
#pragma unroll
                  for (int e2 = 0; e2 < 4; ++e2)
                    o[i][b * W::kVec + jj][e2] +=
                        w * (float)src[(16 * b + 4 * qg + e2) * W::kVec + jj];
            }
          }
        }
    }
  };

  // The drafted tokens' steps, then the chunk's, in turn over the waves. The next
  // step's K is requested as soon as this one's has been multiplied, V likewise,
  // into the same registers: a step's loads are in flight all the time.
  const uint32_t none[MT] = {};
  const T* kdb = p.kd + un.b * at.dks + un.l * at.dkl + un.h * at.dkh;
  const T* vdb = p.vd + un.b * at.dvs + un.l * at.dvl + un.h * at.dvh;
  const int dsteps = drafts ? (S + W::kStep - 1) / W::kStep : 0;
  int r0 = t0 + ((wave - dsteps) & 3) * W::kStep;  // the wave's first step of the chunk
  {
    const bool first = wave < dsteps;
    load_k(first ? kdb : kb, first ? at.dkr : g.kst, first ? wave * W::kStep : r0, first ? S : t1);
    load_v(first ? vdb : vb, first ? at.dvr : g.vst, first ? wave * W::kStep : r0, first ? S : t1);
  }
  float a = 0.0f;
  if constexpr (HIDES) a = load_acc(r0);
  for (int s = wave; s < dsteps; s += 4) {
    const int d0 = s * W::kStep, rows = min(W::kStep, S - d0);
    const bool more = s + 4 < dsteps;
    uint32_t mask[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) mask[i] = row[i] < R ? draft_mask(at, un.b, row[i] % S, S, d0) : 0u;
    const int next = more ? d0 + 4 * W::kStep : r0, end = more ? S : t1;
    step(std::true_type{}, rows == 32 ? ~0u : (1u << rows) - 1, mask, d0,
         [&] { load_k(more ? kdb : kb, more ? at.dkr : g.kst, next, end); },
         [&] { load_v(more ? vdb : vb, more ? at.dvr : g.vst, next, end); });
  }
  for (; r0 < t1; r0 += 4 * W::kStep) {
    const int next = r0 + 4 * W::kStep, rows = min(W::kStep, t1 - r0);
    uint32_t vis = rows == 32 ? ~0u : (1u << rows) - 1;
    if constexpr (HIDES) vis &= ~(uint32_t)__ballot(a < 0.0f);
    step(std::false_type{}, vis, none, r0,
         [&] {
           load_k(kb, g.kst, next, t1);
           if constexpr (HIDES) a = load_acc(next);
         },
         [&] { load_v(vb, g.vst, next, t1); });
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
  constexpr int PER = D / 16;  // channels per thread of the joined tile
  const int jr = tid >> 4, jc = (tid & 15) * PER;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    float top = sm[0][16 * i + m];
    for (int x = 1; x < 4; ++x) top = fmaxf(top, sm[x][16 * i + m]);
    const float f = exp2_fast(ref[i] - top);
    if (i > 0) __syncthreads();
#pragma unroll
    for (int b = 0; b < NL; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < W::kVec; j += 4) {
          const f32x4 x = {o[i][b * W::kVec + j][e] * f, o[i][b * W::kVec + j + 1][e] * f,
                           o[i][b * W::kVec + j + 2][e] * f, o[i][b * W::kVec + j + 3][e] * f};
          *reinterpret_cast<f32x4*>(&red[wave][m][(16 * b + 4 * qg + e) * W::kVec + j]) = x;
        }
    __syncthreads();
    const int r = (rb * MT + i) * 16 + jr;
    float jt = sm[0][16 * i + jr];
    for (int x = 1; x < 4; ++x) jt = fmaxf(jt, sm[x][16 * i + jr]);
    float sum = 0.0f, val[PER];
#pragma unroll
    for (int c = 0; c < PER; ++c) val[c] = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      sum += sl[x][16 * i + jr] * exp2_fast(sm[x][16 * i + jr] - jt);
#pragma unroll
      for (int c = 0; c < PER; ++c) val[c] += red[x][jr][jc + c];
    }
    if (r < R) {
      if (whole) {
        const int head = r / S, pos = r - head * S;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        T* dst = p.out + un.b * at.os + un.l * at.ol + (int64_t)(un.h * g.G + head) * at.oh +
                 pos * at.op + jc;
#pragma unroll
        for (int c = 0; c < PER; ++c) dst[c] = (T)(val[c] * inv);
        if (p.lse && (tid & 15) == 0)
          p.lse[(((int64_t)un.b * g.L + un.l) * g.Hq + un.h * g.G + head) * S + pos] =
              sum == 0.0f ? -INFINITY : (jt + __log2f(sum)) * kLn2;
      } else {
        const int64_t pr = piece * (16 * MT) + 16 * i + jr;
        if ((tid & 15) == 0) p.ml[pr] = float2{jt, sum};
        float* dst = p.part + pr * D + jc;
#pragma unroll
        for (int c = 0; c < PER; ++c) dst[c] = val[c];
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

template <typename T, int D>
static hipError_t attend_typed(const AttnLaunch& A, const AttendSpace& w, const void* q,
                               const void* k, const void* v, const void* kd, const void* vd,
                               void* out, float* lse, const float* acc) {
  const Geo& g = A.base.geo;
  char* ws = A.base.wsp;
  AttendArgs<T> p{(const T*)q, (const T*)k, (const T*)v, (const T*)kd, (const T*)vd, (T*)out, lse,
                  acc, ws_ptr<float2>(ws, w.ml), ws_ptr<float>(ws, w.part),
                  w.keep ? ws_ptr<float>(ws, w.z) : nullptr,
                  w.keep ? ws_ptr<float>(ws, w.zd) : nullptr, ws_ptr<uint32_t>(ws, 0),
                  ws_ptr<int32_t>(ws, w.before)};
  auto go = [&](auto kern) {
    kern<<<w.spans, kThreads, 0, A.base.stream>>>(AttendParams<T>{g, A.at, p, w.row_blocks});
  };
  if constexpr (sizeof(T) == 2) {
    if (w.rw > 0) {
      const int64_t pairs = (int64_t)g.U * w.splits;
      const int64_t grid = w.row_blocks > 1 ? (pairs + 7) / 8 * 8 * w.row_blocks : pairs;
      auto wide = [&](auto kern, int lds) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        kern<<<(unsigned)grid, kWideThreads, lds, A.base.stream>>>(g, A.at, p, QuantArgs{}, w.chunk, w.splits, w.row_blocks,
                                                                w.places);
        return hipGetLastError();
      };
      auto pick = [&](auto rw) {
        constexpr int RW = decltype(rw)::value;
        return acc ? wide(attend_wide_kernel<D, RW, true, false>, Wide<D, RW>::kLds)
                   : wide(attend_wide_kernel<D, RW, false, false>, Wide<D, RW>::kLds);
      };
      if (w.rw == 2) return pick(std::integral_constant<int, 2>{});
      if (w.rw == 4) return pick(std::integral_constant<int, 4>{});
      return pick(std::integral_constant<int, 8>{});
    }
  }
  if (w.keep) go(attend_kernel<T, D, 1, kKeeps>);
  else if (w.mt == 1 && acc) go(attend_kernel<T, D, 1, kHides>);
  else if (w.mt == 1) go(attend_kernel<T, D, 1, kPlain>);
  else if (acc) go(attend_kernel<T, D, 2, kHides>);
  else go(attend_kernel<T, D, 2, kPlain>);
  return hipGetLastError();
}

hipError_t launch_attend(const AttnLaunch& A, const AttendSpace& w, const void* q, const void* k,
                         const void* v, const void* kd, const void* vd, void* out, float* lse,
                         const float* acc) {
  const bool wide = A.base.geo.D == 128;
  if (A.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? attend_typed<__bf16, 128>(A, w, q, k, v, kd, vd, out, lse, acc)
                : attend_typed<__bf16, 64>(A, w, q, k, v, kd, vd, out, lse, acc);
  return wide ? attend_typed<float, 128>(A, w, q, k, v, kd, vd, out, lse, acc)
              : attend_typed<float, 64>(A, w, q, k, v, kd, vd, out, lse, acc);
}

// ---------------------------------------------------------------------------
// Second kernel: joins the chunks of each row (a workgroup per row of a unit, or per
// 1024 / d rows of few chunks: 8064 rows of 8 chunks 18.9 us at one a workgroup, 8.8 so),
// and accumulates the weights of kept logits (a workgroup per kJoinTokens
// tokens of a unit): p = exp2(z - lse) of every row, with lse joined from the
// chunks again rather than waited for.
// ---------------------------------------------------------------------------
template <typename T>
struct JoinArgs {
  T* out;
  float* lse;             // or null (not with kept logits)
  const float2* ml;
  const float* part;
  const int32_t* before;
  const float *z, *zd;    // or null
  float* acc;
  float* acc_draft;       // or null
};

// Where a row's pieces lie: `n` of them (1: the first kernel wrote the result), each
// a (maximum, sum) and an unnormalised output; piece j at row(j).
struct Pieces {
  int n, start, quantum, rows, in_block;  // spans; quantum 0: chunks, start the row's first
  __device__ __forceinline__ int64_t row(int j) const {
    return quantum ? piece_of(start, quantum, j) * rows + in_block : (int64_t)start + j;
  }
};
// spans > 0: attend_kernel's, in groups of `group` tokens and blocks of `rows` rows;
// else attend_wide_kernel's chunks.
struct JoinGeo {
  int chunk, places, spans, group, rows, row_blocks;
};
__device__ __forceinline__ Pieces pieces_of(const Geo& g, const JoinGeo& j, const int32_t* before,
                                            const Unit& un, int u, int r, int R) {
  if (j.spans == 0) {
    const int n = max(1, (un.n + j.chunk - 1) / j.chunk);
    return {n, (int)chunk_place(g, un, j.places, j.chunk, R, r, n), 0, 0, 0};
  }
  const int per_seq = g.L * g.H * j.row_blocks;
  const int q = span_quantum(before[g.B] * per_seq, j.spans, j.group);
  const int run = before[un.b + 1] - before[un.b], c = run - kUnitGroups;
  const int start = before[un.b] * per_seq + ((un.l * g.H + un.h) * j.row_blocks + r / j.rows) * run;
  return {(start + c - 1) / q - start / q + 1, start, q, j.rows, r % j.rows};
}

// ROWS: at least the rows whose logits are kept. APART: the sequences' lengths lie so far
// apart that the accumulators' blocks are those of the tokens there are.
template <typename T, int D, int ROWS, bool APART>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(Geo g, Attn at, JoinArgs<T> p,
                                                               JoinGeo jg, int few, int rows_grid,
                                                               int token_blocks) {
  const int tid = threadIdx.x, S = g.w, R = at.R;
  if ((int)blockIdx.x < rows_grid) {
    // thread: 4 channels. Few pieces: of a row of its own group of D / 4 threads, all
    // pieces in turn; many: of every NG-th piece of the workgroup's one row.
    constexpr int NG = kThreads / (D / 4);
    const int c = tid % (D / 4) * 4, grp = tid / (D / 4);
    const int64_t ur = few ? min((int64_t)blockIdx.x * NG + grp, (int64_t)g.U * R - 1) : blockIdx.x;
    const int u = ur / R, r = ur - (int64_t)u * R;
    Unit un{u / (g.L * g.H), u / g.H % g.L, u % g.H};  // (of the group, not of the workgroup)
    if (jg.spans == 0) {
      const int2 rows = sequence_rows(g, at, un.b);
      un.t0 = rows.x;
      un.n = rows.y;
    }
    const Pieces pc = pieces_of(g, jg, p.before, un, u, r, R);
    // one piece: written by the first kernel (threads of a wave may hold different rows)
    if (pc.n == 1) return;
    const int head = r / S, pos = r - head * S;
    T* out = p.out + un.b * at.os + un.l * at.ol + (int64_t)(un.h * g.G + head) * at.oh + pos * at.op;
    float* lse = p.lse + (((int64_t)un.b * g.L + un.l) * g.Hq + un.h * g.G + head) * S + pos;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float top = kNoMax, l = 0.0f;
    auto add = [&](int s) {
      const int64_t at_row = pc.row(s);
      const float2 ml = p.ml[at_row];
      const float f = exp2_fast(ml.x - top);
      l += ml.y * f;
      sum += *reinterpret_cast<const f32x4*>(p.part + at_row * D + c) * f;
    };
    if (few) {
      for (int s = c / 4; s < pc.n; s += D / 4) top = fmaxf(top, p.ml[pc.row(s)].x);
#pragma unroll
      for (int x = D / 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
#pragma unroll 8
      for (int s = 0; s < pc.n; ++s) add(s);
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[c + e] = (T)(sum[e] * inv);
      if (p.lse && c == 0) *lse = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
      return;
    }
    __shared__ float red[4];
    for (int s = tid; s < pc.n; s += kThreads) top = fmaxf(top, p.ml[pc.row(s)].x);
    top = block_combine(wave_max(top), red, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll 4
    for (int s = grp; s < pc.n; s += NG) add(s);
    __shared__ __align__(16) float so[NG][D];
    __shared__ float sl[NG];
    *reinterpret_cast<f32x4*>(&so[grp][c]) = sum;
    if (c == 0) sl[grp] = l;
    __syncthreads();
    if (tid < D) {
      float a = 0.0f, b = 0.0f;
      for (int x = 0; x < NG; ++x) {
        a += so[x][tid];
        b += sl[x];
      }
      out[tid] = (T)(b == 0.0f ? 0.0f : a / b);
      if (p.lse && tid == 0) *lse = b == 0.0f ? -INFINITY : (top + __log2f(b)) * kLn2;
    }
    return;
  }
  const int item = blockIdx.x - rows_grid;
  __shared__ float slse[kKeepRows], sw[kKeepRows];
  auto accumulate = [&](const Unit& un, int u, int blk) {
  const int t0 = blk * kJoinTokens;
  // The entries and the rows' logits are requested before the rows' lse is joined.
  // Token t0 + tid + 256 x: entry tid % 16 of tile (t0 + tid) / 16 + 16 x.
  const int64_t tr = token_row(g, un) + t0;
  const float* z = p.z + keep_at(g, un, R, t0 / 16 + tid / 16) + tid % 16;
  const int left = un.n - t0;
  constexpr int PER = kJoinTokens / kThreads;
  float old[PER], sum[PER], y[ROWS][PER];
  auto logit = [&](int r, int x) {
    return tid + x * kThreads < left ? z[x * (kThreads / 16) * R * 16 + r * 16] : -INFINITY;
  };
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    old[x] = tid + x * kThreads < left ? p.acc[tr + tid + x * kThreads] : -1.0f;
    sum[x] = 0.0f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (r < R) y[r][x] = logit(r, x);
  }
  {
    // 16 threads per row; a row of one piece has its lse already, as a sum of 1
    const int r = tid >> 4, rc = min(r, R - 1);
    const Pieces pc = pieces_of(g, jg, p.before, un, u, rc, R);
    float top = kNoMax, l = 0.0f;
    if (pc.n == 1) {
      const float ls = p.lse[(int64_t)u * R + rc] * kLog2e;
      if ((tid & 15) == 0 && ls != -INFINITY) {
        top = fminf(ls, kTop);
        l = exp2_fast(ls - top);  // 1, or as infinite or NaN as ls
      }
    } else {
      for (int s = tid & 15; s < pc.n; s += 16) {
        const float2 c = p.ml[pc.row(s)];
        const float now = fmaxf(top, c.x);
        l = l * exp2_fast(top - now) + c.y * exp2_fast(c.x - now);
        top = now;
      }
    }
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) {
      const float t = __shfl_xor(top, x), m = __shfl_xor(l, x);
      const float now = fmaxf(top, t);
      l = l * exp2_fast(top - now) + m * exp2_fast(t - now);
      top = now;
    }
    if ((tid & 15) == 0) {
      float w = 0.0f;
      if (r < R && l != 0.0f) w = at.row_weight ? at.row_weight[(int64_t)un.b * S + r % S] : 1.0f;
      sw[r] = w;
      slse[r] = l == 0.0f ? 0.0f : top + __log2f(l);
    }
  }
  __syncthreads();
  auto add = [&](int r, const float (&v)[PER]) {
    const float w = sw[r], ls = slse[r];
    if (w != 0.0f)
#pragma unroll
      for (int x = 0; x < PER; ++x) sum[x] = __builtin_fmaf(w, exp2_fast(v[x] - ls), sum[x]);
  };
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
    if (r < R) add(r, y[r]);
#pragma unroll
  for (int x = 0; x < PER; ++x)
    if (tid + x * kThreads < left && !(old[x] < 0.0f))
      p.acc[tr + tid + x * kThreads] =
          at.decay > 0.0f ? __builtin_fmaf(at.decay, old[x], sum[x]) : sum[x];
  if (blk == 0 && p.acc_draft && tid < S) {
    float sum = 0.0f;
    for (int r = 0; r < R; ++r)
      if (sw[r] != 0.0f)
        sum = __builtin_fmaf(sw[r], exp2_fast(p.zd[((int64_t)u * R + r) * S + tid] - slse[r]), sum);
    p.acc_draft[(int64_t)u * S + tid] = sum;
  }
  };
  if constexpr (!APART) {
    const int u = item / token_blocks, blk = item - u * token_blocks;
    const Unit un = attention_unit(g, at, u);
    if (blk * kJoinTokens < un.n || blk == 0) accumulate(un, u, blk);
  } else {
    // The blocks of a (layer, KV head) are its sequences' side by side, as they lie in the
    // cache: sequence b's begin behind seq_off[b] / kJoinTokens + b others, which is room for
    // the last, partial one of each. Offsets that go back and forth may put blocks of several
    // sequences here.
    const int lh = item / token_blocks, place = item - lh * token_blocks;
    __shared__ uint64_t here[kThreads / 64];  // of the sequences b0 .., those with a block here
    auto first_block = [&](int b, const int2& rows) {
      return (int)(min(max((int64_t)rows.x, (int64_t)0), g.T) / kJoinTokens) + b;
    };
    for (int b0 = 0; b0 < g.B; b0 += kThreads) {
      const int x = b0 + tid;
      const int2 rows = x < g.B ? sequence_rows(g, at, x) : int2{0, -1};
      const int first = first_block(x, rows);
      const int blocks = rows.y < 0 ? 0 : max(1, (rows.y + kJoinTokens - 1) / kJoinTokens);
      const uint64_t mask = __ballot(place >= first && place < first + blocks);
      if ((tid & 63) == 0) here[tid >> 6] = mask;
      __syncthreads();
      for (int part = 0; part < kThreads / 64; ++part)
        for (uint64_t todo = here[part]; todo; todo &= todo - 1) {
          const int b = __builtin_amdgcn_readfirstlane(b0 + 64 * part + __builtin_ctzll(todo));
          const int2 rows = sequence_rows(g, at, b);
          const Unit un = {b, lh / g.H, lh % g.H, 0, __builtin_amdgcn_readfirstlane(rows.x),
                           __builtin_amdgcn_readfirstlane(rows.y)};
          accumulate(un, b * g.L * g.H + lh, place - first_block(b, rows));
          __syncthreads();  // the rows' lse is read before another block's is written
        }
      __syncthreads();
    }
  }
}

template <typename T, int D>
static hipError_t join_typed(const AttnLaunch& A, const AttendSpace& w, int group, void* out, float* lse,
                             float* acc, float* acc_draft) {
  const Geo& g = A.base.geo;
  char* ws = A.base.wsp;
  JoinArgs<T> p{(T*)out, lse, ws_ptr<float2>(ws, w.ml), ws_ptr<float>(ws, w.part),
                ws_ptr<int32_t>(ws, w.before), w.keep ? ws_ptr<float>(ws, w.z) : nullptr,
                w.keep ? ws_ptr<float>(ws, w.zd) : nullptr, acc, acc_draft};
  const bool wide = w.rw > 0;
  const JoinGeo jg{w.whole ? INT32_MAX / 2 : w.chunk, w.places, wide || w.whole ? 0 : w.spans, group, 16 * w.mt,
                   w.row_blocks};
  // Spans of a batch of many rows hold many units each, so a row has few pieces; of
  // few rows (at most a workgroup's worth per compute unit), as many as there are spans.
  const int64_t UR = (int64_t)g.U * A.at.R;
  const int few = wide ? w.splits <= kJoinFew : UR > kJoinRows;
  const int64_t per = few ? kThreads / (D / 4) : 1;
  const int rows_grid = w.whole || (wide && w.splits == 1) ? 0 : (int)((UR + per - 1) / per);
  // A workgroup that finds its unit without tokens there costs little while others work, the
  // look for a block's sequence 1 us (a block for each of the longest, or those there are:
  // 32 units of 131072 tokens 9.6 us, 10.8; 128 units of 4096 to 32768, about 2000 workgroups
  // more, 15.1, 16.0; 8 units of 131072 beside 56 of 31 to 32768, 7000 more, 21.2, 14.6).
  const int unit_blocks = std::max(1, (g.maxn + kJoinTokens - 1) / kJoinTokens);
  const int head_blocks = (int)(g.T / kJoinTokens) + g.B;  // of a (layer, KV head)
  const bool apart = w.keep && (int64_t)g.L * g.H * ((int64_t)g.B * unit_blocks - head_blocks) > 4096;
  const int token_blocks = apart ? head_blocks : unit_blocks;
  const int64_t grid = rows_grid + (w.keep ? (int64_t)g.L * g.H * (apart ? 1 : g.B) * token_blocks : 0);
  auto go = [&](auto kern) {
    kern<<<(unsigned)grid, kThreads, 0, A.base.stream>>>(g, A.at, p, jg, few, rows_grid, token_blocks);
  };
  if (!w.keep || A.at.R <= 4) apart ? go(attend_join_kernel<T, D, 4, true>) : go(attend_join_kernel<T, D, 4, false>);
  else apart ? go(attend_join_kernel<T, D, kKeepRows, true>) : go(attend_join_kernel<T, D, kKeepRows, false>);
  return hipGetLastError();
}

// (a wide batch of one chunk per unit is written by its kernel)
bool attend_joins(const AttnLaunch& A, const AttendSpace& w) { return w.rw == 0 || w.splits > 1; }

hipError_t launch_attend_join_groups(const AttnLaunch& A, const AttendSpace& w, int group, void* out,
                                     float* lse, float* acc, float* acc_draft) {
  const bool wide = A.base.geo.D == 128;
  if (A.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? join_typed<__bf16, 128>(A, w, group, out, lse, acc, acc_draft)
                : join_typed<__bf16, 64>(A, w, group, out, lse, acc, acc_draft);
  return wide ? join_typed<float, 128>(A, w, group, out, lse, acc, acc_draft)
              : join_typed<float, 64>(A, w, group, out, lse, acc, acc_draft);
}

hipError_t launch_attend_join(const AttnLaunch& A, const AttendSpace& w, void* out, float* lse,
                              float* acc, float* acc_draft) {
  const bool bf16 = A.base.cfg->dtype == JACAP_DTYPE_BF16, wide = A.base.geo.D == 128;
  const int group = bf16 ? (wide ? kGroup<__bf16, 128> : kGroup<__bf16, 64>)
                         : (wide ? kGroup<float, 128> : kGroup<float, 64>);
  return launch_attend_join_groups(A, w, group, out, lse, acc, acc_draft);
}

}  // namespace jacap
