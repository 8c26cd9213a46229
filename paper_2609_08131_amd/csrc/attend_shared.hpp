// What the attention kernels over a cache share, whatever its values are held in
// (k_attend.hip: the cache's own type; k_attend_quant.hip: 8 bits): arguments, the
// cut of the work into spans, and the kernel of many rows.
#pragma once

#include <type_traits>

#include <algorithm>

#include "attention.hpp"
#include "quant.hpp"

namespace jacap {

template <typename T>
struct AttendArgs {
  const T *q, *k, *v, *kd, *vd;
  T* out;
  float* lse;        // of units of one chunk, or null
  const float* acc;  // empty slots, or null
  float2* ml;
  float* part;
  float *z, *zd;     // kept logits, or null
  uint32_t* status;
  int32_t* before;   // groups before each sequence
};

// What the accumulators do in a call, apart in the code: a load or store that
// only some calls make would have the others' waits count it too.
enum Mode { kPlain, kHides, kKeeps };  // not read; hide empty slots; and the logits are kept

// Kept logits lie by 16-token tiles, [R][16] each. A sequence's tiles start behind
// t0 / 16 + b others of its (layer, KV head) row, which leaves room for every
// sequence's last, partial tile.
__host__ __device__ __forceinline__ int64_t keep_tiles(const Geo& g) { return g.T / 16 + g.B + 1; }
__device__ __forceinline__ int64_t keep_at(const Geo& g, const Unit& un, int R, int tile) {
  return ((((int64_t)un.l * g.H + un.h) * keep_tiles(g)) + un.t0 / 16 + un.b + tile) * R * 16;
}

// Which of the drafted tokens j0 .. j0 + 31 the row of position `pos` sees, as bits.
__device__ __forceinline__ uint32_t draft_mask(const Attn& at, int b, int pos, int S, int j0) {
  if (at.tree) return at.tree[((int64_t)b * S + pos) * at.tree_words + (j0 >> 5)] >> (j0 & 31);
  const int last = pos - j0;  // sees 0 .. pos
  return last < 0 ? 0u : last >= 31 ? ~0u : (2u << last) - 1u;
}

// How attend_kernel's work is cut: every unit (and row block of it: L H row_blocks
// of them per sequence, side by side) is a run of groups of 4 steps, one step per
// wave, at least one group (the drafted tokens go with the last), and kUnitGroups
// empty ones after them, the cost of beginning and ending a unit. The runs of all
// units in order are cut into spans of `quantum` groups, one per workgroup, whatever
// the sequences' lengths are when the kernel runs. A workgroup's span begins in one
// unit and ends in one; what it holds of a unit that it shares with others is
// written apart, as piece 2 w (of the unit it begins in) or 2 w + 1, and joined later.
// Against chunks of equal size (16 sequences of 4096 to 32768 tokens, 600 chunks of
// 4096 on 512 places: 206 us) every place has the same work: 176 us.
__device__ __forceinline__ int real_groups(int n, int group) { return max(1, (n + group - 1) / group); }
__device__ __forceinline__ int span_quantum(int groups, int blocks, int group) {
  return max(kSpanMin / group, (groups + blocks - 1) / blocks);
}
// Where piece j of a unit whose groups begin at `start` lies.
__device__ __forceinline__ int64_t piece_of(int start, int quantum, int j) {
  const int w = start / quantum;
  return 2 * (int64_t)(w + j) + (j == 0 && start != w * quantum);
}
// Where the first of the n pieces of row r of a unit cut into chunks lies. A sequence's pieces,
// [R][n], start behind those of t0 / chunk + b chunks of its (layer, KV head), which is room for
// the sequences before it, whatever their lengths.
__device__ __forceinline__ int64_t chunk_place(const Geo& g, const Unit& un, int places, int chunk, int R,
                                               int r, int n) {
  return (((int64_t)un.l * g.H + un.h) * places + un.t0 / chunk + un.b) * R + (int64_t)r * n;
}
// A sequence's first cache row and current length.
__device__ __forceinline__ int2 sequence_rows(const Geo& g, const Attn& at, int b) {
  const int32_t a = g.seq_off[b], e = g.seq_off[b + 1];
  int n = offsets_ok(g, a, e) ? e - a : 0;
  if (g.live) n = live_ok(g, b, n) ? g.live[b] : 0;
  if ((a | e) & at.row_mask) n = 0;  // as whole_blocks
  return int2{a, n};
}
// Inclusive scan over the wave's lanes.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // last lane of rows 0, 2 to 1, 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2, 3
  return v;
}

template <typename T>
struct AttendParams {
  Geo g;
  Attn at;
  AttendArgs<T> p;
  int row_blocks;
};

// ---------------------------------------------------------------------------
// Many rows (a tree of drafted tokens under several query heads), bf16. Row blocks
// of their own would each read K and V again, through an L2 that does not keep
// up with the MFMA; here eight waves share a stage of K and V in LDS: RW waves take
// 32 rows each, and the 8 / RW groups of them take the stage's 32-token steps in
// turn. A unit's rows, up to 256, then read the cache once.
//
// K is staged in operand order (16 bytes per lane; load_row's pieces, of an 8-bit cache
// quant_piece's), V token-major with a pitch
// that is an odd multiple of 32 bytes, read with the transposing LDS read: lane
// (m, q) receives channel m of a 16-channel block for tokens 4 q .. 4 q + 3 of a tile,
// the order in which the weights stand in the lanes. Two buffers, the next
// stage's loads in flight during the products, one barrier a stage. The values of an 8-bit
// cache become bf16 on their way into LDS, once for all waves.
// ---------------------------------------------------------------------------
typedef short s16x4 __attribute__((ext_vector_type(4)));
constexpr int kWideThreads = 512;

template <int D, int RW, bool QUANT = false>
struct Wide {
  static constexpr int kGroups = 8 / RW;                       // token groups of waves
  static constexpr int kTokens = RW == 2 || (QUANT && D == 64) ? 128 : 64;  // per stage
  static constexpr int kSteps = kTokens / 32 / kGroups;        // 32-token steps per wave and stage
  static constexpr int kPitch = D == 128 ? 288 : 160;          // bytes per staged V row
  static constexpr int kBuffer = kTokens * (2 * D + kPitch);   // K then V
  static constexpr int kShare = kTokens * D * 2 / 16 / kWideThreads;  // 16-byte pieces per thread
  static constexpr int kJoin = (kGroups - 1) * RW * 16 * (D + 4) * 4;
  static constexpr int kLds = 2 * kBuffer > kJoin ? 2 * kBuffer : kJoin;
};

template <int D, int RW, bool HIDES, bool QUANT>
__global__ __launch_bounds__(kWideThreads, 2) void attend_wide_kernel(Geo g, Attn at,
                                                                      AttendArgs<__bf16> p, QuantArgs qa,
                                                                      int chunk,
                                                                      int splits, int row_blocks,
                                                                      int places) {
  using T = __bf16;
  using W = Row<T, D>;
  using S_ = Wide<D, RW, QUANT>;
  constexpr int NP = W::kPieces, MT = 2, NB = D / 16, SH = S_::kShare;
  extern __shared__ __align__(16) char lds[];
  __shared__ float sm[8][32], sl[8][32];
  __shared__ uint32_t bad[S_::kTokens / 32];  // drafted tokens with a non-finite value
  __shared__ float signs[2][S_::kTokens];     // the staged tokens' accumulators
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, grp = wave / RW;
  int pair = blockIdx.x, rb = 0;  // as attend_kernel
  if (row_blocks > 1) {
    const int x = pair % (8 * row_blocks);
    rb = x >> 3;
    pair = pair / (8 * row_blocks) * 8 + (x & 7);
  }
  if (pair >= g.U * splits) return;
  const int u = pair % g.U, split = pair / g.U;
  const Unit un = attention_unit(g, at, u);
  const int S = g.w, R = at.R;
  const int nsp = max(1, (un.n + chunk - 1) / chunk);
  if (split >= nsp) return;
  const int t0 = split * chunk, t1 = min(un.n, t0 + chunk);
  const bool drafts = split == nsp - 1;

  uint4 qf[MT][NP];
  int row[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    row[i] = (rb * RW + rw) * 32 + 16 * i + m;
    if constexpr (QUANT)
      load_quant_row<D>(g, unit_queries(g, un, p.q), min(row[i], R - 1), row[i] < R, qg, qf[i]);
    else
      load_row<T, D>(g, unit_queries(g, un, p.q), min(row[i], R - 1), row[i] < R, qg, qf[i]);
  }
  f32x4 o[MT][NB];
  float ref[MT], l[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    ref[i] = kNoMax;
    l[i] = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b) o[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Staging. K piece i of a thread: fragment wave * SH + i (token tile f / NP, piece
  // f % NP), this lane's 16 bytes. V piece i: row, 16 bytes of it in turn.
  constexpr int VL = D / 8;            // lanes per V row
  constexpr int VR = 64 / VL;          // rows per wave load
  const int vrow = lane / VL, vpiece = lane % VL;
  uint4 kh[SH], vh[SH];
  float sign[SH];
  auto fetch = [&](const T* kbase, const T* vbase, int64_t kst, int64_t vst, const float* acc, int r0,
                   int end) {
    const int rows = min(S_::kTokens, end - r0);
    const int32_t ks = (int32_t)(kst * 2), vs = (int32_t)(vst * 2);
    const int kr0 = wave * SH / NP * 16, vr0 = wave * SH * VR;  // the wave's first rows
    const auto kr = buffer_range(kbase + (r0 + kr0) * kst, rows_bytes(min(32, rows - kr0), ks, W::kBytes));
    const auto vr = buffer_range(vbase + (r0 + vr0) * vst, rows_bytes(min(32, rows - vr0), vs, W::kBytes));
#pragma unroll
    for (int i = 0; i < SH; ++i) {
      const int f = wave * SH + i;
      kh[i] = buffer_load16(kr, (f / NP * 16 - kr0 + m) * ks + 64 * (QUANT ? 0 : f % NP) + 16 * qg * (QUANT ? 2 : 1) +
                                    (QUANT ? quant_piece(f % NP) : 0));
    }
#pragma unroll
    for (int i = 0; i < SH; ++i) vh[i] = buffer_load16(vr, (i * VR + vrow) * vs + 16 * vpiece);
    if (acc) {
      const auto ar = buffer_range(acc + r0 + vr0, 4 * max(0, min(32, rows - vr0)));
#pragma unroll
      for (int i = 0; i < SH; ++i) sign[i] = buffer_load_f32(ar, 4 * (i * VR + vrow));
    } else {
#pragma unroll
      for (int i = 0; i < SH; ++i) sign[i] = 0.0f;
    }
  };
  // The same of the 8-bit cache: K's 16 bytes are two pieces, V's 8 bytes one. (A wave's
  // rows are of one block wherever that is 32 tokens or more; of 16, tile by tile.)
  uint4 k8[QUANT ? SH / 2 : 1];
  uint2 v8[QUANT ? SH : 1];
  float ksc[QUANT ? SH / 2 : 1], vsc[QUANT ? SH : 1];
  auto fetch_quant = [&](const float* acc, int r0, int end) {
    if constexpr (QUANT) {
      const int rows = min(S_::kTokens, end - r0);
      const int32_t ks = (int32_t)g.kst, vs = (int32_t)g.vst;
      const int kr0 = wave * SH / NP * 16, vr0 = wave * SH * VR;
      const uint8_t* kbase = qa.k + un.l * g.ksl + un.h * g.ksh + (un.t0 + r0 + kr0) * g.kst;
      const uint8_t* vbase = qa.v + un.l * g.vsl + un.h * g.vsh + (un.t0 + r0 + vr0) * g.vst;
      const auto kr = buffer_range(kbase, rows_bytes(min(32, rows - kr0), ks, D));
      const auto vr = buffer_range(vbase, rows_bytes(min(32, rows - vr0), vs, D));
      const auto sr = scale_range(qa, g, un, un.n);
#pragma unroll
      for (int i = 0; i < SH / 2; ++i) {
        const int f = wave * SH + 2 * i;
        k8[i] = buffer_load16(kr, (f / NP * 16 - kr0 + m) * ks + 64 * (f % NP / 2) + 16 * qg);
        ksc[i] = buffer_load_f32(sr, (r0 + f / NP * 16) >> qa.shift << 3);
      }
#pragma unroll
      for (int i = 0; i < SH; ++i) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(vr, (i * VR + vrow) * vs + 8 * vpiece, 0, 0);
        v8[i] = uint2{x[0], x[1]};
        vsc[i] = buffer_load_f32(sr, ((r0 + vr0 + i * VR) >> qa.shift << 3) + 4);
      }
      if (HIDES) {
        const auto ar = buffer_range(acc + r0 + vr0, 4 * max(0, min(32, rows - vr0)));
#pragma unroll
        for (int i = 0; i < SH; ++i) sign[i] = buffer_load_f32(ar, 4 * (i * VR + vrow));
      }
    }
  };
  auto widen = [&] {
    if constexpr (QUANT) {
#pragma unroll
      for (int i = 0; i < SH / 2; ++i) {
        kh[2 * i] = widen8(k8[i].x, k8[i].y, ksc[i]);
        kh[2 * i + 1] = widen8(k8[i].z, k8[i].w, ksc[i]);
      }
#pragma unroll
      for (int i = 0; i < SH; ++i) vh[i] = widen8(v8[i].x, v8[i].y, vsc[i]);
    }
  };
  auto store = [&](int buf) {
    char* kd = lds + buf * S_::kBuffer;
    char* vd = kd + S_::kTokens * 2 * D;
#pragma unroll
    for (int i = 0; i < SH; ++i)
      *reinterpret_cast<uint4*>(kd + (wave * SH + i) * 1024 + 16 * lane) = kh[i];
#pragma unroll
    for (int i = 0; i < SH; ++i)
      *reinterpret_cast<uint4*>(vd + ((wave * SH + i) * VR + vrow) * S_::kPitch + 16 * vpiece) =
          HIDES && sign[i] < 0.0f ? uint4{0, 0, 0, 0} : vh[i];
    if constexpr (HIDES) {
      if (vpiece == 0)
#pragma unroll
        for (int i = 0; i < SH; ++i) signs[buf][(wave * SH + i) * VR + vrow] = sign[i];
    }
  };

  // One 32-token step from a buffer, at token `j` of the stage.
  auto step = [&](auto draft, int buf, int j, uint32_t vis, const uint32_t (&mask)[MT], int r0) {
    constexpr bool DRAFT = decltype(draft)::value;
    const char* kd = lds + buf * S_::kBuffer + j / 16 * NP * 1024 + 16 * lane;
    const char* vd = lds + buf * S_::kBuffer + S_::kTokens * 2 * D +
                     (j + 4 * qg + (m >> 2)) * S_::kPitch + 8 * (m & 3);
    f32x4 z[MT][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint4 kf[NP];
#pragma unroll
      for (int a = 0; a < NP; ++a) kf[a] = *reinterpret_cast<const uint4*>(kd + (t * NP + a) * 1024);
#pragma unroll
      for (int i = 0; i < MT; ++i) z[i][t] = logits<T, D>(kf, qf[i]);
    }
    if (DRAFT || vis != ~0u) {
      const uint32_t mine = vis >> (4 * qg);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            bool see = mine >> (16 * t + e) & 1;
            if constexpr (DRAFT) see = see && (mask[i] >> (16 * t + 4 * qg + e) & 1);
            z[i][t][e] = see ? z[i][t][e] : -INFINITY;
          }
    }
    // The exponents against the maxima so far, which the largest of them may raise. (Taken of
    // the logits themselves, the maximum would cost a quieting instruction for each.)
    float over = kNoMax;
    f32x4 y[MT][2];
    auto exponents = [&](int i) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[i][t][e] = __builtin_fmaf(z[i][t][e], at.c, -ref[i]);
    };
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      exponents(i);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) over = fmaxf(over, y[i][t][e]);
    }
    if (__ballot(over > kLazyMax) != 0) {
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        float now = fmaxf(max4(z[i][0]), max4(z[i][1])) * at.c;
        now = fmaxf(now, __shfl_xor(now, 16));
        now = fmaxf(now, __shfl_xor(now, 32));
        now = fminf(fmaxf(now, ref[i]), kTop);
        const float f = exp2_fast(ref[i] - now);
        ref[i] = now;
        l[i] *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) o[i][b] *= f;
        exponents(i);
      }
    }
    bf8 pb[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[i][t][e] = exp2_fast(y[i][t][e]);
          pb[i][4 * t + e] = (__bf16)z[i][t][e];
        }
#pragma unroll
    for (int i = 0; i < MT; ++i)
      l[i] += ((z[i][0][0] + z[i][0][1]) + (z[i][0][2] + z[i][0][3])) +
              ((z[i][1][0] + z[i][1][1]) + (z[i][1][2] + z[i][1][3]));
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      uint64_t v[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        v[t] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (__attribute__((address_space(3))) s16x4*)(vd + 16 * t * S_::kPitch + 32 * b)));
      const uint4 a = {(uint32_t)v[0], (uint32_t)(v[0] >> 32), (uint32_t)v[1], (uint32_t)(v[1] >> 32)};
#pragma unroll
      for (int i = 0; i < MT; ++i)
        o[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), pb[i], o[i][b], 0, 0, 0);
    }
    if constexpr (DRAFT) {
      // drafted tokens whose V was staged as 0: added row by row to those that see them
      uint32_t rest = __builtin_amdgcn_readfirstlane(bad[j / 32]);
      while (rest) {
        const int y = __builtin_ctz(rest);  // token 16 t + 4 x + e
        rest &= rest - 1;
        const int t = y >> 4, from = y >> 2 & 3, e = y & 3;
        const T* src = p.vd + un.b * at.dvs + un.l * at.dvl + un.h * at.dvh + (r0 + y) * at.dvr + 4 * qg;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          float w = 0.0f;
#pragma unroll
          for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
            for (int e2 = 0; e2 < 4; ++e2) w = t2 == t && e2 == e ? z[i][t2][e2] : w;
          w = __shfl(w, 16 * from + m);
          if (!(mask[i] >> y & 1)) continue;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e2 = 0; e2 < 4; ++e2) o[i][b][e2] += w * (float)src[16 * b + e2];
        }
      }
    }
  };

  const uint32_t none[MT] = {};
  const T* kb = p.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
  const T* vb = p.v + un.l * g.vsl + un.h * g.vsh + un.t0 * g.vst;
  const float* accb = HIDES ? p.acc + token_row(g, un) : nullptr;
  int buf = 0;
  if (t0 < t1) {
    if constexpr (QUANT) fetch_quant(accb, t0, t1);
    else fetch(kb, vb, g.kst, g.vst, accb, t0, t1);
    widen();
    store(0);
  }
  __syncthreads();
  for (int r0 = t0; r0 < t1; r0 += S_::kTokens) {
    const bool more = r0 + S_::kTokens < t1;
    if (more) {
      if constexpr (QUANT) fetch_quant(accb, r0 + S_::kTokens, t1);
      else fetch(kb, vb, g.kst, g.vst, accb, r0 + S_::kTokens, t1);
    }
#pragma unroll
    for (int x = 0; x < S_::kSteps; ++x) {
      const int j = (x * S_::kGroups + grp) * 32, rows = t1 - r0 - j;
      if (rows <= 0) continue;
      uint32_t vis = rows >= 32 ? ~0u : (1u << rows) - 1;
      if constexpr (HIDES) vis &= ~(uint32_t)__ballot(signs[buf][j + (lane & 31)] < 0.0f);
      step(std::false_type{}, buf, j, vis, none, r0 + j);
    }
    if (more) {
      widen();
      store(buf ^ 1);
    }
    __syncthreads();
    buf ^= 1;
  }
  if (drafts) {
    const T* kdb = p.kd + un.b * at.dks + un.l * at.dkl + un.h * at.dkh;
    const T* vdb = p.vd + un.b * at.dvs + un.l * at.dvl + un.h * at.dvh;
    for (int r0 = 0; r0 < S; r0 += S_::kTokens) {
      fetch(kdb, vdb, at.dkr, at.dvr, nullptr, r0, S);
      if (tid < S_::kTokens / 32) bad[tid] = 0u;
      __syncthreads();
      // a drafted token that some rows see and others do not is added apart if it
      // holds a value that is not finite: its weight 0 would not hide it
#pragma unroll
      for (int i = 0; i < SH; ++i) {
        const uint32_t y[4] = {vh[i].x, vh[i].y, vh[i].z, vh[i].w};
        bool odd = false;
#pragma unroll
        for (int z = 0; z < 4; ++z)
          odd |= (y[z] & 0x7F800000u) == 0x7F800000u || (y[z] & 0x7F80u) == 0x7F80u;
        const int r = (wave * SH + i) * VR + vrow;
        if (odd) atomicOr(&bad[r >> 5], 1u << (r & 31));
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < SH; ++i) {
        const int r = (wave * SH + i) * VR + vrow;
        if (bad[r >> 5] >> (r & 31) & 1) vh[i] = uint4{0, 0, 0, 0};
      }
      store(0);
      __syncthreads();
#pragma unroll
      for (int x = 0; x < S_::kSteps; ++x) {
        const int j = (x * S_::kGroups + grp) * 32, rows = S - r0 - j;
        if (rows <= 0) continue;
        uint32_t mask[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) mask[i] = row[i] < R ? draft_mask(at, un.b, row[i] % S, S, r0 + j) : 0u;
        step(std::true_type{}, 0, j, rows >= 32 ? ~0u : (1u << rows) - 1, mask, r0 + j);
      }
      __syncthreads();
    }
  }

  // Join the groups of waves that took the same rows.
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
  float* red = reinterpret_cast<float*>(lds);
  constexpr int PD = D + 4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    float top = kNoMax, sum = 0.0f;
#pragma unroll
    for (int x = 0; x < S_::kGroups; ++x) top = fmaxf(top, sm[x * RW + rw][16 * i + m]);
#pragma unroll
    for (int x = 0; x < S_::kGroups; ++x)
      sum += sl[x * RW + rw][16 * i + m] * exp2_fast(sm[x * RW + rw][16 * i + m] - top);
    const float f = exp2_fast(ref[i] - top);
    if constexpr (S_::kGroups > 1) {
      if (i > 0) __syncthreads();
      if (grp > 0) {
        float* dst = red + (((grp - 1) * RW + rw) * 16 + m) * PD + 4 * qg;
#pragma unroll
        for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(dst + 16 * b) = o[i][b] * f;
      }
      __syncthreads();
    }
    if (grp > 0 || row[i] >= R) continue;
    const int64_t place = chunk_place(g, un, places, chunk, R, row[i], nsp) + split;
    const int head = row[i] / S, pos = row[i] - head * S;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* dst = p.out + un.b * at.os + un.l * at.ol + (int64_t)(un.h * g.G + head) * at.oh + pos * at.op;
    float* part = p.part + place * D;  // (only where there are pieces)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32x4 val = o[i][b] * f;
#pragma unroll
      for (int x = 1; x < S_::kGroups; ++x)
        val += *reinterpret_cast<const f32x4*>(red + (((x - 1) * RW + rw) * 16 + m) * PD + 16 * b + 4 * qg);
      if (nsp == 1) {
        typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
        const bf4 y = {(__bf16)(val[0] * inv), (__bf16)(val[1] * inv), (__bf16)(val[2] * inv),
                       (__bf16)(val[3] * inv)};
        *reinterpret_cast<bf4*>(dst + 16 * b + 4 * qg) = y;
      } else {
        *reinterpret_cast<f32x4*>(part + 16 * b + 4 * qg) = val;
      }
    }
    if (qg == 0) {
      if (nsp > 1) p.ml[place] = float2{top, sum};
      if (nsp == 1 && p.lse)
        p.lse[(((int64_t)un.b * g.L + un.l) * g.Hq + un.h * g.G + head) * S + pos] =
            sum == 0.0f ? -INFINITY : (top + __log2f(sum)) * kLn2;
    }
  }
  if (blockIdx.x == 0) write_status(g, at, p.status);
}

}  // namespace jacap
