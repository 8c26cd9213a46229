// jacap_attn_weights (and the accumulation of jacap_attend with many rows): the
// attention weight every cached token receives from the rows of a window, of a
// whole prompt or of a tree,
//
//   acc_i <- decay acc_i + sum_r rw_r exp(z_ri - lse_r),  z_ri = scale q_r . k_i.
//
// A token's sum needs every row's lse first, and a row's lse every token, so
// the logits are formed twice: a pass over the rows' blocks for lse (rows in
// registers, keys streamed), and a pass over the tokens' blocks for the sums
// (keys in registers, rows streamed). Neither writes logits. V is not read.
#include <algorithm>

#include "attention.hpp"

namespace jacap {

// ---------------------------------------------------------------------------
// lse: a workgroup takes 16 MT rows of a unit and a chunk of its tokens; the
// waves take the chunk's 16-token steps in turn, each lane with a maximum and
// sum of its own (its row's tokens 4 q .. 4 q + 3), joined at the end.
// ---------------------------------------------------------------------------
template <typename T>
struct LseArgs {
  const T *q, *k;
  const float* acc;
  float* lse;        // [B][L][H_q][w], written here with one chunk
  float2* ml;        // else [U][R][chunks]
};

constexpr float kLazyLse = 8.0f;  // as the attention's: a lane's maximum is raised past this

template <typename T, int D, int MT>
__global__ __launch_bounds__(kThreads) void attn_lse_kernel(Geo g, Attn at, LseArgs<T> p, int chunk,
                                                            int chunks, int row_blocks) {
  using W = Row<T, D>;
  constexpr int NP = W::kPieces;
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int x = blockIdx.x;
  const int split = x % chunks;
  x /= chunks;
  // the last rows of a causal prompt see the most: first
  const int rb = row_blocks - 1 - x % row_blocks, u = x / row_blocks;
  const Unit un = live_unit(g, u);
  const int R = at.R, w = g.w;
  const int first = un.n - w;  // position of row 0 (causal)
  const int rr0 = rb * 16 * MT, rr1 = min(R, rr0 + 16 * MT);
  // tokens the block's rows see: none past the last position among them
  int pmin = 0, pmax = w - 1;
  if (rr0 / w == (rr1 - 1) / w) {
    pmin = rr0 % w;
    pmax = (rr1 - 1) % w;
  }
  const int limit = at.causal ? min(un.n, first + pmax + 1) : un.n;
  const int all = at.causal ? first + pmin + 1 : un.n;  // every row sees the tokens below
  const int t0 = split * chunk, t1 = min(limit, t0 + chunk);

  float mx[MT], thr[MT], ref[MT], l[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    mx[i] = thr[i] = -INFINITY;
    ref[i] = l[i] = 0.0f;
  }
  if (t0 < t1) {
    uint4 qf[MT][NP];
    int last[MT];  // position of the lane's row of each tile
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int r = rr0 + 16 * i + m;
      load_row<T, D>(g, unit_queries(g, un, p.q), min(r, R - 1), r < R, qg, qf[i]);
      last[i] = at.causal ? first + r % w : INT32_MAX;
    }
    const T* kb = p.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
    const int32_t ks = (int32_t)(g.kst * sizeof(T));
    const auto acc_range = buffer_range(p.acc + token_row(g, un) + t0, 4 * (t1 - t0));
    uint4 kf[NP];
    float a;
    // (zeros past the chunk's end)
    auto load = [&](int r0) {
      const auto kr = buffer_range(kb + r0 * g.kst, rows_bytes(min(16, t1 - r0), ks, W::kBytes));
#pragma unroll
      for (int x = 0; x < NP; ++x) kf[x] = buffer_load16(kr, m * ks + 64 * x + 16 * qg);
      a = buffer_load_f32(acc_range, 4 * (r0 - t0 + m));
    };
    load(t0 + 16 * wave);
    for (int r0 = t0 + 16 * wave; r0 < t1; r0 += 64) {
      // the next step's keys are requested before this one is multiplied
      uint4 kc[NP];
#pragma unroll
      for (int x = 0; x < NP; ++x) kc[x] = kf[x];
      const int rows = min(16, t1 - r0);
      const uint32_t vis = ((1u << rows) - 1) & ~(uint32_t)__ballot(a < 0.0f);
      load(r0 + 64);
      const bool masked = r0 + 16 > all || (vis & 0xFFFF) != 0xFFFF;
      const uint32_t seen = vis >> (4 * qg);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        f32x4 z = logits<T, D>(kc, qf[i]);
        if (masked) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            z[e] = (seen >> e & 1) && r0 + 4 * qg + e <= last[i] ? z[e] : -INFINITY;
        }
        const float top = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) * at.c;
        if (top > thr[i]) {
          const float nref = finite_ref(top);
          l[i] *= exp2_fast(mx[i] - nref);
          mx[i] = top;
          thr[i] = top + kLazyLse;
          ref[i] = nref;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) l[i] += exp2_fast(__builtin_fmaf(z[e], at.c, -ref[i]));
      }
    }
  }
  __shared__ float sm[4][16 * MT], sl[4][16 * MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    float top = fmaxf(mx[i], __shfl_xor(mx[i], 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    float s = l[i] * exp2_fast(mx[i] - finite_ref(top));
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (qg == 0) {
      sm[wave][16 * i + m] = top;
      sl[wave][16 * i + m] = s;
    }
  }
  __syncthreads();
  if (tid < 16 * MT && rr0 + tid < R) {
    float top = sm[0][tid];
    for (int y = 1; y < 4; ++y) top = fmaxf(top, sm[y][tid]);
    const float rf = finite_ref(top);
    float s = 0.0f;
    for (int y = 0; y < 4; ++y) s += sl[y][tid] * exp2_fast(sm[y][tid] - rf);
    const int r = rr0 + tid;
    if (chunks > 1) {
      p.ml[((int64_t)u * R + r) * chunks + split] = float2{top, s};
    } else {
      const int head = r / w;
      p.lse[(((int64_t)un.b * g.L + un.l) * g.Hq + un.h * g.G + head) * w + (r - head * w)] =
          s == 0.0f ? -INFINITY : (top + __log2f(s)) * kLn2;
    }
  }
}

// lse of rows of several chunks: 16 threads per row.
__global__ __launch_bounds__(kThreads) void attn_lse_join_kernel(Geo g, Attn at, const float2* ml,
                                                                 float* lse, int chunks) {
  const int64_t ur = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
  const bool live = ur < (int64_t)g.U * at.R;
  float top = -INFINITY, l = 0.0f;
  const float2* src = ml + (live ? ur : 0) * chunks;
  for (int s = threadIdx.x & 15; s < chunks; s += 16) top = fmaxf(top, src[s].x);
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  const float ref = finite_ref(top);
  for (int s = threadIdx.x & 15; s < chunks; s += 16) l += src[s].y * exp2_fast(src[s].x - ref);
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) l += __shfl_xor(l, x);
  if (live && (threadIdx.x & 15) == 0)
    // rows of a unit: heads h G .. h G + G - 1, so [U][R] is [B][L][H_q][w]
    lse[ur] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
}

template <typename T, int D, int MT>
static hipError_t lse_typed(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                            const float* acc, float* lse) {
  const Geo& g = A.base.geo;
  LseArgs<T> p{(const T*)q, (const T*)k, acc, lse, ws_ptr<float2>(A.base.wsp, w.ml)};
  const int64_t grid = (int64_t)g.U * w.row_blocks * w.chunks;
  attn_lse_kernel<T, D, MT><<<(unsigned)grid, kThreads, 0, A.base.stream>>>(g, A.at, p, w.chunk,
                                                                            w.chunks, w.row_blocks);
  if (w.chunks > 1) {
    const int64_t rows = (int64_t)g.U * A.at.R;
    attn_lse_join_kernel<<<(unsigned)((rows + 15) / 16), kThreads, 0, A.base.stream>>>(
        g, A.at, p.ml, lse, w.chunks);
  }
  return hipGetLastError();
}

hipError_t launch_attn_lse(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                           const float* acc, float* lse) {
  const bool wide = A.base.geo.D == 128;
  if (A.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? lse_typed<__bf16, 128, kLseTilesBf16>(A, w, q, k, acc, lse)
                : lse_typed<__bf16, 64, kLseTilesBf16>(A, w, q, k, acc, lse);
  return wide ? lse_typed<float, 128, kLseTilesFp32>(A, w, q, k, acc, lse)
              : lse_typed<float, 64, kLseTilesFp32>(A, w, q, k, acc, lse);
}

// ---------------------------------------------------------------------------
// Sums: a workgroup takes 64 NT tokens of a unit, 16 NT per wave with their keys in
// registers, and a part of the rows, kStageRows at a time through LDS (two
// buffers, the next rows requested a stage ahead). A lane adds the weights its
// query row gives its tokens; the 16 lanes of a tile's rows are added at the
// end. DRAFT: the tokens are the drafted ones, seen by the tree's mask.
//
// A staged row has 16 bytes of padding: the 16 lanes that read one piece of 16
// rows then touch all banks.
// ---------------------------------------------------------------------------
template <typename T>
struct SumArgs {
  const T *q, *k;
  const float* lse;   // [B][L][H_q][w]
  float* acc;         // updated with one row part (drafts: [U][S], written)
  float* part;        // else [row_splits][L][H][T]
  uint32_t* status;   // or null
};

constexpr int kStageRows = 32;

template <typename T, int D, int NT, bool DRAFT>
__global__ __launch_bounds__(kThreads) void attn_sum_kernel(Geo g, Attn at, SumArgs<T> p, int blocks,
                                                            int row_splits) {
  using W = Row<T, D>;
  constexpr int NP = W::kPieces;
  constexpr int PITCH = W::kBytes + 16;
  constexpr int SHARE = kStageRows * W::kBytes / 16 / kThreads;  // 16-byte pieces per thread and stage
  constexpr int LANES = W::kBytes / 16 / SHARE;                  // threads per staged row
  static_assert(LANES * kStageRows == kThreads, "a thread stages one row's pieces");
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // row parts of a token block together; a causal prompt's first tokens, which
  // the most rows see, first
  int x = blockIdx.x;
  const int part = x % row_splits;
  x /= row_splits;
  const int u = x % g.U, blk = x / g.U;
  const Unit un = live_unit(g, u);
  const int n = DRAFT ? g.w : un.n;
  const int btok = blk * 64 * NT;            // the workgroup's first token
  const int tok = btok + wave * 16 * NT;     // the wave's
  const int R = at.R, w = g.w;
  const bool causal = !DRAFT && at.causal;
  const int first = causal ? un.n - w : 0;
  const int stages = (R + kStageRows - 1) / kStageRows;
  const int per = (stages + row_splits - 1) / row_splits;
  const int stage1 = min(stages, (part + 1) * per);
  // The first stage from s on with a row that sees the workgroup's tokens: whole
  // stages of one head whose positions all lie before them are skipped.
  auto useful = [&](int s) {
    if (causal && s < stage1) {
      const int r0 = s * kStageRows, head = r0 / w, p0 = r0 - head * w;
      if (p0 + kStageRows <= w && first + p0 + kStageRows - 1 < btok)
        s = (head * w + min(w, btok - first)) / kStageRows;
    }
    return s;
  };

  if (btok < n) {
    const int64_t kst = DRAFT ? at.dkr : g.kst;
    const T* kb = DRAFT ? p.k + un.b * at.dks + un.l * at.dkl + un.h * at.dkh
                        : p.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
    const int32_t ks = (int32_t)(kst * sizeof(T));
    uint4 kf[NT][NP];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r0 = tok + 16 * t;
      const auto kr = buffer_range(kb + r0 * kst, rows_bytes(min(16, n - r0), ks, W::kBytes));
#pragma unroll
      for (int a = 0; a < NP; ++a) kf[t][a] = buffer_load16(kr, m * ks + 64 * a + 16 * qg);
    }
    const T* qu = unit_queries(g, un, p.q);
    const float* lseu = p.lse + ((int64_t)un.b * g.L + un.l) * g.Hq * w + (int64_t)un.h * R;
    const float* rwu = at.row_weight ? at.row_weight + (int64_t)un.b * w : nullptr;

    __shared__ __align__(16) char rows_lds[2][kStageRows * PITCH];
    struct Meta { float lse, weight; int last, pos; };  // last position seen, -1: adds nothing
    __shared__ Meta meta[2][kStageRows];
    const int srow = tid / LANES, spiece = tid % LANES * SHARE;
    uint4 held[SHARE];
    Meta mine;
    auto fetch = [&](int s) {
      const int r = min(s * kStageRows + srow, R - 1);
      const int head = r / w, pos = r - head * w;
      const char* src = reinterpret_cast<const char*>(qu + head * g.qsh + pos * g.qsp);
#pragma unroll
      for (int i = 0; i < SHARE; ++i) held[i] = *reinterpret_cast<const uint4*>(src + 16 * (spiece + i));
      mine.lse = lseu[r];
      mine.weight = rwu ? rwu[pos] : 1.0f;
      mine.pos = pos;
      mine.last = s * kStageRows + srow < R ? (causal ? first + pos : INT32_MAX) : -1;
    };
    auto store = [&](int buf) {
      const bool live = mine.last >= 0 && mine.weight != 0.0f && mine.lse != -INFINITY;
#pragma unroll
      for (int i = 0; i < SHARE; ++i)
        *reinterpret_cast<uint4*>(&rows_lds[buf][srow * PITCH + 16 * (spiece + i)]) =
            live ? held[i] : uint4{0, 0, 0, 0};
      if (spiece == 0)
        meta[buf][srow] = Meta{live ? mine.lse * kLog2e : 0.0f, live ? mine.weight : 0.0f,
                               live ? mine.last : -1, mine.pos};
    };

    f32x4 sum[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    int s = useful(part * per), buf = 0;
    if (s < stage1) {
      fetch(s);
      store(0);
    }
    __syncthreads();
    while (s < stage1) {
      const int next = useful(s + 1);
      if (next < stage1) fetch(next);
#pragma unroll
      for (int h = 0; h < kStageRows / 16; ++h) {
        const Meta me = meta[buf][16 * h + m];
        // nothing to add where no row of the tile sees a token of the wave
        if (__ballot(me.last >= tok) == 0) continue;
        const bool masked = DRAFT || __ballot(me.last < tok + 16 * NT) != 0;
        uint4 qf[NP];
#pragma unroll
        for (int a = 0; a < NP; ++a)
          qf[a] = *reinterpret_cast<const uint4*>(&rows_lds[buf][(16 * h + m) * PITCH + 64 * a + 16 * qg]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const f32x4 z = logits<T, D>(kf[t], qf);
          if (masked) {
            uint32_t bits = 0;
            if constexpr (DRAFT) {
              const int j0 = tok + 16 * t;
              if (me.last >= 0 && j0 < n) {
                if (at.tree)
                  bits = at.tree[((int64_t)un.b * w + me.pos) * at.tree_words + (j0 >> 5)] >> (j0 & 31);
                else
                  bits = me.pos < j0 ? 0u : me.pos - j0 >= 31 ? ~0u : (2u << (me.pos - j0)) - 1u;
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool see = DRAFT ? (bits >> (4 * qg + e) & 1) : tok + 16 * t + 4 * qg + e <= me.last;
              const float y = exp2_fast(__builtin_fmaf(z[e], at.c, -me.lse));
              sum[t][e] = see ? __builtin_fmaf(y, me.weight, sum[t][e]) : sum[t][e];
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sum[t][e] = __builtin_fmaf(exp2_fast(__builtin_fmaf(z[e], at.c, -me.lse)), me.weight, sum[t][e]);
          }
        }
      }
      if (next < stage1) store(buf ^ 1);
      __syncthreads();
      buf ^= 1;
      s = next;
    }
    // over the tile's 16 rows: every lane of a 16-lane group ends with the sums
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float mine = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float s = sum[t][e];
        s += dpp_f32<kDppQuadXor1>(s);
        s += dpp_f32<kDppQuadXor2>(s);
        s += dpp_f32<kDppHalfMirror>(s);
        s += dpp_f32<kDppMirror>(s);
        mine = m == e ? s : mine;
      }
      const int j = tok + 16 * t + 4 * qg + m;
      if (m < 4 && j < n) {
        if constexpr (DRAFT) {
          p.acc[(int64_t)u * w + j] = mine;
        } else {
          const int64_t i = token_row(g, un) + j;
          if (row_splits > 1) {
            p.part[(int64_t)part * g.L * g.H * g.T + i] = mine;
          } else {
            const float old = p.acc[i];
            if (!(old < 0.0f)) p.acc[i] = at.decay > 0.0f ? __builtin_fmaf(at.decay, old, mine) : mine;
          }
        }
      }
    }
  }
  if (blockIdx.x == 0 && p.status) write_status(g, p.status);
}

// The row parts' sums, in order.
__global__ __launch_bounds__(kThreads) void attn_sum_join_kernel(Geo g, Attn at, const float* part,
                                                                 float* acc, int row_splits) {
  const Unit un = live_unit(g, blockIdx.y);
  const int64_t tr = token_row(g, un), pitch = (int64_t)g.L * g.H * g.T;
  const int t = blockIdx.x * kThreads + threadIdx.x;
  if (t >= un.n) return;
  const float old = acc[tr + t];
  if (old < 0.0f) return;
  float sum = 0.0f;
  for (int s = 0; s < row_splits; ++s) sum += part[s * pitch + tr + t];
  acc[tr + t] = at.decay > 0.0f ? __builtin_fmaf(at.decay, old, sum) : sum;
}

template <typename T, int D, int NT>
static hipError_t sum_typed(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                            const float* lse, float* acc, uint32_t* status) {
  const Geo& g = A.base.geo;
  SumArgs<T> p{(const T*)q, (const T*)k, lse, acc, ws_ptr<float>(A.base.wsp, w.part), status};
  const int64_t grid = (int64_t)g.U * std::max(1, w.blocks) * w.row_splits;
  attn_sum_kernel<T, D, NT, false><<<(unsigned)grid, kThreads, 0, A.base.stream>>>(
      g, A.at, p, w.blocks, w.row_splits);
  if (w.row_splits > 1 && g.maxn > 0)
    attn_sum_join_kernel<<<dim3((g.maxn + kThreads - 1) / kThreads, g.U), kThreads, 0,
                           A.base.stream>>>(g, A.at, p.part, acc, w.row_splits);
  return hipGetLastError();
}

hipError_t launch_attn_sum(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                           const float* lse, float* acc, uint32_t* status) {
  const bool wide = A.base.geo.D == 128;
  if (A.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? sum_typed<__bf16, 128, kSumTilesBf16>(A, w, q, k, lse, acc, status)
                : sum_typed<__bf16, 64, kSumTilesBf16>(A, w, q, k, lse, acc, status);
  return wide ? sum_typed<float, 128, kSumTilesFp32>(A, w, q, k, lse, acc, status)
              : sum_typed<float, 64, kSumTilesFp32>(A, w, q, k, lse, acc, status);
}

template <typename T, int D>
static hipError_t draft_typed(const AttnLaunch& A, const void* q, const void* kd, const float* lse,
                              float* acc_draft) {
  const Geo& g = A.base.geo;
  SumArgs<T> p{(const T*)q, (const T*)kd, lse, acc_draft, nullptr, nullptr};
  const int blocks = (g.w + 63) / 64;
  attn_sum_kernel<T, D, 1, true><<<(unsigned)((int64_t)g.U * blocks), kThreads, 0, A.base.stream>>>(
      g, A.at, p, blocks, 1);
  return hipGetLastError();
}

hipError_t launch_draft_sum(const AttnLaunch& A, const void* q, const void* kd, const float* lse,
                            float* acc_draft) {
  const bool wide = A.base.geo.D == 128;
  if (A.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? draft_typed<__bf16, 128>(A, q, kd, lse, acc_draft)
                : draft_typed<__bf16, 64>(A, q, kd, lse, acc_draft);
  return wide ? draft_typed<float, 128>(A, q, kd, lse, acc_draft)
              : draft_typed<float, 64>(A, q, kd, lse, acc_draft);
}

}  // namespace jacap
