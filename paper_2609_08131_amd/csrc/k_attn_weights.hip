// jacap_attn_weights (and the accumulation of jacap_attend with many rows): the
// attention weight every cached token receives from the rows of a window, of a
// whole prompt or of a tree,
//
//   acc_i <- decay acc_i + sum_r rw_r exp(z_ri - lse_r),  z_ri = scale q_r . k_i.
//
// A token's sum needs every row's lse first, and a row's lse every token, so
// the logits are formed twice: a pass over the rows' blocks for lse (rows in
// registers, keys streamed), and a pass over the tokens' blocks for the sums
// (keys in registers, rows from LDS). Neither writes logits. V is not read.
#include <algorithm>

#include "attention.hpp"

namespace jacap {

// Asks for the vector operations of one 16-row tile's logits, then in turn for one MFMA
// and the operations of one logit (an FMA, an exponential, an addition) over the rest of the
// block it stands in: the MFMAs run while the others are issued, and a chain's
// next MFMA finds its predecessor done. fp32 products take longer than the exponentials
// anyway.
template <bool BF16, int MFMAS>
__device__ __forceinline__ void interleave() {
  if constexpr (BF16) {
    __builtin_amdgcn_sched_group_barrier(0x002, 12, 0);
#pragma unroll
    for (int i = 0; i < MFMAS; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
    }
  }
}

// The sum over a tile's 16 query rows of each of its tokens: lane (m, q) receives
// that of token 4 q + m for m < 4.
__device__ __forceinline__ float tile_sum(const f32x4& x, int m) {
  float mine = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float s = x[e];
    s += dpp_f32<kDppQuadXor1>(s);
    s += dpp_f32<kDppQuadXor2>(s);
    s += dpp_f32<kDppHalfMirror>(s);
    s += dpp_f32<kDppMirror>(s);
    mine = m == e ? s : mine;
  }
  return mine;
}

// An accumulator's new value.
__device__ __forceinline__ float decayed(const Attn& at, float old, float sum) {
  return at.decay > 0.0f ? __builtin_fmaf(at.decay, old, sum) : sum;
}

// ---------------------------------------------------------------------------
// The rows' lse: rows in registers, keys streamed. A workgroup takes 16 MT rows of a
// unit and a chunk of its tokens; the waves take the chunk's 16-token steps in turn.
// Each lane keeps a maximum and sum of its own (its row's tokens 4 q .. 4 q + 3), joined
// at the end.
//
// The loop holds a step's logits, and forms the next step's tile by tile in their
// place as they are added: no branch between, so that a tile's products run beside
// the exponentials of the next. Keys are requested a step ahead of their products.
// ---------------------------------------------------------------------------
constexpr int kFlush = 8;

template <typename T>
struct RowArgs {
  const T *q, *k;
  const float* acc;  // empty slots
  float* lse;        // [B][L][H_q][w], written here with one chunk
  float2* ml;        // ... or [U][R][chunks]
};

template <typename T, int D, int MT>
__global__ __launch_bounds__(kThreads, 2) void attn_rows_kernel(Geo g, Attn at, RowArgs<T> p,
                                                                int chunk, int chunks,
                                                                int row_blocks) {
  using W = Row<T, D>;
  constexpr int NP = W::kPieces;
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // The last rows of a causal prompt see the most: they go first, in every unit.
  // Units innermost: the workgroups of one unit then share few XCDs and their L2.
  const int u = blockIdx.x % g.U, x = blockIdx.x / g.U;
  const int split = x % chunks, rb = row_blocks - 1 - x / chunks;
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

  // Minus the lane's maximum, and its sum, which is
  // taken by kFlush steps first: added one by one to that of a token which dominates the
  // row, most of the others' small weights would be lost to rounding, always to the
  // same side (a 128K window's accumulators off by 2e-6 relative, 2e-7 so).
  float nref[MT], l[MT], li[MT];
  int steps = 0;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    nref[i] = -kNoMax;
    l[i] = li[i] = 0.0f;
  }
  if (t0 < t1) {
    uint4 qf[MT][NP];
    int last[MT];  // position of the lane's row of each tile
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int r = rr0 + 16 * i + m, rc = min(r, R - 1);
      load_row<T, D>(g, unit_queries(g, un, p.q), rc, r < R, qg, qf[i]);
      last[i] = at.causal ? first + rc % w : INT32_MAX;
    }
    const T* kb = p.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
    const int32_t ks = (int32_t)(g.kst * sizeof(T));
    const int64_t tr = token_row(g, un) + t0;
    const auto acc_range = buffer_range(p.acc + tr, 4 * (t1 - t0));
    struct Keys {
      uint4 k[NP];
      float a;  // the accumulator of token m
    };
    // (zeros past the chunk's end)
    auto load = [&](Keys& y, int r0) {
      const auto kr = buffer_range(kb + r0 * g.kst, rows_bytes(min(16, t1 - r0), ks, W::kBytes));
#pragma unroll
      for (int a = 0; a < NP; ++a) y.k[a] = buffer_load16(kr, m * ks + 64 * a + 16 * qg);
      y.a = buffer_load_f32(acc_range, 4 * (r0 - t0 + m));
    };
    int r0 = t0 + 16 * wave;
    Keys ka, kb2;
    load(ka, r0);
    f32x4 z[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) z[i] = logits<T, D>(ka.k, qf[i]);
    float sign = ka.a;  // of the step that z is of
    load(kb2, r0 + 64);
    // One step: z's logits are added, `next` gives the following step's, and `far`
    // takes the keys of the one after that.
    auto step = [&](const Keys& next, Keys& far) {
      const uint32_t vis = ((1u << min(16, t1 - r0)) - 1) & ~(uint32_t)__ballot(sign < 0.0f);
      sign = next.a;
      load(far, r0 + 128);
      if (vis != 0xFFFFu || r0 + 16 > all) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = 4 * qg + e;
            z[i][e] = (vis >> j & 1) && r0 + j <= last[i] ? z[i][e] : -INFINITY;
          }
      }
      float top[MT], over = kNoMax;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        top[i] = max4(z[i]);
        over = fmaxf(over, __builtin_fmaf(top[i], at.c, nref[i]));
      }
      if (__ballot(over > kLazyMax) != 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const float now = fminf(fmaxf(-nref[i], top[i] * at.c), kTop);
          const float f = exp2_fast(-nref[i] - now);
          l[i] *= f;
          li[i] *= f;
          nref[i] = -now;
        }
      }
      if ((++steps & (kFlush - 1)) == 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          l[i] += li[i];
          li[i] = 0.0f;
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = exp2_fast(__builtin_fmaf(z[i][e], at.c, nref[i]));
        li[i] += (y[0] + y[1]) + (y[2] + y[3]);
        z[i] = logits<T, D>(next.k, qf[i]);
      }
      interleave<W::kBf16, MT * NP>();
      r0 += 64;
    };
    while (r0 < t1) {
      step(kb2, ka);
      if (r0 >= t1) break;
      step(ka, kb2);
    }
  }
  __shared__ float sm[4][16 * MT], sl[4][16 * MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    float top = fmaxf(-nref[i], __shfl_xor(-nref[i], 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    float s = (l[i] + li[i]) * exp2_fast(-nref[i] - top);
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
    float s = 0.0f;
    for (int y = 0; y < 4; ++y) s += sl[y][tid] * exp2_fast(sm[y][tid] - top);
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
  float top = kNoMax, l = 0.0f;
  const float2* src = ml + (live ? ur : 0) * chunks;
  for (int s = threadIdx.x & 15; s < chunks; s += 16) top = fmaxf(top, src[s].x);
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
  for (int s = threadIdx.x & 15; s < chunks; s += 16) l += src[s].y * exp2_fast(src[s].x - top);
#pragma unroll
  for (int x = 8; x > 0; x >>= 1) l += __shfl_xor(l, x);
  if (live && (threadIdx.x & 15) == 0)
    // rows of a unit: heads h G .. h G + G - 1, so [U][R] is [B][L][H_q][w]
    lse[ur] = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
}

template <typename T, int D, int MT>
static hipError_t rows_typed(const AttnLaunch& A, const WeightsSpace& w, const RowArgs<T>& p) {
  const Geo& g = A.base.geo;
  attn_rows_kernel<T, D, MT>
      <<<(unsigned)((int64_t)g.U * w.row_blocks * w.chunks), kThreads, 0, A.base.stream>>>(
          g, A.at, p, w.chunk, w.chunks, w.row_blocks);
  return hipGetLastError();
}

template <typename T, int D>
static hipError_t rows_tiles(const AttnLaunch& A, const WeightsSpace& w, const RowArgs<T>& p) {
  if constexpr (sizeof(T) == 2) {
    if (w.mt == 8) return rows_typed<T, D, 8>(A, w, p);
    if (w.mt == 4) return rows_typed<T, D, 4>(A, w, p);
  }
  return rows_typed<T, D, 2>(A, w, p);
}

template <typename T, int D>
static hipError_t lse_typed(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                            const float* acc, float* lse) {
  const Geo& g = A.base.geo;
  RowArgs<T> p{(const T*)q, (const T*)k, acc, lse, ws_ptr<float2>(A.base.wsp, w.ml)};
  const hipError_t e = rows_tiles<T, D>(A, w, p);
  if (e != hipSuccess || w.chunks == 1) return e;
  const int64_t rows = (int64_t)g.U * A.at.R;
  attn_lse_join_kernel<<<(unsigned)((rows + 15) / 16), kThreads, 0, A.base.stream>>>(
      g, A.at, p.ml, lse, w.chunks);
  return hipGetLastError();
}

hipError_t launch_attn_lse(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                           const float* acc, float* lse) {
  const bool wide = A.base.geo.D == 128;
  if (A.base.cfg->dtype == JACAP_DTYPE_BF16)
    return wide ? lse_typed<__bf16, 128>(A, w, q, k, acc, lse)
                : lse_typed<__bf16, 64>(A, w, q, k, acc, lse);
  return wide ? lse_typed<float, 128>(A, w, q, k, acc, lse)
              : lse_typed<float, 64>(A, w, q, k, acc, lse);
}

// ---------------------------------------------------------------------------
// Sums: a workgroup takes 64 NT tokens of a unit, 16 NT per wave with their keys in
// registers, and a part of the rows, a stage of them at a time through LDS (two
// buffers, the next rows requested a stage ahead). A lane adds the weights its
// query row gives its tokens; the 16 lanes of a tile's rows are added at the
// end. DRAFT: the tokens are the drafted ones, seen by the tree's mask.
// The weights of a whole prompt are many and may be nearly equal (a token that every row
// attends to), and one by one in fp32 they would round to the same side: R = 524288 rows of
// weights near 0.9 lose 5e-5 of their sum, however exact each is. kSumFlush stages (of 64 rows
// in bf16, 32 in fp32: at most 64 additions a lane) are summed in fp32, their sums in fp64.
// ---------------------------------------------------------------------------
constexpr int kSumFlush = 16;

template <typename T>
struct SumArgs {
  const T *q, *k;
  const float* lse;   // [B][L][H_q][w]
  float* acc;         // updated with one row part (drafts: [U][S], written)
  float* part;        // else [row_splits][L][H][T]
  uint32_t* status;   // or null
};

template <typename T, int D, int NT, bool DRAFT>
__global__ __launch_bounds__(kThreads, D == 64 ? 3 : 2) void attn_sum_kernel(Geo g, Attn at, SumArgs<T> p, int blocks,
                                                            int row_splits) {
  using W = Row<T, D>;
  constexpr int NP = W::kPieces;
  constexpr int TILES = W::kBf16 ? 4 : 2;        // 16-row tiles per stage
  constexpr int ROWS = 16 * TILES;
  constexpr int PW = TILES * NP / 4;             // pieces per thread and stage, of one row
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // units innermost, as above; a causal prompt's first tokens, which the most rows
  // see, first
  const int u = blockIdx.x % g.U, x = blockIdx.x / g.U;
  const int part = x % row_splits, blk = x / row_splits;
  const Unit un = live_unit(g, u);
  const int n = DRAFT ? g.w : un.n;
  const int btok = blk * 64 * NT;            // the workgroup's first token
  const int tok = btok + wave * 16 * NT;     // the wave's
  const int R = at.R, w = g.w;
  const bool causal = !DRAFT && at.causal;
  const int first = causal ? un.n - w : 0;
  const int stages = (R + ROWS - 1) / ROWS;
  const int per = (stages + row_splits - 1) / row_splits;
  const int stage1 = min(stages, (part + 1) * per);

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

    // Staged rows lie as the MFMA takes them: piece a of tile h, 16 bytes per lane.
    __shared__ __align__(16) uint4 rows_lds[2][TILES][NP][64];
    struct Meta { float lse, weight; int last, pos; };  // last position seen, -1: adds nothing
    __shared__ Meta meta[2][ROWS];
    // The row a thread stages: row m of tile `stile`, pieces sa .. sa + PW - 1. Its head
    // and position are carried from stage to stage (a division each would cost more
    // than a row's logits).
    const int stile = wave * PW / NP, sa = wave * PW % NP;
    int stage = 0, row = 0, pos = 0, head = 0;
    int p0 = 0, h0 = 0;  // of the stage's first row
    auto seek = [&](int to) {
      stage = to;
      h0 = to * ROWS / w;
      p0 = to * ROWS - h0 * w;
      row = to * ROWS + stile * 16 + m;
      head = row / w;
      pos = row - head * w;
    };
    // The next stage with a row that sees the workgroup's tokens: stages of one
    // head whose positions all lie before them are skipped.
    auto skip = [&] {
      while (causal && stage < stage1 && p0 + ROWS <= w && first + p0 + ROWS - 1 < btok)
        seek((h0 * w + min(w, btok - first)) / ROWS);
    };
    auto advance = [&] {
      ++stage;
      p0 += ROWS;
      while (p0 >= w) {
        p0 -= w;
        ++h0;
      }
      row += ROWS;
      pos += ROWS;
      while (pos >= w) {
        pos -= w;
        ++head;
      }
      skip();
    };
    uint4 held[PW];
    Meta mine;
    auto fetch = [&] {
      // (rows past the last are its copies, and add nothing)
      const int hh = row < R ? head : g.G - 1, pp = row < R ? pos : w - 1;
      const char* src = reinterpret_cast<const char*>(qu + hh * g.qsh + pp * g.qsp) + 64 * sa + 16 * qg;
#pragma unroll
      for (int i = 0; i < PW; ++i) held[i] = *reinterpret_cast<const uint4*>(src + 64 * i);
      mine.lse = lseu[min(row, R - 1)];
      mine.weight = rwu ? rwu[pp] : 1.0f;
      mine.pos = pp;
      mine.last = row < R ? (causal ? first + pp : INT32_MAX) : -1;
    };
    auto store = [&](int buf) {
      const bool live = mine.last >= 0 && mine.weight != 0.0f && mine.lse != -INFINITY;
#pragma unroll
      for (int i = 0; i < PW; ++i)
        rows_lds[buf][stile][sa + i][lane] = live ? held[i] : uint4{0, 0, 0, 0};
      if (sa == 0 && qg == 0)
        meta[buf][stile * 16 + m] = Meta{live ? mine.lse * kLog2e : 0.0f, live ? mine.weight : 0.0f,
                                         live ? mine.last : -1, mine.pos};
    };

    // z: the logits of the last row tile, not added yet; its rows' lse and weight
    // sum: the weights of the last kSumFlush stages, by row; total: of those before, each
    // token's read and written by one lane. In LDS, and the registers bounded: three waves
    // of d = 64 share a SIMD so (a prompt of 8192: 480 us, 512 with total in registers).
    f32x4 sum[NT], z[NT];
    __shared__ double total[64 * NT];
    float ls = 0.0f, weight = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      z[t] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    }
    auto flush = [&](bool first) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        double& x = total[(wave * NT + t) * 16 + 4 * qg + (m & 3)];
        const float mine = tile_sum(sum[t], m);
        if (m < 4) x = first ? (double)mine : x + (double)mine;
        sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    auto add = [&](int t) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sum[t][e] = __builtin_fmaf(exp2_fast(__builtin_fmaf(z[t][e], at.c, -ls)), weight, sum[t][e]);
    };
    int buf = 0, done = 0;
    seek(part * per);
    skip();
    bool more = stage < stage1;
    if (more) {
      fetch();
      store(0);
    }
    __syncthreads();
    while (more) {
      advance();
      more = stage < stage1;
      if (more) fetch();
      Meta me[TILES];
      bool masked = DRAFT;
#pragma unroll
      for (int h = 0; h < TILES; ++h) {
        me[h] = meta[buf][16 * h + m];
        masked = masked || __ballot(me[h].last < tok + 16 * NT) != 0;
      }
      auto row_tile = [&](int h, uint4 (&qf)[NP]) {
#pragma unroll
        for (int a = 0; a < NP; ++a)
          qf[a] = rows_lds[buf][h][a][lane];
      };
      if (!masked) {
        // Every row sees every token: no branch in here. z holds the tile before; each
        // of its logits is added and the new tile's formed in its place, so that the
        // exponentials run beside the products, across the stages' ends too.
#pragma unroll
        for (int h = 0; h < TILES; ++h) {
          uint4 qf[NP];
          row_tile(h, qf);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            add(t);
            z[t] = logits<T, D>(kf[t], qf);
          }
          ls = me[h].lse;
          weight = me[h].weight;
        }
      } else {
#pragma unroll
        for (int h = 0; h < TILES; ++h) {
          // nothing to add where no row of the tile sees a token of the wave
          if (__ballot(me[h].last >= tok) == 0) continue;
          uint4 qf[NP];
          row_tile(h, qf);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            add(t);
            z[t] = logits<T, D>(kf[t], qf);
            uint32_t bits = 0;
            if constexpr (DRAFT) {
              const int j0 = tok + 16 * t;
              if (me[h].last >= 0 && j0 < n) {
                if (at.tree)
                  bits = at.tree[((int64_t)un.b * w + me[h].pos) * at.tree_words + (j0 >> 5)] >> (j0 & 31);
                else
                  bits = me[h].pos < j0 ? 0u : me[h].pos - j0 >= 31 ? ~0u : (2u << (me[h].pos - j0)) - 1u;
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool see =
                  DRAFT ? (bits >> (4 * qg + e) & 1) : tok + 16 * t + 4 * qg + e <= me[h].last;
              z[t][e] = see ? z[t][e] : -INFINITY;
            }
          }
          ls = me[h].lse;
          weight = me[h].weight;
        }
      }
      if (more) store(buf ^ 1);
      if ((++done & (kSumFlush - 1)) == 0) flush(done == kSumFlush);
      __syncthreads();
      buf ^= 1;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) add(t);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float mine = tile_sum(sum[t], m);
      if (done >= kSumFlush && m < 4)
        mine = (float)(total[(wave * NT + t) * 16 + 4 * qg + (m & 3)] + (double)mine);
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
            if (!(old < 0.0f)) p.acc[i] = decayed(at, old, mine);
          }
        }
      }
    }
  }
  if (blockIdx.x == 0 && p.status) write_status(g, p.status);
}

// ---------------------------------------------------------------------------
// Sums from the few rows of a window or a tree: all of a unit's rows lie in LDS for the
// whole of a workgroup's stretch of tokens. A wave takes its stretch's blocks of 16 NT tokens in turn (their keys in registers, the next block's
// requested during the last row tile) past the rows, with no barrier after the first.
// z is carried over the blocks' ends too: a block's last logits are added, and its
// accumulators written, as the next one's first are formed. A tile of 16 x 16 logits
// is 96 cycles of vector instructions (an FMA, an exponential at a quarter of the rate
// and an FMA per logit) and 64 of MFMA at d = 128: busy 59% and 40% of the cycles, 10% both
// at once. 256 rows, 32 units of 131072 tokens: 320 us, 430 over calls without a pause, as
// the clock falls; a large library product of as many operations takes 240, and with the
// rows staged for every 256 tokens it was 530 to 590.
// ---------------------------------------------------------------------------
template <typename T, int D, int NT>
__global__ __launch_bounds__(kThreads, 2) void attn_sum_held_kernel(Geo g, Attn at, SumArgs<T> p,
                                                                   int chunk) {
  using W = Row<T, D>;
  constexpr int NP = W::kPieces, WAVES = kThreads / 64;
  constexpr int STAGE = W::kBf16 ? 4 : 2;  // row tiles unrolled
  constexpr int ROWS = held_rows(W::kBytes);
  constexpr int STEP = 16 * NT * WAVES;
  const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, qg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int u = blockIdx.x % g.U;
  const Unit un = live_unit(g, u);
  const int begin = blockIdx.x / g.U * chunk, end = begin + min(chunk, un.n - begin);
  const int R = at.R, w = g.w;
  const int first = un.n - w;  // position of row 0 (causal)
  __shared__ __align__(16) uint4 rows_lds[ROWS / 16][NP][64];  // as the MFMA takes them
  struct Meta { float lse, weight; };
  __shared__ Meta meta[ROWS];
  __shared__ int last_lds[ROWS];  // last position seen, -1: adds nothing
  // The row tiles with a row that adds nothing: its logits are replaced, since 0 times the
  // weight of a key that holds an infinity or NaN would not be 0.
  __shared__ uint32_t dead_lds[ROWS / 16];

  if (begin < end) {
    const T* kb = p.k + un.l * g.ksl + un.h * g.ksh + un.t0 * g.kst;
    const int32_t ks = (int32_t)(g.kst * sizeof(T));
    float* accu = p.acc + token_row(g, un);
    uint4 kf[NT][NP];
    float old[NT];
    int tok = begin + wave * 16 * NT;
    auto fetch = [&](int t, int b) {  // tile t of the block at b (zeros past the stretch's end)
      const int r0 = b + 16 * t;
      const auto kr = buffer_range(kb + r0 * g.kst, rows_bytes(min(16, end - r0), ks, W::kBytes));
#pragma unroll
      for (int a = 0; a < NP; ++a) kf[t][a] = buffer_load16(kr, m * ks + 64 * a + 16 * qg);
    };
#pragma unroll
    for (int t = 0; t < NT; ++t) fetch(t, tok);

    const T* qu = unit_queries(g, un, p.q);
    const float* lseu = p.lse + ((int64_t)un.b * g.L + un.l) * g.Hq * w + (int64_t)un.h * R;
    const float* rwu = at.row_weight ? at.row_weight + (int64_t)un.b * w : nullptr;
    const int stages = (R + 16 * STAGE - 1) / (16 * STAGE);
    for (int h = wave; h < STAGE * stages; h += WAVES) {
      const int row = min(16 * h + m, R - 1), pos = row % w;
      const float lse = lseu[row], weight = rwu ? rwu[pos] : 1.0f;
      // (rows past the last are its copies, and add nothing)
      const bool live = 16 * h + m < R && weight != 0.0f && lse != -INFINITY;
      uint4 qf[NP];
      load_row<T, D>(g, qu, row, live, qg, qf);
#pragma unroll
      for (int a = 0; a < NP; ++a) rows_lds[h][a][lane] = qf[a];
      if (qg == 0) {
        meta[16 * h + m] = Meta{live ? lse * kLog2e : 0.0f, live ? weight : 0.0f};
        last_lds[16 * h + m] = !live ? -1 : at.causal ? first + pos : INT32_MAX;
      }
      const bool any = __ballot(!live) != 0;
      if (lane == 0) dead_lds[h] = any;
    }
    __syncthreads();
    const uint32_t dead = (uint32_t)__ballot(lane < STAGE * stages && dead_lds[lane % (ROWS / 16)]);

    f32x4 sum[NT], z[NT];
    float ls = 0.0f, weight = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[t] = z[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](int t) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sum[t][e] = __builtin_fmaf(exp2_fast(__builtin_fmaf(z[t][e], at.c, -ls)), weight, sum[t][e]);
    };
    // the accumulators of the block at b
    auto entries = [&](int b) {
#pragma unroll
      for (int t = 0; t < NT; ++t) old[t] = accu[min(b + 16 * t + 4 * qg + (m & 3), end - 1)];
    };
    auto write = [&](int t, int b) {
      const float mine = tile_sum(sum[t], m);
      const int j = b + 16 * t + 4 * qg + m;
      if (m < 4 && j < end && !(old[t] < 0.0f)) accu[j] = decayed(at, old[t], mine);
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    int before = -1;  // the block whose last logits z holds
    for (; tok < end; tok += STEP) {
      const bool edge = at.causal && tok + 16 * NT > first + 1;
      const uint32_t masked = edge ? ~0u : dead;  // row tiles
      for (int s = 0; s < stages; ++s) {
#pragma unroll
        for (int x = 0; x < STAGE; ++x) {
          const int h = s * STAGE + x;
          uint4 qf[NP];
#pragma unroll
          for (int a = 0; a < NP; ++a) qf[a] = rows_lds[h][a][lane];
          const Meta me = meta[16 * h + m];
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            add(t);
            z[t] = logits<T, D>(kf[t], qf);
          }
          if (x == 0 && s == 0) {
            if (before >= 0) {
#pragma unroll
              for (int t = 0; t < NT; ++t) write(t, before);
            }
            entries(tok);
            before = tok;
          }
          if (masked >> h & 1) {
            if (edge) {
              const int last = last_lds[16 * h + m];
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  z[t][e] = tok + 16 * t + 4 * qg + e <= last ? z[t][e] : -INFINITY;
            } else {
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) z[t][e] = me.weight != 0.0f ? z[t][e] : -INFINITY;
            }
          }
          ls = me.lse;
          weight = me.weight;
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) fetch(t, tok + STEP);
    }
    if (before >= 0) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        add(t);
        write(t, before);
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
  double sum = 0.0;
  for (int s = 0; s < row_splits; ++s) sum += (double)part[s * pitch + tr + t];
  acc[tr + t] = decayed(at, old, (float)sum);
}

template <typename T, int D, int NT>
static hipError_t sum_typed(const AttnLaunch& A, const WeightsSpace& w, const void* q, const void* k,
                            const float* lse, float* acc, uint32_t* status) {
  const Geo& g = A.base.geo;
  float* part = ws_ptr<float>(A.base.wsp, w.part);
  hipError_t e;
  if (w.held) {
    attn_sum_held_kernel<T, D, NT>
        <<<(unsigned)((int64_t)g.U * std::max(1, w.blocks)), kThreads, 0, A.base.stream>>>(
            g, A.at, SumArgs<T>{(const T*)q, (const T*)k, lse, acc, nullptr, status}, w.held);
    e = hipGetLastError();
  } else {
    SumArgs<T> p{(const T*)q, (const T*)k, lse, acc, part, status};
    attn_sum_kernel<T, D, NT, false>
        <<<(unsigned)((int64_t)g.U * std::max(1, w.blocks) * w.row_splits), kThreads, 0,
           A.base.stream>>>(g, A.at, p, w.blocks, w.row_splits);
    e = hipGetLastError();
  }
  if (e != hipSuccess || w.row_splits == 1 || g.maxn == 0) return e;
  attn_sum_join_kernel<<<dim3((g.maxn + kThreads - 1) / kThreads, g.U), kThreads, 0, A.base.stream>>>(
      g, A.at, part, acc, w.row_splits);
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
