// jacap_verify: which drafted tokens the target accepts, and its next one.
//
// The first kernel reads every row's logits once, for its largest and the sum of its
// exponentials (greedy: the place of the largest): bound by that read (1024 rows of 128256
// bf16 logits, 263 MB: 47 us, 5.6 TB/s). The second walks
// from row 0 to the last accepted one. Its tests need one logit (and one draft
// probability) of each row's token, fetched for all rows at once; then the draw passes
// over the last row again, from L2, a slice a workgroup, and the workgroup that finishes
// last joins the slices' sums and finds the token in one of them. Every slice's workgroup walks
// for itself: it costs less than a launch while the walk needs no sum over the vocabulary. With
// draft probabilities it needs one for every further sibling of a rejected row, and each of the
// sequence's workgroups makes it for itself: 64 us a sibling at 128256 tokens (16 sequences of
// one row and 1, 2, 4 and 8 children that are mostly rejected: 24, 97, 236 and 483 us), 18 at
// 32000.
//
// (16 trees of 64 rows: 16.5 us; 31 before lanes shared a row's parts and the draw's place.)
//
// The draw's sums are fp64: the exponentials have 24 bits, and the draw's border must not move
// with the order in which 128256 of them are added. A row's total is fp64 too, of the
// exponentials of 16 bytes of logits added in fp32 first.
#include <type_traits>

#include "verify.hpp"

namespace jacap {

namespace {

constexpr int kSliceVecs = kVerifyThreads * kVerifyVecs;
constexpr int kRowLanes = 4;  // that join the parts of a row

// How far a row's total may be from the sum of the weights that the draw uses, relative to it.
// Of a weight 2^-a (at most 1, the largest's): a pair's fp32 additions 3 x 2^-24; two exponents
// of about a, each the product of a rounded difference, 4 a 2^-24; the joins of up to 2048 slices
// by four lanes, 2^-23 for each that raises the maximum, at most 520 in a row. The weights' mean
// of a is at most log2 V <= 24, so all are below (3 + 96 + 1040) 2^-24 < 2^-13.
constexpr double kTotalError = 0x1p-13;
// ... and of the sum of at most 2^24 weights by 256 threads in fp64: 2^16 + 10 additions in a row.
constexpr double kSumError = 0x1p-36;

// A row of V logits as 16-byte pieces: piece v holds elements v VE - off .., off that of the
// row's first in its own. lo .. hi are the pieces inside the row.
template <typename T>
struct LogitRow {
  static constexpr int VE = 16 / (int)sizeof(T);
  const T* base;
  int off, V, pieces, lo, hi;
  __device__ __forceinline__ LogitRow(const T* row, int V_) : base(row), V(V_) {
    off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    pieces = (off + V + VE - 1) / VE;
    lo = off > 0 ? 1 : 0;
    hi = (off + V) / VE - 1;
  }
  __device__ __forceinline__ bool inside(int v) const { return v >= lo && v <= hi; }
  // Pieces v0, v0 + step ... as fp32, -inf outside the row. The loads are requested together,
  // with no branch between them (a branch each, and each was waited for: 1024 rows of
  // 128256 62 us, 46 so); a piece at an end of the row is put in afterwards.
  template <int N>
  __device__ __forceinline__ void load(int v0, int step, float (&x)[N][VE]) const {
    uint4 y[N];
    if (lo <= hi) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        y[i] = *reinterpret_cast<const uint4*>(base + min(max(v0 + i * step, lo), hi) * VE - off);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t w[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
        const bool in = inside(v0 + i * step);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const uint32_t u = sizeof(T) == 4 ? w[e * (int)sizeof(T) / 4]
                                            : (e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16;
          x[i][e] = in ? __uint_as_float(u) : -INFINITY;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) x[i][e] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = v0 + i * step;
      if (v >= 0 && v < pieces && !inside(v)) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int at = v * VE - off + e;
          if (at >= 0 && at < V) x[i][e] = (float)base[at];
        }
      }
    }
  }
  // The same of the draft's probabilities q of the row (0 outside).
  template <int N>
  __device__ __forceinline__ void load_draft(const float* q, int v0, int step, float (&x)[N][VE]) const {
    const bool whole = (reinterpret_cast<uintptr_t>(q - off) & 15) == 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = v0 + i * step, first = min(max(v, lo), hi) * VE - off;
      if (whole && lo <= hi) {
#pragma unroll
        for (int e = 0; e < VE; e += 4) {
          const float4 y = *reinterpret_cast<const float4*>(q + first + e);
          x[i][e] = y.x;
          x[i][e + 1] = y.y;
          x[i][e + 2] = y.z;
          x[i][e + 3] = y.w;
        }
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) x[i][e] = q[min(max(v * VE - off + e, 0), V - 1)];
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = v0 + i * step;
      if (!inside(v)) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const int at = v * VE - off + e;
          x[i][e] = at >= 0 && at < V ? q[at] : 0.0f;
        }
      }
    }
  }
};

__device__ __forceinline__ float expo(float z, float top, float k) { return __builtin_amdgcn_exp2f((z - top) * k); }

// What is left of e after c q; a NaN stays one.
__device__ __forceinline__ double rest(double e, double c, double q) {
  const double w = e - c * q;
  return w < 0.0 ? 0.0 : w;
}

template <typename T, typename Op>
__device__ __forceinline__ T block_all(T v, T* red, Op op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T r = red[0];
#pragma unroll
  for (int i = 1; i < kVerifyThreads / 64; ++i) r = op(r, red[i]);
  return r;
}

// A piece's values added pair by pair.
template <int N>
__device__ __forceinline__ float add_pairs(const float (&x)[N]) {
  float y[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) y[i] = x[2 * i] + x[2 * i + 1];
  if constexpr (N == 2) return y[0];
  else return add_pairs(y);
}

// The largest of two parts, and their sums in units of it. (A part of -inf only has the sum
// 0; one with a NaN or +inf a NaN, which stays.)
__device__ __forceinline__ void join(float& top, double& sum, float t, double s, float k) {
  const float now = fmaxf(top, t);
  sum = (sum == 0.0 ? 0.0 : sum * (double)expo(top, now, k)) + (s == 0.0 ? 0.0 : s * (double)expo(t, now, k));
  top = now;
}

}  // namespace

// A wave keeps kRowVecs pieces a lane in registers between its own maximum and its sum: the
// waves meet once, at the end. Eight exponentials are added in fp32 pair by pair (three
// roundings beside their own), the rest in fp64: a conversion and an addition for each would be
// as much vector work as the exponentials.
template <typename T, bool GREEDY>
__global__ __launch_bounds__(kVerifyThreads) void verify_rows_kernel(VerifyLaunch p) {
  using Row = LogitRow<T>;
  constexpr int VE = Row::VE, WAVES = kVerifyThreads / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / p.row_slices, slice = blockIdx.x - row * p.row_slices;
  const int b = row / p.S, r = row - b * p.S;
  if (blockIdx.x == 0) {
    for (int i = tid; i < p.B; i += kVerifyThreads) p.arrived[i] = 0;
    if (tid == 0) *p.status = 0;
  }
  const Row z((const T*)p.logits + b * p.lss + r * p.lsr, p.V);
  const int v0 = (slice * WAVES + wave) * kRowVecs * 64 + lane;
  float x[kRowVecs][VE];
  z.load(v0, 64, x);
  RowPart* part = p.parts + blockIdx.x;
  if constexpr (GREEDY) {
    float top = -INFINITY;
    int at = INT32_MAX;
#pragma unroll
    for (int i = 0; i < kRowVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (x[i][e] > top) {  // (never a NaN; in ascending order)
          top = x[i][e];
          at = (v0 + 64 * i) * VE - z.off + e;
        }
    auto take = [&](float t, int a) {
      const bool more = t > top || (t == top && a < at);
      top = more ? t : top;
      at = more ? a : at;
    };
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) take(__shfl_xor(top, o), __shfl_xor(at, o));
    __shared__ float tops[WAVES];
    __shared__ int ats[WAVES];
    if (lane == 0) {
      tops[wave] = top;
      ats[wave] = at;
    }
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < WAVES; ++i) take(tops[i], ats[i]);
      *part = RowPart{top, at, 0.0};
    }
  } else {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kRowVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) top = fmaxf(top, x[i][e]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float ref = top == -INFINITY ? 0.0f : top;  // (a wave's all -inf: its sum is 0)
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kRowVecs; ++i) {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[i][e] = expo(x[i][e], ref, p.k);
      sum += (double)add_pairs(x[i]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    __shared__ float tops[WAVES];
    __shared__ double sums[WAVES];
    if (lane == 0) {
      tops[wave] = top;
      sums[wave] = sum;
    }
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < WAVES; ++i) join(top, sum, tops[i], sums[i], p.k);
      *part = RowPart{top, 0, sum};
    }
  }
}

// The path is the sequence's alone: the workgroup of its first slice writes it.
template <typename T, bool GREEDY>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(VerifyLaunch p) {
  using Row = LogitRow<T>;
  constexpr int VE = Row::VE;
  const int tid = threadIdx.x, lane = tid & 63;
  const int slices = GREEDY ? 1 : p.slices;
  const int b = blockIdx.x / slices, slice = blockIdx.x - b * slices;
  const int S = p.S;
  __shared__ float top[kMaxVerifyRows];      // a row's largest logit
  __shared__ double total[kMaxVerifyRows];   // ... its sum of exponentials (NaN: not to be used)
  __shared__ int16_t parent[kMaxVerifyRows]; // -1: not tested
  __shared__ int32_t token[kMaxVerifyRows];  // of a row; greedy: ...
  __shared__ int32_t best[GREEDY ? kMaxVerifyRows : 1];  // the row's own choice (-1: none)
  __shared__ float weight[kMaxVerifyRows];   // exponential of the row's token at its parent
  __shared__ float chance[kMaxVerifyRows];   // its draft probability there
  __shared__ uint8_t taken[kMaxVerifyRows];  // the row is accepted
  __shared__ int16_t gone[kMaxVerifyRows];   // rejected children of the current row
  __shared__ double redd[kVerifyThreads / 64];
  __shared__ float uniform[kMaxVerifyRows];  // its number
  __shared__ int at_row, at_next, num_gone, num_path;
  __shared__ double mult, left;              // C; N, what is left of the weights (greedy: not used)

  const T* const logits = (const T*)p.logits + b * p.lss;
  const float* const draft = p.draft ? p.draft + b * p.qss : nullptr;
  // A row's parent, token and number, and its token's logit at the parent (requested
  // before the rows' statistics, which kRowLanes lanes a row join).
  for (int r = tid; r < S; r += kVerifyThreads) {
    const int up = r == 0 ? -1 : p.parents ? p.parents[(int64_t)b * S + r] : r - 1;
    const int x = r == 0 ? -1 : p.tokens[(int64_t)b * S + r];
    const bool tested = up >= 0 && up < r && (uint32_t)x < (uint32_t)p.V;
    parent[r] = (int16_t)(tested ? up : -1);
    token[r] = x;
    taken[r] = r == 0;
    if constexpr (!GREEDY) {
      uniform[r] = p.uniform[(int64_t)b * S + r];
      weight[r] = tested ? (float)logits[up * p.lsr + x] : 0.0f;
      chance[r] = tested && draft ? draft[up * p.qsr + x] : 0.0f;
    }
  }
  for (int r0 = 0; r0 < S; r0 += kVerifyThreads / kRowLanes) {
    const int r = r0 + tid / kRowLanes, sub = tid % kRowLanes;
    const RowPart* parts = p.parts + ((int64_t)b * S + min(r, S - 1)) * p.row_slices;
    float t = -INFINITY;
    if constexpr (GREEDY) {
      int a = INT32_MAX;
      auto take = [&](float y, int z) {
        if (y > t || (y == t && z < a)) {
          t = y;
          a = z;
        }
      };
      for (int i = sub; i < p.row_slices; i += kRowLanes) take(parts[i].top, parts[i].at);
#pragma unroll
      for (int o = kRowLanes / 2; o > 0; o >>= 1) take(__shfl_xor(t, o), __shfl_xor(a, o));
      if (sub == 0 && r < S) best[r] = t > -INFINITY ? a : -1;
    } else {
      double s = 0.0;
#pragma unroll 4
      for (int i = sub; i < p.row_slices; i += kRowLanes) {
        const RowPart part = parts[i];
        join(t, s, part.top, part.sum, p.k);
      }
#pragma unroll
      for (int o = kRowLanes / 2; o > 0; o >>= 1) {
        const float y = __shfl_xor(t, o);
        const double z = __shfl_xor(s, o);
        join(t, s, y, z, p.k);
      }
      if (sub == 0 && r < S) {
        top[r] = t;
        total[r] = t > -INFINITY ? s : __builtin_nan("");
      }
    }
  }
  if (tid == 0) {
    at_row = 0;
    at_next = 1;
    num_gone = 0;
    num_path = 1;
    mult = 0.0;
  }
  __syncthreads();
  if constexpr (!GREEDY) {
    for (int r = tid; r < S; r += kVerifyThreads)
      if (parent[r] >= 0) weight[r] = expo(weight[r], top[parent[r]], p.k);
    if (tid == 0) left = total[0];
    __syncthreads();
  }
  // The weights max(e - mul q, 0) of pieces v0, v0 + step ... of a row z of largest logit t (0
  // outside it), those of the first n_gone rejected tokens 0.
  auto weights = [&](const Row& z, const float* q, float t, double mul, int n_gone, int v0, int step,
                     double (&w)[kVerifyVecs][VE]) __attribute__((always_inline)) {
    float x[kVerifyVecs][VE], y[kVerifyVecs][VE];
    z.load(v0, step, x);
    if (mul != 0.0) z.load_draft(q, v0, step, y);
    uint32_t out = 0;  // bit VE i + e: a rejected token
    for (int g = 0; g < n_gone; ++g) {
      const int x = token[gone[g]] + z.off, v = x / VE - v0;
      if (v >= 0 && v % step == 0 && v / step < kVerifyVecs) out |= 1u << (v / step * VE + x % VE);
    }
#pragma unroll
    for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        w[i][e] = (double)(out >> (VE * i + e) & 1 ? 0.0f : expo(x[i][e], t, p.k));
        if (mul != 0.0) w[i][e] = rest(w[i][e], mul, (double)y[i][e]);
      }
  };
  // One sweep over the rows in order meets every child of an accepted row after it. Without draft
  // probabilities N is the row's total less the rejected tokens' weights, which may be wrong by as
  // much as the total is: a test that this could turn is made with the sum of the weights
  // themselves, which a last child that has all that is left needs (16 trees of 64 rows: 16.5
  // us, 15.5 without).
  for (bool summed = false;; summed = true) {  // summed: N is that sum, for the first test
    if (tid < 64) {
      // (every lane has the same values, and stores them; the ballots tell the compiler so)
      int row = at_row, n_gone = num_gone, n_path = num_path, r = at_next;
      double c = mult, n = GREEDY ? 0.0 : left;
      bool stale = false, stop = false;  // N is not that of the weights
      bool fresh = summed;
      double slack = GREEDY ? 0.0 : summed ? n * kSumError : n * kTotalError;  // N is known to
      for (int r0 = r & ~63; r0 < S && !stop; r0 += 64) {
        const int up = r0 + lane < S ? parent[r0 + lane] : -1;
        uint64_t todo = __ballot(up == row) & (r > r0 ? ~0ull << (r - r0) : ~0ull);
        while (todo) {
          const int i = __builtin_ctzll(todo);
          r = r0 + i;
          if (stale) {
            stop = true;
            break;
          }
          todo &= todo - 1;
          bool accept;
          if constexpr (GREEDY) {
            accept = token[r] == best[row];
          } else {
            const double u = (double)uniform[r], e = (double)weight[r];
            if (draft) {
              const double q = (double)chance[r];
              accept = __ballot(u * q * n < rest(e, c, q)) != 0;
              if (!accept) {
                c += n;
                stale = true;
              }
            } else {
              bool again = false;  // the token of a sibling already rejected
              for (int y = lane; y < n_gone; y += 64) again |= token[gone[y]] == token[r];
              again = __ballot(again) != 0 || e == 0.0;
              const double past = u * n - e, far = fresh ? 0.0 : slack;
              accept = __ballot(!again && past < -far) != 0;
              if (!accept && __ballot(!again && past <= far && far > 0.0) != 0) {
                stop = true;
                break;
              }
              if (!accept && !again) {
                gone[n_gone++] = (int16_t)r;
                n = rest(n, 1.0, e);
                fresh = false;
              }
            }
          }
          if (accept) {
            row = r;
            taken[r] = 1;
            ++n_path;
            n_gone = 0;
            c = 0.0;
            stale = false;
            fresh = false;
            if (!GREEDY) {
              n = total[row];
              slack = n * kTotalError;
            }
            todo = __ballot(up == row) & (i == 63 ? 0ull : ~0ull << (i + 1));
          }
        }
        if (!stop) r = max(r, r0 + 64);
      }
      if (lane == 0) {
        at_row = row;
        at_next = stop ? r : S;
        num_gone = n_gone;
        num_path = n_path;
        mult = c;
        if (!GREEDY) left = n;
      }
    }
    __syncthreads();
    if (at_next >= S) break;
    // N by the whole workgroup
    if constexpr (!GREEDY) {
      const int row = at_row, n_gone = num_gone;
      const double c = mult;
      const Row z(logits + row * p.lsr, p.V);
      const float* q = draft ? draft + row * p.qsr : nullptr;
      const float t = top[row];
      double sum = 0.0;
      for (int v = tid; v < z.pieces; v += kVerifyThreads * kVerifyVecs) {
        double w[kVerifyVecs][VE];
        weights(z, q, t, c, n_gone, v, kVerifyThreads, w);
#pragma unroll
        for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
          for (int e = 0; e < VE; ++e) sum += w[i][e];
      }
      sum = block_all(sum, redd, [](double a, double d) { return a + d; });
      if (tid == 0) left = sum;
    }
    __syncthreads();
  }
  const int row = at_row;
  if (slice == 0) {
    // the accepted rows in order: ascending, as each comes after its parent
    __shared__ uint64_t accepted[kMaxVerifyRows / 64];
    for (int r = tid; r < kMaxVerifyRows; r += kVerifyThreads) {
      const uint64_t mask = __ballot(r < S && taken[r]);
      if (lane == 0) accepted[r >> 6] = mask;
    }
    __syncthreads();
    for (int r = tid; r < S; r += kVerifyThreads) {
      const bool in = accepted[r >> 6] >> (r & 63) & 1;
      int place = __builtin_popcountll(accepted[r >> 6] & ((1ull << (r & 63)) - 1));
      for (int y = 0; y < r >> 6; ++y) place += __builtin_popcountll(accepted[y]);
      if (in) p.path[(int64_t)b * S + place] = r;
      if (r >= num_path) p.path[(int64_t)b * S + r] = -1;
      if (p.row_weight) p.row_weight[(int64_t)b * S + r] = in ? 1.0f : 0.0f;
    }
    if (tid == 0) p.count[b] = num_path;
  }
  if constexpr (GREEDY) {
    if (tid == 0) {
      p.next[b] = best[row];
      if (best[row] < 0) atomicOr(p.status, (uint32_t)JACAP_FLAG_NONFINITE);
    }
  } else {
    const Row z(logits + row * p.lsr, p.V);
    const float* q = draft ? draft + row * p.qsr : nullptr;
    const float t = top[row];
    const double c = mult;
    int n_gone = num_gone;
    auto slice_sum = [&](int s, double mul) __attribute__((always_inline)) {
      double w[kVerifyVecs][VE], sum = 0.0;
      weights(z, q, t, mul, n_gone, s * kSliceVecs + tid, kVerifyThreads, w);
#pragma unroll
      for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) sum += w[i][e];
      return block_all(sum, redd, [](double a, double d) { return a + d; });
    };
    __shared__ int last;
    double* mass = p.mass + (int64_t)b * slices;
    // (known from the row's sum: at a rejected token, whose weight is left out above, it would
    // not be seen below)
    if (!(total[row] < INFINITY)) {  // a NaN or an infinity, or -inf only: not a row to draw from
      if (slice == 0 && tid == 0) {
        p.next[b] = -1;
        atomicOr(p.status, (uint32_t)JACAP_FLAG_NONFINITE);
      }
      return;
    }
    const double mine = slice_sum(slice, c);
    if (tid == 0) {
      __hip_atomic_store(&mass[slice], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(&p.arrived[b], 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
             (uint32_t)slices - 1;
    }
    __syncthreads();
    if (!last) return;
    auto load_mass = [&](int s) {
      return __hip_atomic_load(&mass[s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    // Their sum, and the slice in which the running one passes the goal (else the last of
    // positive sum): 64 slices at a time in the lanes, each wave for itself.
    double mul = c, all = 0.0;
    auto scan = [&](double v) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(v, o);
        if (lane >= o) v += y;
      }
      return v;
    };
    double first = 0.0, upto = 0.0;  // of the slices in the lanes: the first 64's are kept
    auto sum_all = [&] {
      double run = 0.0;
      for (int s = 0; s < slices; s += 64) {
        const double m = s + lane < slices ? load_mass(s + lane) : 0.0, incl = scan(m);
        if (s == 0) {
          first = m;
          upto = incl;
        }
        run += __shfl(incl, 63);
      }
      return run;
    };
    all = sum_all();
    if (all == 0.0 && (c > 0.0 || n_gone > 0)) {  // nothing is left: the row's own weights
      mul = 0.0;
      n_gone = 0;
      __syncthreads();
      for (int s = 0; s < slices; ++s) {
        const double m = slice_sum(s, mul);
        if (tid == 0) __hip_atomic_store(&mass[s], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __threadfence();  // before the barrier: the other waves read what thread 0 stored
      __syncthreads();
      all = sum_all();
    }
    if (!(all > 0.0) || !(all < INFINITY)) {  // draft probabilities to draw by that are not numbers
      if (tid == 0) {
        p.next[b] = -1;
        atomicOr(p.status, (uint32_t)JACAP_FLAG_NONFINITE);
      }
      return;
    }
    const double goal = (double)uniform[0] * all;
    int in = -1;
    double before = 0.0, run = 0.0;
    for (int s = 0; s < slices; s += 64) {
      const double m = s == 0 ? first : s + lane < slices ? load_mass(s + lane) : 0.0;
      const double incl = s == 0 ? upto : run + scan(m);
      const uint64_t some = __ballot(m > 0.0), past = __ballot(m > 0.0 && incl > goal);
      const uint64_t from = past ? past & -past : some;
      if (from) {
        const int i = 63 - __builtin_clzll(from);
        in = s + i;
        before = __shfl(incl - m, i);
      }
      if (past) break;
      run = __shfl(incl, 63);
    }
    // Its pieces, kVerifyVecs in order to a thread.
    double sum = 0.0, w[kVerifyVecs][VE];
    int final = -1;  // the last token of positive weight
    const int v0 = in * kSliceVecs + tid * kVerifyVecs;
    weights(z, q, t, mul, n_gone, v0, 1, w);
#pragma unroll
    for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        sum += w[i][e];
        if (w[i][e] > 0.0) final = (v0 + i) * VE - z.off + e;
      }
    const double incl_wave = scan(sum);
    __syncthreads();
    if (lane == 63) redd[tid >> 6] = incl_wave;
    __syncthreads();
    for (int i = 0; i < tid >> 6; ++i) before += redd[i];
    const double incl = incl_wave;
    int found = INT32_MAX;
    double mass_to = before + (incl - sum);
#pragma unroll
    for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        mass_to += w[i][e];
        if (w[i][e] > 0.0 && mass_to > goal) found = min(found, (v0 + i) * VE - z.off + e);
      }
    // the first thread that found one (they are in the tokens' order), else the last of
    // positive weight
    const uint64_t any = __ballot(found != INT32_MAX), some = __ballot(final >= 0);
    __shared__ int firsts[kVerifyThreads / 64], lasts[kVerifyThreads / 64];
    const int f = any ? __builtin_amdgcn_readlane(found, __builtin_ctzll(any)) : INT32_MAX;
    const int g = some ? __builtin_amdgcn_readlane(final, 63 - __builtin_clzll(some)) : -1;
    if (lane == 0) {
      firsts[tid >> 6] = f;
      lasts[tid >> 6] = g;
    }
    __syncthreads();
    found = firsts[0];
    final = lasts[0];
    for (int i = 1; i < kVerifyThreads / 64; ++i) {
      found = min(found, firsts[i]);
      final = max(final, lasts[i]);
    }
    if (tid == 0) p.next[b] = found != INT32_MAX ? found : final;
  }
}

template <typename T>
static void rows_typed(const VerifyLaunch& A) {
  const unsigned grid = (unsigned)((int64_t)A.B * A.S * A.row_slices);
  if (A.k > 0.0f) verify_rows_kernel<T, false><<<grid, kVerifyThreads, 0, A.stream>>>(A);
  else verify_rows_kernel<T, true><<<grid, kVerifyThreads, 0, A.stream>>>(A);
}

hipError_t launch_verify_rows(const VerifyLaunch& A) {
  if (A.dtype == JACAP_DTYPE_BF16) rows_typed<__bf16>(A);
  else rows_typed<float>(A);
  return hipGetLastError();
}

template <typename T>
static void verify_typed(const VerifyLaunch& A) {
  if (A.k > 0.0f) verify_kernel<T, false><<<(unsigned)(A.B * A.slices), kVerifyThreads, 0, A.stream>>>(A);
  else verify_kernel<T, true><<<(unsigned)A.B, kVerifyThreads, 0, A.stream>>>(A);
}

hipError_t launch_verify(const VerifyLaunch& A) {
  if (A.dtype == JACAP_DTYPE_BF16) verify_typed<__bf16>(A);
  else verify_typed<float>(A);
  return hipGetLastError();
}

}  // namespace jacap
