// jacap_verify: which drafted tokens the target accepts, and its next one.
//
// The first kernel reads every row's logits once, for its largest and the sum of its
// exponentials (greedy: the place of the largest): bound by that read. The second walks
// from row 0 to the last accepted one. Its tests need one logit (and one draft
// probability) of each row's token, fetched for all rows at once; then the draw passes
// over the last row again, from L2, a slice a workgroup, and the workgroup that finishes
// last joins the slices' sums and finds the token in one of them. Every slice's workgroup walks
// for itself: it costs less than a launch.
//
// Sums are fp64: the exponentials have 24 bits, and the draw's border must not move with
// the order in which 128256 of them are added.
#include <type_traits>

#include "verify.hpp"

namespace jacap {

namespace {

constexpr int kSliceVecs = kVerifyThreads * kVerifyVecs;

// A row of V logits as 16-byte pieces: piece v holds elements v VE - off .., off that of the
// row's first in its own.
template <typename T>
struct LogitRow {
  static constexpr int VE = 16 / (int)sizeof(T);
  const T* base;
  int off, V, pieces;
  __device__ __forceinline__ LogitRow(const T* row, int V_) : base(row), V(V_) {
    off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    pieces = (off + V + VE - 1) / VE;
  }
  // The piece's logits as fp32; -inf outside the row.
  __device__ __forceinline__ void load(int v, float (&x)[VE]) const {
    const int x0 = v * VE - off;
    if (x0 >= 0 && x0 + VE <= V) {
      const uint4 y = *reinterpret_cast<const uint4*>(base + x0);
      const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < VE; ++i)
        x[i] = sizeof(T) == 4 ? __uint_as_float(w[i * (int)sizeof(T) / 4])
                              : __uint_as_float((i & 1) ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) x[i] = x0 + i >= 0 && x0 + i < V ? (float)base[x0 + i] : -INFINITY;
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

struct Best {
  float top;
  int at;
};
__device__ __forceinline__ Best better(const Best& a, const Best& b) {
  return b.top > a.top || (b.top == a.top && b.at < a.at) ? b : a;
}

}  // namespace

template <typename T, bool GREEDY>
__global__ __launch_bounds__(kVerifyThreads) void verify_rows_kernel(VerifyLaunch p) {
  using Row = LogitRow<T>;
  constexpr int VE = Row::VE;
  const int tid = threadIdx.x;
  const int row = blockIdx.x / p.slices, slice = blockIdx.x - row * p.slices;
  const int b = row / p.S, r = row - b * p.S;
  if (blockIdx.x == 0) {
    for (int i = tid; i < p.B; i += kVerifyThreads) p.arrived[i] = 0;
    if (tid == 0) *p.status = 0;
  }
  const Row z((const T*)p.logits + b * p.lss + r * p.lsr, p.V);
  float x[kVerifyVecs][VE];
#pragma unroll
  for (int i = 0; i < kVerifyVecs; ++i) {
    const int v = slice * kSliceVecs + i * kVerifyThreads + tid;
    if (v < z.pieces) {
      z.load(v, x[i]);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[i][e] = -INFINITY;
    }
  }
  RowPart* part = p.parts + blockIdx.x;
  if constexpr (GREEDY) {
    Best best{-INFINITY, INT32_MAX};
#pragma unroll
    for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (x[i][e] > best.top)  // (never a NaN; pieces in ascending order)
          best = Best{x[i][e], (slice * kSliceVecs + i * kVerifyThreads + tid) * VE - z.off + e};
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = better(best, Best{__shfl_xor(best.top, o), __shfl_xor(best.at, o)});
    __shared__ Best red[kVerifyThreads / 64];
    if ((tid & 63) == 0) red[tid >> 6] = best;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < kVerifyThreads / 64; ++i) best = better(best, red[i]);
      *part = RowPart{best.top, best.at, 0.0};
    }
  } else {
    __shared__ float redf[kVerifyThreads / 64];
    __shared__ double redd[kVerifyThreads / 64];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) top = fmaxf(top, x[i][e]);
    top = block_all(top, redf, [](float a, float c) { return fmaxf(a, c); });
    const float ref = top == -INFINITY ? 0.0f : top;  // (a slice of -inf: its sum is 0)
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kVerifyVecs; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) sum += (double)expo(x[i][e], ref, p.k);
    sum = block_all(sum, redd, [](double a, double c) { return a + c; });
    if (tid == 0) *part = RowPart{top, 0, sum};
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
  __shared__ float top[kMaxVerifyRows];      // of a row
  __shared__ double total[kMaxVerifyRows];   // ... its sum of exponentials (NaN: not to be used)
  __shared__ int16_t parent[kMaxVerifyRows]; // -1: not tested
  __shared__ int32_t token[kMaxVerifyRows];  // of a row; greedy: ...
  __shared__ int32_t best[GREEDY ? kMaxVerifyRows : 1];  // the row's own choice (-1: none)
  __shared__ float weight[kMaxVerifyRows];   // exponential of the row's token at its parent
  __shared__ float chance[kMaxVerifyRows];   // its draft probability there
  __shared__ uint8_t taken[kMaxVerifyRows];  // the row is accepted
  __shared__ int16_t gone[kMaxVerifyRows];   // rejected children of the current row
  __shared__ double redd[kVerifyThreads / 64];
  __shared__ int redi[kVerifyThreads / 64];
  __shared__ float uniform[kMaxVerifyRows];  // its number
  __shared__ int at_row, at_next, num_gone, num_path;
  __shared__ double mult, left;              // C; N, what is left of the weights (greedy: not used)

  const T* const logits = (const T*)p.logits + b * p.lss;
  const float* const draft = p.draft ? p.draft + b * p.qss : nullptr;
  for (int r = tid; r < S; r += kVerifyThreads) {
    const RowPart* parts = p.parts + ((int64_t)b * S + r) * p.slices;
    float t = -INFINITY;
    for (int i = 0; i < p.slices; ++i) t = fmaxf(t, parts[i].top);
    if constexpr (GREEDY) {
      int a = -1;
      for (int i = p.slices - 1; i >= 0; --i)
        if (parts[i].top == t && t > -INFINITY) a = parts[i].at;
      best[r] = a;
    } else {
      double s = 0.0;
      for (int i = 0; i < p.slices; ++i)
        if (parts[i].sum != 0.0) s += parts[i].sum * (double)expo(parts[i].top, t, p.k);
      total[r] = t > -INFINITY ? s : __builtin_nan("");
    }
    top[r] = t;
    const int up = r == 0 ? -1 : p.parents ? p.parents[(int64_t)b * S + r] : r - 1;
    const int x = r == 0 ? -1 : p.tokens[(int64_t)b * S + r];
    parent[r] = (int16_t)(up >= 0 && up < r && (uint32_t)x < (uint32_t)p.V ? up : -1);
    token[r] = x;
    taken[r] = r == 0;
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
    for (int r = tid; r < S; r += kVerifyThreads) {
      const int up = parent[r];
      uniform[r] = p.uniform[(int64_t)b * S + r];
      if (up < 0) continue;
      weight[r] = expo((float)logits[up * p.lsr + token[r]], top[up], p.k);
      chance[r] = draft ? draft[up * p.qsr + token[r]] : 0.0f;
    }
    if (tid == 0) left = total[0];
    __syncthreads();
  }
  // One sweep over the rows in order meets every child of an accepted row after it.
  for (;;) {
    if (tid < 64) {
      // (every lane has the same values, and stores them)
      int row = at_row, n_gone = num_gone, n_path = num_path, r = at_next;
      double c = mult, n = GREEDY ? 0.0 : left;
      bool stale = false, stop = false;  // N is not that of the weights
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
              accept = u * q * n < rest(e, c, q);
              if (!accept) {
                c += n;
                stale = true;
              }
            } else {
              bool again = false;  // the token of a sibling already rejected
              for (int y = lane; y < n_gone; y += 64) again |= token[gone[y]] == token[r];
              again = __ballot(again) != 0;
              accept = !again && u * n < e;
              if (!accept && !again) {
                gone[n_gone++] = (int16_t)r;
                n = rest(n, 1.0, e);
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
            if (!GREEDY) n = total[row];
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
    // N = sum of max(e - C q, 0) over the current row, by the whole workgroup
    if constexpr (!GREEDY) {
      const int row = at_row;
      const double c = mult;
      const Row z(logits + row * p.lsr, p.V);
      const float* q = draft + row * p.qsr;
      double sum = 0.0;
      for (int v = tid; v < z.pieces; v += kVerifyThreads) {
        float x[VE];
        z.load(v, x);
        const int x0 = v * VE - z.off;
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (x0 + e >= 0 && x0 + e < p.V) sum += rest((double)expo(x[e], top[row], p.k), c, (double)q[x0 + e]);
      }
      sum = block_all(sum, redd, [](double a, double d) { return a + d; });
      if (tid == 0) left = sum;
    }
    __syncthreads();
  }
  const int row = at_row;
  if (slice == 0) {
    // the accepted rows in order: ascending, as each comes after its parent
    for (int r = tid; r < S; r += kVerifyThreads) {
      int before = 0;
      if (taken[r])
        for (int y = 0; y < r; ++y) before += taken[y];
      if (taken[r]) p.path[(int64_t)b * S + before] = r;
      if (r >= num_path) p.path[(int64_t)b * S + r] = -1;
      if (p.row_weight) p.row_weight[(int64_t)b * S + r] = taken[r] ? 1.0f : 0.0f;
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
    const int n_gone = num_gone;
    // Weights of a piece. The rejected tokens of a plain row are compared with its range.
    auto weights = [&](int v, double mul, double (&w)[VE]) {
      float x[VE];
      z.load(v, x);
      const int x0 = v * VE - z.off;
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        w[e] = (double)expo(x[e], t, p.k);
        if (mul != 0.0 && x0 + e >= 0 && x0 + e < p.V) w[e] = rest(w[e], mul, (double)q[x0 + e]);
      }
      for (int y = 0; y < n_gone; ++y) {
        const int i = token[gone[y]] - x0;
#pragma unroll
        for (int e = 0; e < VE; ++e) w[e] = i == e ? 0.0 : w[e];
      }
    };
    auto slice_sum = [&](int s, double mul) {
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < kVerifyVecs; ++i) {
        const int v = s * kSliceVecs + i * kVerifyThreads + tid;
        if (v < z.pieces) {
          double w[VE];
          weights(v, mul, w);
#pragma unroll
          for (int e = 0; e < VE; ++e) sum += w[e];
        }
      }
      return block_all(sum, redd, [](double a, double d) { return a + d; });
    };
    __shared__ int last;
    double* mass = p.mass + (int64_t)b * slices;
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
    double mul = c, all = 0.0;
    for (int s = 0; s < slices; ++s) all += load_mass(s);
    if (all == 0.0 && c > 0.0) {  // rounding left nothing: the row's own weights
      mul = 0.0;
      __syncthreads();
      for (int s = 0; s < slices; ++s) {
        const double m = slice_sum(s, mul);
        if (tid == 0) __hip_atomic_store(&mass[s], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      __threadfence();
      all = 0.0;
      for (int s = 0; s < slices; ++s) all += load_mass(s);
    }
    if (!(all > 0.0) || !(all < INFINITY)) {  // not a row to draw from
      if (tid == 0) {
        p.next[b] = -1;
        atomicOr(p.status, (uint32_t)JACAP_FLAG_NONFINITE);
      }
      return;
    }
    const double goal = (double)p.uniform[(int64_t)b * S] * all;
    // The slice in which the running sum passes the goal (else the last of positive sum).
    int in = -1;
    double before = 0.0, run = 0.0;
    for (int s = 0; s < slices; ++s) {
      const double m = load_mass(s);
      if (!(m > 0.0)) continue;
      in = s;
      before = run;
      run += m;
      if (run > goal) break;
    }
    // Its pieces, kVerifyVecs in order to a thread.
    double sum = 0.0;
    int final = -1;  // the last token of positive weight
    const int v0 = in * kSliceVecs + tid * kVerifyVecs;
    for (int i = 0; i < kVerifyVecs && v0 + i < z.pieces; ++i) {
      double w[VE];
      weights(v0 + i, mul, w);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        sum += w[e];
        if (w[e] > 0.0) final = (v0 + i) * VE - z.off + e;
      }
    }
    double incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(incl, o);
      if (lane >= o) incl += y;
    }
    __syncthreads();
    if (lane == 63) redd[tid >> 6] = incl;
    __syncthreads();
    for (int i = 0; i < tid >> 6; ++i) before += redd[i];
    int found = INT32_MAX;
    double mass_to = before + (incl - sum);
    if (before + incl > goal) {
      for (int i = 0; i < kVerifyVecs && v0 + i < z.pieces && found == INT32_MAX; ++i) {
        double w[VE];
        weights(v0 + i, mul, w);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          mass_to += w[e];
          if (w[e] > 0.0 && mass_to > goal && found == INT32_MAX) found = (v0 + i) * VE - z.off + e;
        }
      }
    }
    found = block_all(found, redi, [](int a, int d) { return min(a, d); });
    __syncthreads();
    final = block_all(final, redi, [](int a, int d) { return max(a, d); });
    if (tid == 0) p.next[b] = found != INT32_MAX ? found : final;
  }
}

template <typename T>
static void rows_typed(const VerifyLaunch& A) {
  const unsigned grid = (unsigned)((int64_t)A.B * A.S * A.slices);
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
