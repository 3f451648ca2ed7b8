// Log probabilities of given tokens, entropy and the most likely classes of rows of logits; the logits' gradient.
//
// Forward: one pass over a row with the running maximum m and, relative to it, z = sum e^(x-m) and t = sum (x-m) e^(x-m):
//   lse = m + log z,   entropy = log z - t / z,   logp = (x[label] - m) - log z.
// A row belongs to one workgroup, or to several that each take a part of the classes where rows are few; a second, small kernel
// joins parts.
//
// Alternatives.  Every thread notes the largest value of its vectors and which vector holds it.  The `top`-th best of those
// (value, vector) pairs over the threads is a bound: `top` elements at least are as good, so an element below it is none of the
// best.  Only threads whose own best reaches the bound, about `top` of them, read their part again; what reaches the bound
// goes to a list in LDS, out of which the best are taken by counting.  A list that overflows, where one thread holds
// very many of the best, is given up for `top` searches over the whole part.
#include <math.h>

#include <algorithm>

#include "tok.h"

namespace {

using namespace tok;

constexpr int kThreads = 256, kWaves = kThreads / PARLE_WAVE;
constexpr int kList = 1024;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kGroup = kThreads * kVec;  // classes that a workgroup takes at a time

// Order of floats as unsigned integers; -0 counts as 0, so that equal values have equal keys.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// (value, index) as one number, larger is better: equal values by the lower index.
__device__ __forceinline__ uint64_t pair_of(uint32_t order, uint32_t index) { return (uint64_t)order << 32 | (0xffffffffu - index); }
__device__ __forceinline__ uint32_t index_of(uint64_t pair) { return 0xffffffffu - (uint32_t)pair; }

// e^d for d <= 0: the hardware's power of two, 0 below 2^-126, next to a sum of at least 1.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Running statistics of a set of values.  The difference x - m is taken before it is scaled to base 2: it is exact where it
// counts, and a mask of the type's lowest value stays finite.
struct Stats {
  float m = -INFINITY, z = 0.f, t = 0.f;
  // Sums relative to a maximum that is now `to` >= m.
  __device__ __forceinline__ void raise(float to) {
    const float d = m - to, f = m > -INFINITY ? exp_of(d) : 0.f;
    t = f > 0.f ? (t + z * d) * f : 0.f;
    z *= f;
    m = to;
  }
  __device__ __forceinline__ void join(Stats o) {
    const float most = fmaxf(m, o.m);
    if (most == -INFINITY) {  // nothing in either, or NaN
      z += o.z, t += o.t;
      return;
    }
    raise(most), o.raise(most);
    z += o.z, t += o.t;
  }
};

__device__ __forceinline__ Stats wave_join(Stats s) {
#pragma unroll
  for (int o = 1; o < PARLE_WAVE; o <<= 1) {
    Stats u;
    u.m = __shfl_xor(s.m, o, PARLE_WAVE), u.z = __shfl_xor(s.z, o, PARLE_WAVE), u.t = __shfl_xor(s.t, o, PARLE_WAVE);
    s.join(u);
  }
  return s;
}

struct Part {  // of one workgroup, where several share a row
  float m, z, t, pad;
};

struct FwdArgs {
  const int32_t *labels;
  float *logp, *entropy, *lse;
  int32_t *top_ids;
  float *top_logp;
  Part *parts;      // [rows][splits]
  uint64_t *best;   // [rows][splits][top]
  long long ld, rows;
  int C, top, splits, span;  // span: classes of a part, a multiple of kGroup
};

struct Lds {
  Part part[kWaves];
  uint64_t best[kThreads];
  uint64_t list[kList];
  int count;
  uint64_t bound;
};

// The `top` best of the `count` pairs in lds.list, in order, to out[0 .. top); those that are missing are 0.
__device__ __forceinline__ void take_best(Lds &lds, int count, int top, uint64_t *out) {
  for (int i = threadIdx.x; i < top; i += kThreads)
    if (i >= count) out[i] = 0;
  for (int i = threadIdx.x; i < count; i += kThreads) {
    const uint64_t me = lds.list[i];
    int better = 0;
    for (int j = 0; j < count; ++j) better += lds.list[j] > me;
    if (better < top) out[better] = me;
  }
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int o = PARLE_WAVE / 2; o > 0; o >>= 1) {
    const uint64_t u = __shfl_xor((unsigned long long)v, o, PARLE_WAVE);
    v = u > v ? u : v;
  }
  return v;
}

// The results of a row from its joined statistics (natural units) and its best pairs.
__device__ __forceinline__ void finish_row(const FwdArgs &a, long long row, Stats s, float label_value, int label, const uint64_t *best) {
  const float lz = logf(s.z), lse = s.m > -INFINITY ? s.m + lz : s.z != s.z ? s.z : -INFINITY;
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = s.m > -INFINITY ? lz - s.t / s.z : s.z != s.z ? s.z : 0.f;
    if (a.logp) a.logp[row] = label < 0 || label >= a.C ? 0.f : lse == -INFINITY ? -INFINITY : (label_value - s.m) - lz;
  }
  for (int i = threadIdx.x; i < a.top; i += kThreads) {
    const uint64_t p = best[i];
    a.top_ids[row * a.top + i] = p ? (int)index_of(p) : -1;
    a.top_logp[row * a.top + i] = p ? (value_of((uint32_t)(p >> 32)) - s.m) - lz : -INFINITY;
  }
}

// grid: (splits, rows)
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_logprob_fwd(const T *logits, FwdArgs a) {
  __shared__ Lds lds;
  __shared__ uint64_t best[PARLE_LOGPROB_MAX_TOP];
  const long long row = blockIdx.y + (long long)gridDim.y * blockIdx.z;
  if (row >= a.rows) return;
  const T *x = logits + row * a.ld;
  const int c0 = blockIdx.x * a.span, c1 = min(c0 + a.span, a.C);
  Stats s;
  float most = -INFINITY;  // this thread's best, and the vector that holds it first
  int at = 0;
  for (int c = c0 + threadIdx.x * kVec; c < c1; c += kGroup) {
    float v[kVec];
    load8(x + c, c1 - c, -INFINITY, v);
    float vm = v[0];
#pragma unroll
    for (int i = 1; i < kVec; ++i) vm = fmaxf(vm, v[i]);
    if (vm > most) most = vm, at = c;
    if (vm > s.m) s.raise(vm);
    if (s.m > -INFINITY) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float d = v[i] - s.m, e = exp_of(d);
        s.z += e;
        s.t += e * fmaxf(d, -1e30f);  // 0 where e is; a NaN comes along in e
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (v[i] != v[i]) s.z += v[i];
    }
  }
  const uint64_t mine = most > -INFINITY ? pair_of(order_of(most), at) : 0;
  s = wave_join(s);
  const int wave = threadIdx.x / PARLE_WAVE, lane = threadIdx.x & (PARLE_WAVE - 1);
  if (lane == 0) lds.part[wave] = Part{s.m, s.z, s.t, 0.f};
  if (TOP) {
    lds.best[threadIdx.x] = mine;
    if (threadIdx.x == 0) lds.count = 0, lds.bound = 0;
  }
  __syncthreads();
  s.m = lds.part[0].m, s.z = lds.part[0].z, s.t = lds.part[0].t;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    Stats u;
    u.m = lds.part[w].m, u.z = lds.part[w].z, u.t = lds.part[w].t;
    s.join(u);
  }
  if (TOP) {
    // the bound: the pair with top - 1 better ones (0, everything, where there are fewer)
    int better = 0;
    for (int j = 0; j < kThreads; ++j) better += lds.best[j] > mine;
    if (better == a.top - 1 && mine) lds.bound = mine;
    __syncthreads();
    const uint64_t bound = lds.bound;
    const uint32_t b_order = (uint32_t)(bound >> 32), b_at = index_of(bound);
    if (mine && mine >= bound) {
      for (int c = c0 + threadIdx.x * kVec; c < c1; c += kGroup) {
        float v[kVec];
        load8(x + c, c1 - c, -INFINITY, v);
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
          const uint32_t k = order_of(v[i]);
          if (v[i] > -INFINITY && (k > b_order || (k == b_order && (uint32_t)c <= b_at))) {
            const int slot = atomicAdd(&lds.count, 1);
            if (slot < kList) lds.list[slot] = pair_of(k, c + i);
          }
        }
      }
    }
    __syncthreads();
    const int count = lds.count;
    if (count <= kList) {
      take_best(lds, count, a.top, best);
    } else {
      uint64_t last = ~0ull;
      for (int j = 0; j < a.top; ++j) {
        uint64_t b = 0;
        for (int c = c0 + threadIdx.x * kVec; c < c1; c += kGroup) {
          float v[kVec];
          load8(x + c, c1 - c, -INFINITY, v);
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const uint64_t p = v[i] > -INFINITY ? pair_of(order_of(v[i]), c + i) : 0;
            if (p < last && p > b) b = p;
          }
        }
        b = wave_max(b);
        __syncthreads();
        if (lane == 0) lds.best[wave] = b;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) b = lds.best[w] > b ? lds.best[w] : b;
        if (threadIdx.x == 0) best[j] = b;
        last = b;
      }
    }
    __syncthreads();
  }
  if (a.splits == 1) {
    const int label = a.logp ? a.labels[row] : -1;
    float lv = 0.f;
    if (label >= 0 && label < a.C) {
      const T raw = x[label];
      lv = sizeof(T) == 2 ? bf16_to_f32((bf16_t)raw) : (float)raw;
    }
    finish_row(a, row, s, lv, label, best);
  } else {
    const long long slot = row * a.splits + blockIdx.x;
    if (threadIdx.x == 0) a.parts[slot] = Part{s.m, s.z, s.t, 0.f};
    if (TOP && (int)threadIdx.x < a.top) a.best[slot * a.top + threadIdx.x] = best[threadIdx.x];
  }
}

// Joins the parts of a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprob_join(const T *logits, FwdArgs a) {
  __shared__ Lds lds;
  __shared__ uint64_t best[PARLE_LOGPROB_MAX_TOP];
  const long long row = blockIdx.x;
  Stats s;
  for (int i = threadIdx.x; i < a.splits; i += kThreads) {
    const Part p = a.parts[row * a.splits + i];
    Stats u;
    u.m = p.m, u.z = p.z, u.t = p.t;
    s.join(u);
  }
  s = wave_join(s);
  const int wave = threadIdx.x / PARLE_WAVE;
  if ((threadIdx.x & (PARLE_WAVE - 1)) == 0) lds.part[wave] = Part{s.m, s.z, s.t, 0.f};
  __syncthreads();
  s.m = lds.part[0].m, s.z = lds.part[0].z, s.t = lds.part[0].t;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    Stats u;
    u.m = lds.part[w].m, u.z = lds.part[w].z, u.t = lds.part[w].t;
    s.join(u);
  }
  if (a.top > 0) {
    // splits * top pairs, at most kList at a time: the best so far stay at the list's front
    const uint64_t *from = a.best + row * a.splits * a.top;
    const int all = a.splits * a.top, room = kList - a.top;
    int held = 0;
    for (int i0 = 0; i0 < all; i0 += room) {
      const int more = min(room, all - i0);
      if (threadIdx.x == 0) lds.count = held;
      __syncthreads();
      for (int i = threadIdx.x; i < held; i += kThreads) lds.list[i] = best[i];
      for (int i = threadIdx.x; i < more; i += kThreads) {
        const uint64_t p = from[i0 + i];
        if (p) lds.list[atomicAdd(&lds.count, 1)] = p;
      }
      __syncthreads();
      const int count = lds.count;
      take_best(lds, count, a.top, best);
      __syncthreads();
      held = min(count, a.top);
    }
  }
  const int label = a.logp ? a.labels[row] : -1;
  float lv = 0.f;
  if (label >= 0 && label < a.C) {
    const T raw = logits[row * a.ld + label];
    lv = sizeof(T) == 2 ? bf16_to_f32((bf16_t)raw) : (float)raw;
  }
  finish_row(a, row, s, lv, label, best);
}

// d = gl (onehot - p) - dH p (log p + H) with p = e^(x - lse).  grid: (parts of a row, rows)
template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprob_bwd(const T *logits, const int32_t *labels, const float *lse, const float *entropy,
                                                          const float *dlogp, const float *dentropy, T *dlogits, int C, long long ld, long long rows) {
  const long long row = blockIdx.y + (long long)gridDim.y * blockIdx.z;
  const int c = blockIdx.x * kGroup + threadIdx.x * kVec;
  if (c >= C || row >= rows) return;
  float v[kVec], o[kVec];
  load8(logits + row * ld + c, C - c, -INFINITY, v);
  const float l = lse[row];
  const int label = labels[row];
  const float gl = label >= 0 && label < C ? dlogp[row] : 0.f, dh = dentropy ? dentropy[row] : 0.f, h = dentropy ? entropy[row] : 0.f;
  const bool some = l != -INFINITY;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const float lp = v[i] - l, p = exp_of(lp);
    const float inner = gl + (p > 0.f ? dh * (lp + h) : 0.f);
    const float d = (c + i == label ? gl : 0.f) - p * inner;
    o[i] = some ? d : 0.f;
  }
  store8(dlogits + row * ld + c, C - c, o);
}

// Rows may be more than a grid's y dimension takes.
dim3 row_grid(int x, long long rows) {
  const long long y = std::min<long long>(rows, 65535);
  return dim3(x, (unsigned)y, (unsigned)ceil_div(rows, y));
}

struct Plan {
  int splits, span;
  long long parts, best;
};
Plan plan_of(const parle_logprob_desc &d) {
  Plan p;
  const long long rows = (long long)d.n * d.rows;
  const int groups = ceil_div(d.classes, kGroup);
  // A row to a workgroup where rows fill the chip; else parts of one group of classes at least.
  const int want = rows >= 512 || rows == 0 ? 1 : ceil_div(1024, rows);
  const int each = ceil_div(groups, std::min(want, groups));
  p.span = each * kGroup;
  p.splits = ceil_div(groups, each);
  p.parts = p.splits > 1 ? round_up(rows * p.splits * (long long)sizeof(Part), 256) : 0;
  p.best = p.splits > 1 ? rows * p.splits * d.top * 8 : 0;
  return p;
}

template <typename T>
hipError_t fwd(hipStream_t st, const parle_logprob_desc &d, const void *logits, FwdArgs a) {
  const dim3 grid = row_grid(a.splits, a.rows);
  if (d.top)
    k_logprob_fwd<T, true><<<grid, kThreads, 0, st>>>((const T *)logits, a);
  else
    k_logprob_fwd<T, false><<<grid, kThreads, 0, st>>>((const T *)logits, a);
  if (a.splits > 1) k_logprob_join<T><<<dim3((unsigned)a.rows), kThreads, 0, st>>>((const T *)logits, a);
  return hipGetLastError();
}

}  // namespace

int64_t logprob_scratch_bytes(const parle_logprob_desc &d) {
  const Plan p = plan_of(d);
  return p.parts + p.best;
}

hipError_t launch_logprob_fwd(hipStream_t st, const parle_logprob_desc &d, const void *logits, const int32_t *labels, void *scratch,
                              float *logp, float *entropy, float *lse, int32_t *top_ids, float *top_logp) {
  const Plan p = plan_of(d);
  FwdArgs a;
  a.labels = labels, a.logp = logp, a.entropy = entropy, a.lse = lse, a.top_ids = top_ids, a.top_logp = top_logp;
  a.parts = (Part *)scratch, a.best = (uint64_t *)((char *)scratch + p.parts);
  a.ld = d.ld, a.rows = (long long)d.n * d.rows, a.C = d.classes, a.top = d.top, a.splits = p.splits, a.span = p.span;
  return d.dtype ? fwd<bf16_t>(st, d, logits, a) : fwd<float>(st, d, logits, a);
}

hipError_t launch_logprob_bwd(hipStream_t st, const parle_logprob_desc &d, const void *logits, const int32_t *labels, const float *lse,
                              const float *entropy, const float *dlogp, const float *dentropy, void *dlogits) {
  const long long rows = (long long)d.n * d.rows;
  const dim3 grid = row_grid(ceil_div(d.classes, kGroup), rows);
  if (d.dtype)
    k_logprob_bwd<bf16_t><<<grid, kThreads, 0, st>>>((const bf16_t *)logits, labels, lse, entropy, dlogp, dentropy, (bf16_t *)dlogits, d.classes, d.ld, rows);
  else
    k_logprob_bwd<float><<<grid, kThreads, 0, st>>>((const float *)logits, labels, lse, entropy, dlogp, dentropy, (float *)dlogits, d.classes, d.ld, rows);
  return hipGetLastError();
}
