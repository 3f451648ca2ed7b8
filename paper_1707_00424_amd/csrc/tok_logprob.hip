// Log probabilities of given tokens, entropy and the most likely classes of rows of logits; the logits' gradient.
//
// Forward: one pass over a row with the running maximum m and, relative to it, z = sum e^(x-m) and t = sum (x-m) e^(x-m):
//   lse = m + log z,   entropy = log z - t / z,   logp = (x[label] - m) - log z.
// Odd numbers of classes put rows anywhere; vectors are taken at 16-byte boundaries of memory, whatever the row's.  A row belongs to one
// workgroup, or to several that each take a part of the classes where rows are few; a second, small kernel joins parts.
//
// 4096 rows of 50001 bf16 with 5 alternatives: 94 us, 4.4 TB/s; reading alone would take 58, and the vector unit's work 53 (per element an
// exponential at a quarter of its rate, 21 us together, and six instructions beside it): the two overlap in part.  Four rows of 128000 with 20: 7.7 + 4.8 us, latency.  The gradient, a pass that reads and
// writes: 6144 rows of 32000 in 139 us, 5.6 TB/s.
//
// Alternatives.  Every thread notes the largest value of its vectors and which vector holds it.  The `top`-th best of those
// (value, vector) pairs over 64 groups of four threads is a bound: `top` elements at least are as good, so an element below it is none
// of the best.  Only threads whose own best reaches the bound, about `top` of them, read their part again; vectors that reach the bound
// go to a list in LDS, their elements that do to another, out of which the best are taken by counting.  A list that overflows, where
// few threads hold very many of the best, is given up for `top` searches over the whole part.  (The code is kept short on purpose, as a
// workgroup runs through it once: with 53 KiB of it the 4096 rows took 137 us, with 13 KiB 96.)
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "tok.h"

namespace {

using namespace tok;

constexpr int kThreads = 256, kWaves = kThreads / PARLE_WAVE;
constexpr int kList = 1024, kVectors = 512;  // candidates, and vectors that hold any
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kNear = 1e6f, kFloor = -kNear;
constexpr int kGroup = kThreads * kVec;  // classes of one vector per thread

// Order of floats as unsigned integers; -0 counts as 0, so that equal values have equal keys.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// (value, index) as one number, larger is better: equal values by the lower index.
__device__ __forceinline__ uint64_t pair_of(uint32_t order, uint32_t index) { return (uint64_t)order << 32 | (0xffffffffu - index); }
__device__ __forceinline__ uint32_t index_of(uint64_t pair) { return 0xffffffffu - (uint32_t)pair; }

// The hardware's power of two: 0 below 2^-126, next to a sum of at least 1.
__device__ __forceinline__ float exp2_of(float d) { return __builtin_amdgcn_exp2f(d); }
__device__ __forceinline__ float exp_of(float d) { return exp2_of(d * kLog2e); }

// Statistics of a set of values: the largest, and relative to it z = sum e^(x-m), t = sum (x-m) e^(x-m).
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
    if (most == -INFINITY) return;  // nothing in either
    raise(most), o.raise(most);
    z += o.z, t += o.t;
  }
};

// The same while a thread reads its values, in base 2: an element costs one multiply-add, v log2 e - m2, in front of the
// exponential.  m2 is m log2 e rounded; what the rounding took is put back once, at the end.  It is an exponent's error until then, 2^-4 at
// kNear and 2^9 at 1e10, so this holds for maxima between kFloor and kNear.  m starts at kFloor rather than -inf, so that no difference of
// infinities arises either: values below it count as nothing.  A part whose largest value lies outside is summed again by slow_stats, whatever
// came out here; inside, a thread that holds only values below kFloor adds e^-(10^6), nothing, to those of the others.
struct Running {
  float m = kFloor, m2 = kFloor * kLog2e, z = 0.f, t = 0.f;
  __device__ __forceinline__ void raise(float to) {
    const float to2 = to * kLog2e, d = m2 - to2, f = exp2_of(d);
    t = f > 0.f ? (t + z * d) * f : 0.f;
    z *= f;
    m = to, m2 = to2;
  }
  __device__ __forceinline__ void add(float v) {
    const float d = __builtin_fmaf(v, kLog2e, -m2), e = exp2_of(d);
    z += e;
    t = __builtin_fmaf(e, fmaxf(d, kFloor), t);  // 0 where e is; a NaN comes along in e
  }
  __device__ __forceinline__ Stats result() const {
    Stats s;
    const float r = __builtin_fmaf(m, kLog2e, -m2), f = exp2_of(-r);
    s.m = m, s.z = z * f, s.t = (t - z * r) * f * kLn2;
    return s;
  }
};

__device__ __forceinline__ Stats wave_join(Stats s) {
  const float most = wave_max_all(s.m);
  if (most > s.m) s.raise(most);
  s.z = wave_sum_all(s.z), s.t = wave_sum_all(s.t);
  return s;
}
// The best of the pairs of four neighbouring lanes.
__device__ __forceinline__ uint64_t best_of_four(uint64_t v) {
  const uint64_t a = (uint64_t)from_lane<kLaneXor1>((uint32_t)(v >> 32)) << 32 | from_lane<kLaneXor1>((uint32_t)v);
  v = a > v ? a : v;
  const uint64_t b = (uint64_t)from_lane<kLaneXor2>((uint32_t)(v >> 32)) << 32 | from_lane<kLaneXor2>((uint32_t)v);
  return b > v ? b : v;
}
__device__ __forceinline__ uint64_t wave_best(uint64_t v) {
#pragma unroll
  for (int o = PARLE_WAVE / 2; o > 0; o >>= 1) {
    const uint64_t u = __shfl_xor((unsigned long long)v, o, PARLE_WAVE);
    v = u > v ? u : v;
  }
  return v;
}

struct Part {  // of one workgroup, where several share a row
  float m, z, t, pad;
};
__device__ __forceinline__ Part part_of(const Stats &s) { return Part{s.m, s.z, s.t, 0.f}; }
__device__ __forceinline__ Stats stats_of(const Part &p) {
  Stats s;
  s.m = p.m, s.z = p.z, s.t = p.t;
  return s;
}

struct FwdArgs {
  const int32_t *labels;
  float *logp, *entropy, *lse;
  int32_t *top_ids;
  float *top_logp;
  Part *parts;      // [rows][splits]
  uint64_t *best;   // [rows][splits][top], in order
  long long ld, rows;
  int C, top, splits, span;  // span: classes of a part, a multiple of kGroup
};

struct Lds {
  Part part[kWaves];
  uint64_t best[kThreads];
  uint64_t bound;
  uint64_t list[kList];
  int vector[kVectors];
  int count, vectors;
};

// A row as vectors of eight elements from a boundary of 16 bytes on: its class 0 lies `off` elements behind the boundary that `base`
// points to, and vector j holds elements j .. j + 7 of base, of which the row's are off .. end - 1.
template <typename T>
struct Row {
  const T *base;
  int off, end;
  __device__ __forceinline__ Row(const T *x, int C) {
    off = (int)((uintptr_t)x % 16 / sizeof(T));
    base = x - off;
    end = off + C;
  }
};
struct RawBf16 {
  us8 v;
  __device__ __forceinline__ float at(int i) const { return bf16_to_f32(v[i]); }
  __device__ __forceinline__ void clear(int i) { v[i] = 0xff80; }
};
struct RawF32 {
  f4 a, b;
  __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  __device__ __forceinline__ void clear(int i) {
    if (i < 4)
      a[i] = -INFINITY;
    else
      b[i - 4] = -INFINITY;
  }
};
// 16 bytes that hold an element of the row are read whole, no others; `left`: elements from p to the row's end.
__device__ __forceinline__ void read(const bf16_t *p, int left, RawBf16 &x) { x.v = *(const us8 *)p; }
__device__ __forceinline__ void read(const float *p, int left, RawF32 &x) {
  x.a = *(const f4 *)p;
  x.b = left > 4 ? *(const f4 *)(p + 4) : f4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
}
template <typename T>
using Raw = std::conditional_t<sizeof(T) == 2, RawBf16, RawF32>;
// Vector j < end; -inf in the places of elements that are not the row's.
template <typename T>
__device__ __forceinline__ Raw<T> fetch(const Row<T> &r, int j, bool live) {
  Raw<T> x;
  if (live) {
    read(r.base + j, r.end - j, x);
    if (j < r.off || j + kVec > r.end) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (j + i < r.off || j + i >= r.end) x.clear(i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) x.clear(i);
  }
  return x;
}
template <typename R>
__device__ __forceinline__ float most_of(const R &x) {
  float m = x.at(0);
#pragma unroll
  for (int i = 1; i < kVec; ++i) m = fmaxf(m, x.at(i));
  return m;
}
__device__ __forceinline__ float logit_at(const bf16_t *x, int i) { return bf16_to_f32(x[i]); }
__device__ __forceinline__ float logit_at(const float *x, int i) { return x[i]; }

// Statistics of a part whose largest value m is far from zero: differences are taken before they are scaled.  For elements j0 .. j1 - 1.
template <typename T>
__device__ __forceinline__ Stats slow_stats(const Row<T> &row, int j0, int j1, float m) {
  constexpr int kAhead = 2;
  Stats s;
  s.m = m;
#pragma unroll 1
  for (int j = j0 + threadIdx.x * kVec; j < j1; j += kAhead * kGroup) {
    Raw<T> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) raw[u] = fetch(row, j + u * kGroup, j + u * kGroup < j1);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float d = raw[u].at(i) - m, e = exp_of(d);
        s.z += e;
        s.t += e * fmaxf(d, kFloor);
      }
  }
  return s;
}

// put(place, pair) for the `top` best of the `count` pairs in lds.list; 0 in the places of those that are missing.  Four neighbouring
// threads count what is better than a pair, a quarter of the list each.
template <typename Put>
__device__ __forceinline__ void take_best(const Lds &lds, int count, int top, const Put &put) {
  for (int i = threadIdx.x; i < top; i += kThreads)
    if (i >= count) put(i, 0);
#pragma unroll 1
  for (int i = threadIdx.x >> 2; i < count; i += kThreads / 4) {
    const uint64_t me = lds.list[i];
    uint32_t better = 0;
#pragma unroll 8
    for (int j = threadIdx.x & 3; j < count; j += 4) better += lds.list[j] > me;
    better += from_lane<kLaneXor1>(better);
    better += from_lane<kLaneXor2>(better);
    if ((threadIdx.x & 3) == 0 && (int)better < top) put(better, me);
  }
}

// The pair of 64 (lds.best[0], [stride], ...) that has top - 1 better ones there, 0 where there are fewer; for every wavefront by itself.
__device__ __forceinline__ uint64_t find_bound(const Lds &lds, int stride, int top) {
  const int lane = threadIdx.x & (PARLE_WAVE - 1);
  const uint64_t mine = lds.best[lane * stride];
  int better = 0;
#pragma unroll 16
  for (int j = 0; j < PARLE_WAVE; ++j) better += lds.best[j * stride] > mine;
  const uint64_t found = __ballot(better == top - 1 && mine);
  if (found == 0) return 0;
  const int at = __builtin_ctzll(found);
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(mine >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)mine, at);
}
// The same over the 256 pairs of lds.best, for every thread's own one `mine`; a barrier.
__device__ __forceinline__ uint64_t find_bound_of_all(Lds &lds, uint64_t mine, int top) {
  int better = 0;
#pragma unroll 16
  for (int j = 0; j < kThreads; ++j) better += lds.best[j] > mine;
  if (better == top - 1 && mine) lds.bound = mine;
  __syncthreads();
  return lds.bound;
}

// The results of a row from its joined statistics.
struct RowOut {
  const FwdArgs &a;
  long long row;
  float m, lz;
  __device__ __forceinline__ RowOut(const FwdArgs &args, long long at, const Stats &s) : a(args), row(at), m(s.m), lz(logf(s.z)) {}
  __device__ __forceinline__ void stats(const Stats &s, int label, float label_value) const {
    if (threadIdx.x != 0) return;
    if (a.lse) a.lse[row] = m > -INFINITY ? m + lz : -INFINITY;
    if (a.entropy) a.entropy[row] = m > -INFINITY ? lz - s.t / s.z : 0.f;
    if (a.logp) a.logp[row] = label < 0 || label >= a.C ? 0.f : m > -INFINITY ? (label_value - m) - lz : -INFINITY;
  }
  __device__ __forceinline__ void operator()(int i, uint64_t p) const {
    a.top_ids[row * a.top + i] = p ? (int)index_of(p) : -1;
    a.top_logp[row * a.top + i] = p ? (value_of((uint32_t)(p >> 32)) - m) - lz : -INFINITY;
  }
};

// Joins the wavefronts' statistics for everyone; one barrier.
__device__ __forceinline__ Stats block_join(Lds &lds, Stats s) {
  s = wave_join(s);
  if ((threadIdx.x & (PARLE_WAVE - 1)) == 0) lds.part[threadIdx.x / PARLE_WAVE] = part_of(s);
  __syncthreads();
  s = stats_of(lds.part[0]);
#pragma unroll
  for (int w = 1; w < kWaves; ++w) s.join(stats_of(lds.part[w]));
  return s;
}

// The best of classes c0 .. c1 - 1 by `top` searches: put(0), put(1), ...
template <typename T, typename Put>
__device__ __forceinline__ void search_best(Lds &lds, const T *x, int c0, int c1, int top, const Put &put) {
  uint64_t last = ~0ull;
#pragma unroll 1
  for (int n = 0; n < top; ++n) {
    uint64_t b = 0;
#pragma unroll 1
    for (int c = c0 + threadIdx.x; c < c1; c += kThreads) {
      const float v = logit_at(x, c);
      const uint64_t p = v > -INFINITY ? pair_of(order_of(v), c) : 0;
      if (p < last && p > b) b = p;
    }
    b = wave_best(b);
    __syncthreads();
    if ((threadIdx.x & (PARLE_WAVE - 1)) == 0) lds.best[threadIdx.x / PARLE_WAVE] = b;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) b = lds.best[w] > b ? lds.best[w] : b;
    if (threadIdx.x == 0) put(n, b);
    last = b;
  }
}

// grid: (splits, rows)
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_logprob_fwd(const T *logits, FwdArgs a) {
  constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;  // vectors in flight per thread
  __shared__ Lds lds;
  const long long row_at = blockIdx.y + (long long)gridDim.y * blockIdx.z;
  if (row_at >= a.rows) return;
  const T *x = logits + row_at * a.ld;
  const Row<T> row(x, a.C);
  const int j0 = blockIdx.x * a.span, j1 = min(j0 + a.span, row.end);
  const int lane = threadIdx.x & (PARLE_WAVE - 1);
  Running run;
  float most = -INFINITY;  // this thread's largest, and the vector that holds it first
  int at = 0;
  for (int j = j0; j < j1; j += kAhead * kGroup) {
    const int mine = j + threadIdx.x * kVec;
    Raw<T> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) raw[u] = fetch(row, mine + u * kGroup, mine + u * kGroup < j1);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const float vm = most_of(raw[u]);
      if (vm > most) most = vm, at = mine + u * kGroup;
    }
    if (most > run.m) run.raise(most);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (u > 0 && j + u * kGroup >= j1) break;  // the same for all threads
#pragma unroll
      for (int i = 0; i < kVec; ++i) run.add(raw[u].at(i));
    }
  }
  const uint64_t mine = most > -INFINITY ? pair_of(order_of(most), at) : 0;
  if (TOP) {
    const uint64_t four = best_of_four(mine);
    if ((lane & 3) == 0) lds.best[threadIdx.x] = four;
    if (threadIdx.x == 0) lds.count = lds.vectors = 0, lds.bound = 0;
  }
  Stats s = block_join(lds, run.result());
  const int c0 = max(j0 - row.off, 0), c1 = j1 - row.off;  // the part's classes
  if (!(s.m > kFloor && s.m <= kNear)) {  // s.m is the part's largest value, or kFloor: the same for all threads
    const float w = wave_max_all(most);
    __syncthreads();
    if (lane == 0) lds.part[threadIdx.x / PARLE_WAVE].pad = w;
    __syncthreads();
    float all = lds.part[0].pad;
#pragma unroll
    for (int w2 = 1; w2 < kWaves; ++w2) all = fmaxf(all, lds.part[w2].pad);
    __syncthreads();
    if (all > -INFINITY)
      s = block_join(lds, slow_stats(row, j0, j1, all));
    else if (s.z == 0.f)
      s = Stats();  // nothing there; a NaN beside nothing stays
  }
  const int label = a.logp && a.splits == 1 ? a.labels[row_at] : -1;
  const long long slot = row_at * a.splits + blockIdx.x;
  RowOut out(a, row_at, s);
  if (a.splits == 1)
    out.stats(s, label, label >= 0 && label < a.C ? logit_at(x, label) : 0.f);
  else if (threadIdx.x == 0)
    a.parts[slot] = part_of(s);
  if (!TOP) return;
  const auto put = [&](int i, uint64_t p) {
    if (a.splits == 1)
      out(i, p);
    else
      a.best[slot * a.top + i] = p;
  };
  uint64_t bound = find_bound(lds, 4, a.top);
  if (bound == 0 && a.top > 1) {  // fewer groups than that hold anything, as behind a mask: over all threads
    __syncthreads();
    lds.best[threadIdx.x] = mine;
    __syncthreads();
    bound = find_bound_of_all(lds, mine, a.top);
  }
  // vectors that reach the bound, by the threads that know of one
  if (mine && mine >= bound) {
    for (int j = j0 + threadIdx.x * kVec; j < j1; j += kAhead * kGroup) {
      Raw<T> raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) raw[u] = fetch(row, j + u * kGroup, j + u * kGroup < j1);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const float vm = most_of(raw[u]);
        if (vm > -INFINITY && pair_of(order_of(vm), j + u * kGroup) >= bound) {
          const int n = atomicAdd(&lds.vectors, 1);
          if (n < kVectors) lds.vector[n] = j + u * kGroup;
        }
      }
    }
  }
  __syncthreads();
  // their elements that do
  const int vectors = lds.vectors;
  const uint32_t b_order = (uint32_t)(bound >> 32), b_at = index_of(bound);
  for (int e = threadIdx.x; e < min(vectors, kVectors) * kVec; e += kThreads) {
    const int j = lds.vector[e / kVec], c = j + e % kVec - row.off;
    if (c < 0 || c >= a.C) continue;
    const float v = logit_at(x, c);
    const uint32_t k = order_of(v);
    if (v > -INFINITY && (k > b_order || (k == b_order && (uint32_t)j <= b_at))) {
      const int n = atomicAdd(&lds.count, 1);
      if (n < kList) lds.list[n] = pair_of(k, c);
    }
  }
  __syncthreads();
  const int count = lds.count;
  if (vectors <= kVectors && count <= kList)
    take_best(lds, count, a.top, put);
  else
    search_best(lds, x, c0, c1, a.top, put);
}

// Joins the parts of a row.  Their lists are in order: a list whose pair `depth` reaches a bound has depth + 1 pairs that do, so the
// ceil(top / (depth + 1))-th best of the lists' pairs at that depth bounds what can be among the best.  (depth: about half of the lists
// are to reach it.)
template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprob_join(const T *logits, FwdArgs a) {
  __shared__ Lds lds;
  __shared__ uint64_t best[PARLE_LOGPROB_MAX_TOP];
  const long long row = blockIdx.x;
  const int label = a.logp ? a.labels[row] : -1;
  const float label_value = label >= 0 && label < a.C ? logit_at(logits + row * a.ld, label) : 0.f;
  // a thread's pairs, all at once (the first kHeld of them)
  constexpr int kHeld = 8;
  const uint64_t *from = a.best + row * a.splits * a.top;
  const int all = a.splits * a.top;
  uint64_t mine[kHeld];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) mine[u] = (int)threadIdx.x + u * kThreads < all ? from[threadIdx.x + u * kThreads] : 0;
  const int lists = min(a.splits, PARLE_WAVE), depth = a.top > 0 ? (a.top - 1) / max(1, lists / 2) : 0;
  if (threadIdx.x < PARLE_WAVE) lds.best[threadIdx.x] = a.top > 0 && (int)threadIdx.x < lists ? from[threadIdx.x * a.top + depth] : 0;
  if (threadIdx.x == 0) lds.count = 0;
  Stats s;
  for (int i = threadIdx.x; i < a.splits; i += kThreads) s.join(stats_of(a.parts[row * a.splits + i]));
  s = block_join(lds, s);
  const RowOut out(a, row, s);
  out.stats(s, label, label_value);
  if (a.top == 0) return;
  const uint64_t bound = find_bound(lds, 1, a.top / (depth + 1) + (a.top % (depth + 1) != 0));
  const auto keep = [&](uint64_t p) {
    if (p && p >= bound) {
      const int slot = atomicAdd(&lds.count, 1);
      if (slot < kList) lds.list[slot] = p;
    }
  };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) keep(mine[u]);
  for (int i = threadIdx.x + kHeld * kThreads; i < all; i += kThreads) keep(from[i]);
  __syncthreads();
  const int count = lds.count;
  if (count <= kList) {
    take_best(lds, count, a.top, out);
    return;
  }
  // too many: kList at a time, the best so far at the list's front
  const int room = kList - a.top;
  int held = 0;
  for (int i0 = 0; i0 < all; i0 += room) {
    const int more = min(room, all - i0);
    __syncthreads();
    if (threadIdx.x == 0) lds.count = held;
    __syncthreads();
    for (int i = threadIdx.x; i < held; i += kThreads) lds.list[i] = best[i];
    for (int i = threadIdx.x; i < more; i += kThreads) {
      const uint64_t p = from[i0 + i];
      if (p) lds.list[atomicAdd(&lds.count, 1)] = p;
    }
    __syncthreads();
    const int n = lds.count;
    take_best(lds, n, a.top, [&](int i, uint64_t p) { best[i] = p; });
    __syncthreads();
    held = min(n, a.top);
  }
  for (int i = threadIdx.x; i < a.top; i += kThreads) out(i, best[i]);
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
  const int groups = ceil_div(d.classes + kVec - 1, kGroup);  // a row may begin inside its first vector
  // A row to a workgroup where rows fill the chip.  Fewer are split into parts of two vectors per thread at least: four rows of 128000
  // classes with 20 alternatives take 7.2 + 5.7 us in 63 parts of one vector and 7.3 + 5.5 in 32 of two, but a part that a mask
  // leaves a few hundred classes of finds its bound among too few threads, and takes 11 us for 8.
  const int want = rows >= 512 || rows == 0 ? 1 : ceil_div(1024, rows);
  const int each = std::max(ceil_div(groups, want), want > 1 ? 2 : 1);
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
