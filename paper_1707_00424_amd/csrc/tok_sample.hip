// A class of every row from a given random number, behind temperature, top-k, top-p and min-p.
//
// In the order of falling logit (the lower class first where two are equal) every rule keeps a beginning, so all are questions of one kind: where does
// the count, or the sum of the weights e^((x - max) / T), reach a number?  Weights are whole multiples of 2^-s of the largest, so sums are
// exact in 64-bit integers, in any order, and the answers the same every time; they are formed in 64 bits, as a number next to a border is on one
// side of it or the other.
// Nothing is sorted but a few: counts and sums over kBuckets steps of the weight's logarithm say in which step an answer lies, the row is read again
// for the classes of that step, and up to kList of those are sorted.  More of them (many equal logits) are counted again in finer steps of value and class.
#include "tok.h"

namespace {

using namespace tok;
typedef unsigned long long u64;

constexpr int kThreads = 1024, kWaves = kThreads / PARLE_WAVE;
constexpr int kBuckets = 2048, kPer = kBuckets / kThreads;
constexpr int kList = kThreads;
constexpr int kIdBits = 22;  // classes <= 2^22

struct Args {
  const void *logits;
  const float *uniform, *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
  int32_t *tokens, *kept;
  float *logp;
  int classes, bits;  // s
  long long ld;
};

// Value and class as one number that ascends in the order of the classes.
__device__ __forceinline__ u64 rank_of(float x, int id) {
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 is 0
  const uint32_t up = u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
  return ((u64)~up << kIdBits) | (uint32_t)id;
}
__device__ __forceinline__ float value_of(u64 rank) {
  const uint32_t up = ~(uint32_t)(rank >> kIdBits);
  return __uint_as_float(up ^ ((up >> 31) ? 0x80000000u : 0xffffffffu));
}

// The weights of a row.
struct Scale {
  double most, per;  // the largest logit; log2(e) / temperature
  int bits;
  // the weight's logarithm, base 2, <= 0
  __device__ __forceinline__ double log_of(float x) const { return (double)x == most ? 0.0 : ((double)x - most) * per; }
  __device__ __forceinline__ u64 units(double t) const {
    if (!(t > -(double)(bits + 1))) return 0;
    const double v = exp2(t + bits) + 4503599627370496.0;  // 2^52: the whole part is in the low bits, rounded to nearest
    return (u64)__double_as_longlong(v) & ((1ull << 52) - 1);
  }
  // the last step holds what has no weight
  __device__ __forceinline__ int bucket(double t) const {
    const double range = bits + 1;
    if (!(t > -range)) return kBuckets - 1;
    const int b = (int)(-t * ((kBuckets - 1) / range));
    return b < kBuckets - 2 ? b : kBuckets - 2;
  }
};

struct Shared {
  uint32_t count[kBuckets], sub_count[kBuckets];
  u64 mass[kBuckets], sub_mass[kBuckets];
  u64 list[kList];
  u64 wave_sum[kWaves];
  uint32_t wave_count[kWaves];
  float wave_max[kWaves];
  u64 low, high;
  // an answer: classes before its last one and with it, their sum, and the last one
  u64 found_mass, found_rank;
  uint32_t found_count, found_bucket, listed;
};

// f(x, class) for all classes of a row, in no order
template <typename T, typename F>
__device__ __forceinline__ void for_row(const T *row, int classes, F &&f) {
  for (int at = threadIdx.x * kVec; at < classes; at += kThreads * kVec) {
    float x[kVec];
    load8(row + at, classes - at, -INFINITY, x);
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (x[i] > -INFINITY) f(x[i], at + i);
  }
}

__device__ __forceinline__ u64 wave_scan(u64 v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 w = __shfl_up(v, o);
    if (lane >= o) v += w;
  }
  return v;
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t w = __shfl_up(v, o);
    if (lane >= o) v += w;
  }
  return v;
}
// Sums over the threads up to and with this one.
__device__ __forceinline__ void block_scan(Shared &sh, u64 &m, uint32_t &c) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  m = wave_scan(m), c = wave_scan(c);
  if (lane == 63) sh.wave_sum[wave] = m, sh.wave_count[wave] = c;
  __syncthreads();
  for (int w = 0; w < wave; ++w) m += sh.wave_sum[w], c += sh.wave_count[w];
  __syncthreads();
}
// Counts and masses of buckets become those up to and with each.
__device__ __forceinline__ void scan_buckets(Shared &sh, uint32_t *count, u64 *mass) {
  u64 m = 0;
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) m += mass[threadIdx.x * kPer + i], c += count[threadIdx.x * kPer + i];
  u64 mi = m;
  uint32_t ci = c;
  block_scan(sh, mi, ci);
  mi -= m, ci -= c;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    mi += mass[threadIdx.x * kPer + i], ci += count[threadIdx.x * kPer + i];
    mass[threadIdx.x * kPer + i] = mi, count[threadIdx.x * kPer + i] = ci;
  }
  __syncthreads();
}

// What is asked: the beginning of `n` classes, or the shortest one whose mass is at least, or more than, `target`.
enum Ask { kCount, kAtLeast, kMore };
__device__ __forceinline__ bool reached(Ask ask, uint32_t n, double target, uint32_t c, u64 m) {
  return ask == kCount ? c >= n : ask == kAtLeast ? (double)m >= target : (double)m > target;
}
// The first bucket behind which it is reached; `c0` and `m0` lie before the first bucket.  Found by one thread, known to all.
__device__ __forceinline__ int find_bucket(Shared &sh, const uint32_t *count, const u64 *mass, uint32_t c0, u64 m0, Ask ask, uint32_t n, double target) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = threadIdx.x * kPer + i;
    const bool here = reached(ask, n, target, c0 + count[b], m0 + mass[b]);
    const bool before = b > 0 && reached(ask, n, target, c0 + count[b - 1], m0 + mass[b - 1]);
    if (here && !before) sh.found_bucket = b;
  }
  __syncthreads();
  const int b = sh.found_bucket;
  __syncthreads();
  return b;
}

// The answer inside step `b` of the row, with found_count, found_mass (from the row's first class on) and found_rank set.
template <typename T>
__device__ void resolve(Shared &sh, const T *row, const Scale &sc, int classes, int b, Ask ask, uint32_t n, double target) {
  const int tid = threadIdx.x;
  uint32_t c0 = b ? sh.count[b - 1] : 0, size = sh.count[b] - c0;
  u64 m0 = b ? sh.mass[b - 1] : 0;
  u64 lo = 0, hi = ~0ull;
  if (size > kList) {
    if (tid == 0) sh.low = ~0ull, sh.high = 0;
    __syncthreads();
    u64 least = ~0ull, most = 0;
    for_row(row, classes, [&](float x, int id) {
      if (sc.bucket(sc.log_of(x)) == b) {
        const u64 r = rank_of(x, id);
        least = r < least ? r : least, most = r > most ? r : most;
      }
    });
    atomicMin(&sh.low, least), atomicMax(&sh.high, most);
    __syncthreads();
    lo = sh.low, hi = sh.high;
    __syncthreads();
    while (size > kList) {  // ranks differ, so steps of 2^shift end at one rank each
      const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > 11 ? bits - 11 : 0;
      for (int i = tid; i < kBuckets; i += kThreads) sh.sub_count[i] = 0, sh.sub_mass[i] = 0;
      __syncthreads();
      for_row(row, classes, [&](float x, int id) {
        const u64 r = rank_of(x, id);
        if (r >= lo && r <= hi) {
          const int at = (int)((r - lo) >> shift);
          atomicAdd(&sh.sub_count[at], 1u);
          atomicAdd(&sh.sub_mass[at], sc.units(sc.log_of(x)));
        }
      });
      __syncthreads();
      scan_buckets(sh, sh.sub_count, sh.sub_mass);
      const int at = find_bucket(sh, sh.sub_count, sh.sub_mass, c0, m0, ask, n, target);
      size = sh.sub_count[at] - (at ? sh.sub_count[at - 1] : 0);
      if (at) c0 += sh.sub_count[at - 1], m0 += sh.sub_mass[at - 1];
      lo += (u64)at << shift;
      const u64 end = lo + ((1ull << shift) - 1);
      hi = end < hi ? end : hi;
      __syncthreads();
    }
  }
  if (tid == 0) sh.listed = 0;
  __syncthreads();
  for_row(row, classes, [&](float x, int id) {
    if (sc.bucket(sc.log_of(x)) == b) {
      const u64 r = rank_of(x, id);
      if (r >= lo && r <= hi) sh.list[atomicAdd(&sh.listed, 1u)] = r;
    }
  });
  __syncthreads();
  // sorted by exchanges in a network; what the list does not fill stays behind
  if (tid >= (int)size) sh.list[tid] = ~0ull;
  int span = 2;
  while (span < (int)size) span <<= 1;
  __syncthreads();
  for (int k = 2; k <= span; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      const int other = tid ^ j;
      if (tid < span && other > tid) {
        const u64 x = sh.list[tid], y = sh.list[other];
        if ((x > y) == ((tid & k) == 0)) sh.list[tid] = y, sh.list[other] = x;
      }
      __syncthreads();
    }
  const u64 r = sh.list[tid];
  const u64 w = tid < (int)size ? sc.units(sc.log_of(value_of(r))) : 0;
  u64 m = w;
  uint32_t c = tid < (int)size;
  block_scan(sh, m, c);
  if (tid < (int)size && reached(ask, n, target, c0 + c, m0 + m) && (tid == 0 || !reached(ask, n, target, c0 + c - 1, m0 + m - w)))
    sh.found_count = c0 + c, sh.found_mass = m0 + m, sh.found_rank = r;
  __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_sample(Args g) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long at = blockIdx.x;
  const T *row = (const T *)g.logits + at * g.ld;

  float most = -INFINITY;
  bool nan = false;
  for (int i = tid * kVec; i < g.classes; i += kThreads * kVec) {
    float x[kVec];
    load8(row + i, g.classes - i, -INFINITY, x);
#pragma unroll
    for (int j = 0; j < kVec; ++j) most = fmaxf(most, x[j]), nan |= x[j] != x[j];
  }
  most = wave_max_all(most);
  if (lane == 0) sh.wave_max[wave] = most;
  nan = __syncthreads_or(nan);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) most = fmaxf(most, sh.wave_max[w]);
  if (nan || most == -INFINITY) {
    if (tid == 0) {
      g.tokens[at] = -1;
      if (g.kept) g.kept[at] = 0;
      if (g.logp) g.logp[at] = nan ? NAN : -INFINITY;
    }
    return;
  }

  const float temperature = g.temperature ? g.temperature[at] : 1.f;
  if (!(temperature > 0.f)) {
    if (tid == 0) sh.listed = 0xffffffffu;
    __syncthreads();
    uint32_t first = 0xffffffffu;
    for_row(row, g.classes, [&](float x, int id) {
      if (x == most) first = min(first, (uint32_t)id);
    });
    if (first != 0xffffffffu) atomicMin(&sh.listed, first);
    __syncthreads();
    if (tid == 0) {
      g.tokens[at] = (int32_t)sh.listed;
      if (g.kept) g.kept[at] = 1;
      if (g.logp) g.logp[at] = 0.f;
    }
    return;
  }

  const Scale sc{(double)most, 1.4426950408889634074 / (double)temperature, g.bits};
  for (int i = tid; i < kBuckets; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
  __syncthreads();
  uint32_t none = 0;  // without weight: no sum to add, and often most of a row
  for_row(row, g.classes, [&](float x, int) {
    const double t = sc.log_of(x);
    const int b = sc.bucket(t);
    if (b == kBuckets - 1) {
      ++none;
    } else {
      atomicAdd(&sh.count[b], 1u);
      atomicAdd(&sh.mass[b], sc.units(t));
    }
  });
  if (none) atomicAdd(&sh.count[kBuckets - 1], none);
  __syncthreads();
  scan_buckets(sh, sh.count, sh.mass);

  uint32_t kept = sh.count[kBuckets - 1];
  u64 mass = sh.mass[kBuckets - 1];
  const uint32_t k = g.top_k && g.top_k[at] > 0 ? (uint32_t)g.top_k[at] : kept;
  if (k < kept) {
    const int b = find_bucket(sh, sh.count, sh.mass, 0, 0, kCount, k, 0.0);
    kept = k, mass = sh.mass[b];
    if (b < kBuckets - 1 && sh.count[b] != k) {
      resolve(sh, row, sc, g.classes, b, kCount, k, 0.0);
      mass = sh.found_mass;
      __syncthreads();
    }
  }
  const float p = g.top_p ? g.top_p[at] : 1.f;
  if (p < 1.f) {
    const double target = (double)p * (double)mass;
    resolve(sh, row, sc, g.classes, find_bucket(sh, sh.count, sh.mass, 0, 0, kAtLeast, 0, target), kAtLeast, 0, target);
    kept = sh.found_count, mass = sh.found_mass;
    __syncthreads();
  }
  const float least = g.min_p ? g.min_p[at] : 0.f;
  if (least > 0.f) {
    const int b = sc.bucket(log2((double)least));
    const uint32_t c0 = b ? sh.count[b - 1] : 0;
    if (c0 < kept) {
      uint32_t c = 0;
      u64 m = 0;
      for_row(row, g.classes, [&](float x, int) {
        const double t = sc.log_of(x);
        if (sc.bucket(t) == b && exp2(t) >= (double)least) ++c, m += sc.units(t);
      });
      block_scan(sh, m, c);
      if (tid == kThreads - 1) sh.found_count = c0 + c, sh.found_mass = (b ? sh.mass[b - 1] : 0) + m;
      __syncthreads();
      if (sh.found_count < kept) kept = sh.found_count, mass = sh.found_mass;
      if (kept == 0) kept = 1, mass = sc.units(0.0);
      __syncthreads();
    }
  }
  const float u = fminf(fmaxf(g.uniform[at], 0.f), 0.99999994f);
  const double target = (double)u * (double)mass;
  resolve(sh, row, sc, g.classes, find_bucket(sh, sh.count, sh.mass, 0, 0, kMore, 0, target), kMore, 0, target);
  if (tid == 0) {
    g.tokens[at] = (int32_t)(sh.found_rank & ((1u << kIdBits) - 1));
    if (g.kept) g.kept[at] = (int32_t)kept;
    if (g.logp) g.logp[at] = (float)((sc.log_of(value_of(sh.found_rank)) + g.bits - log2((double)mass)) * 0.69314718055994530942);
  }
}

}  // namespace

int64_t sample_scratch_bytes(const parle_sample_desc &) { return 0; }

hipError_t launch_sample(hipStream_t st, const parle_sample_desc &d, const void *logits, const float *uniform, const float *temperature,
                         const int32_t *top_k, const float *top_p, const float *min_p, void *, int32_t *tokens, int32_t *kept, float *logp) {
  int bits = 50;
  while (d.classes > 1LL << (62 - bits)) --bits;
  Args g{logits, uniform, temperature, top_k, top_p, min_p, tokens, kept, logp, d.classes, bits, d.ld};
  const int rows = d.n * d.rows;
  if (d.dtype)
    k_sample<bf16_t><<<rows, kThreads, 0, st>>>(g);
  else
    k_sample<float><<<rows, kThreads, 0, st>>>(g);
  return hipGetLastError();
}
