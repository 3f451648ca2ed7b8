// A class of every row from a given random number, behind temperature, top-k, top-p and min-p.
//
// In the order of falling logit (the lower class first where two are equal) every rule keeps a beginning, so all are questions of one kind: where does
// the count, or the sum of the weights e^((x - max) / T), reach a number?  Weights are whole multiples of 2^-s of the largest, so sums are
// exact in 64-bit integers, in any order, and the answers the same every time; they are formed in 64 bits, as a number next to a border is on one
// side of it or the other.
//
// A workgroup has a row.  Where few classes can stay, they are listed and sorted, and the list has all answers: a row of up to kList classes; the classes at
// or above the k-th largest of the threads' largest logits, which the k largest of all are among; or, without top-k, those that min-p leaves, with the
// sum of all the others' weights.  Else counts and sums over steps of 1/32 power of two say in which step an answer lies, and the row is read again
// for the classes of that step, up to kList of which are sorted.  More of them (many equal logits) are counted again in finer steps of value and class.
//
// A row of bf16 is counted by value first (by_values), so that 4096 weights are formed in 64 bits and not one for each class.
//
// What bounds it: 4 rows of 128000 bf16 with top-k 50 (20 us) are latency, two passes of a row by one workgroup and a chain of scans and a sort; 1024 rows of 50001
// bf16 with top-p and min-p (93 us, 102 MB read three times, twice from cache) the vector unit, about 35 operations for a class.  The same of fp32 with top-p
// takes 212, with min-p too 169, in weights of 64 bits for every class.
#include <type_traits>

#include "tok.h"

namespace {

using namespace tok;
typedef unsigned long long u64;

constexpr int kBuckets = 2048;
constexpr int kSteps = 32;    // steps of a power of two
constexpr int kNear = 12 * kSteps;
constexpr int kValues = 4096;  // values of a bf16 row that are counted: 32 octaves of 128
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
  static constexpr double kMagic = 6755399441055744.0 / kSteps;  // 1.5 * 2^52 / kSteps: a sum with it is rounded to steps, their number in its low bits
  static constexpr double kWhole = 4503599627370496.0;           // 2^52: a sum with it is rounded to whole numbers, in its low bits
  double most, per;     // the largest logit; log2(e) / temperature
  bool infinite;        // the largest logit is: it counts as 0, and all others as next to nothing
  int bits;
  const __attribute__((address_space(3))) double *table;  // 2^(j / kSteps)
  __device__ __forceinline__ Scale(float largest, float temperature, int bits_, const double *t)
      : most(largest), per(1.4426950408889634074 / (double)temperature), infinite(largest == INFINITY), bits(bits_),
        table((const __attribute__((address_space(3))) double *)t) {
    if (infinite) most = 0.0, per = 1.0;
  }
  // the weight's logarithm, base 2, <= 0; what has no weight, -inf too, is somewhere below
  __device__ __forceinline__ double log_of(float x) const {
    const float y = infinite ? (x == INFINITY ? 0.f : -1e30f) : x;
    return fmax(((double)y - most) * per, -(double)(bits + 2));
  }
  // the nearest step to t, counted downwards from the largest weight's; the last one holds what has no weight
  __device__ __forceinline__ int bucket(double t) const {
    if (!(t > -(double)(bits + 1))) return kBuckets - 1;
    return -(int)(uint32_t)__double_as_longlong(t + kMagic);
  }
  // 2^(t + up) for t >= -(bits + 2).  t = step / 32 + r, |r| <= 1/64: 2^t = 2^(step / 32) e^(r ln 2), by five terms of the series, the next of which
  // is below 3e-15
  __device__ __forceinline__ double power(double t, int up) const {
    const double z = t + kMagic, r = t - (z - kMagic);
    const int step = (int)(uint32_t)__double_as_longlong(z);
    constexpr double c = 0.69314718055994530942;
    double p = __builtin_fma(r, c * c * c * c * c / 120, c * c * c * c / 24);
    p = __builtin_fma(r, p, c * c * c / 6);
    p = __builtin_fma(r, p, c * c / 2);
    p = __builtin_fma(r, p, c);
    p *= r;
    const double base = table[step & (kSteps - 1)];
    return ldexp(__builtin_fma(base, p, base), (step >> 5) + up);
  }
  __device__ __forceinline__ u64 raw_units(double t) const { return (u64)__double_as_longlong(power(t, bits) + kWhole); }  // as kWhole and that
  __device__ __forceinline__ u64 units(double t) const { return t > -(double)(bits + 1) ? raw_units(t) - (u64)__double_as_longlong(kWhole) : 0; }
  // whether a class' weight is at least `least` > 0, fp32's smallest included: also of one too small to be counted
  __device__ __forceinline__ bool at_least(float x, float least) const {
    const float y = infinite ? (x == INFINITY ? 0.f : -1e30f) : x;
    return power(fmax(((double)y - most) * per, -160.0), 0) >= (double)least;
  }
};

__device__ __forceinline__ void hide(Raw8<bf16_t> &r, int i) { r.v[i] = 0xff80; }
__device__ __forceinline__ void hide(Raw8<float> &r, int i) { i < 4 ? r.a[i] = -INFINITY : r.b[i - 4] = -INFINITY; }
// A lane's value from another, without LDS: `ctrl` is the pattern of a row of sixteen; 0 where there is none.
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRows, 0xf, true);
}
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ u64 dpp(u64 v) {
  return (u64)dpp<kCtrl, kRows>((uint32_t)(v >> 32)) << 32 | dpp<kCtrl, kRows>((uint32_t)v);
}
// Sums over the lanes of a row of sixteen, or of the wavefront, up to and with this one.
template <typename V>
__device__ __forceinline__ V row_scan(V v) {
  v += dpp<0x111>(v), v += dpp<0x112>(v), v += dpp<0x114>(v), v += dpp<0x118>(v);  // from 1, 2, 4, 8 lanes below
  return v;
}
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
  v = row_scan(v);
  v += dpp<0x142, 0xa>(v), v += dpp<0x143, 0xc>(v);  // the last lane of a row to the next row, of the first half to the second
  return v;
}
// The largest value of the wavefront, in its last lane.
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
  v = max(v, dpp<0x111>(v)), v = max(v, dpp<0x112>(v)), v = max(v, dpp<0x114>(v)), v = max(v, dpp<0x118>(v));
  v = max(v, dpp<0x142, 0xa>(v)), v = max(v, dpp<0x143, 0xc>(v));
  return v;
}
// The value of lane ^ kBit.
template <int kBit>
__device__ __forceinline__ uint32_t across(uint32_t v) {
  if constexpr (kBit == 1) return dpp<0xb1>(v);
  if constexpr (kBit == 2) return dpp<0x4e>(v);
  if constexpr (kBit == 4) return dpp<0x1b>(dpp<0x141>(v));  // eight lanes mirrored, then each four
  if constexpr (kBit == 8) return dpp<0x128>(v);
  if constexpr (kBit == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return threadIdx.x & 32 ? r[0] : r[1];
}
__device__ __forceinline__ uint32_t least_of(const us8 &v) {
  typedef unsigned short us4 __attribute__((ext_vector_type(4)));
  typedef unsigned short us2 __attribute__((ext_vector_type(2)));
  const us4 a = __builtin_elementwise_min(__builtin_shufflevector(v, v, 0, 1, 2, 3), __builtin_shufflevector(v, v, 4, 5, 6, 7));
  const us2 b = __builtin_elementwise_min(__builtin_shufflevector(a, a, 0, 1), __builtin_shufflevector(a, a, 2, 3));
  return min((uint32_t)b[0], (uint32_t)b[1]);
}
// What is asked: the beginning of `n` classes, or the shortest one whose mass is at least, or more than, `target`.
enum Ask { kCount, kAtLeast, kMore };
__device__ __forceinline__ bool reached(Ask ask, uint32_t n, double target, uint32_t c, u64 m) {
  return ask == kCount ? c >= n : ask == kAtLeast ? (double)m >= target : (double)m > target;
}
struct Rules {
  float u, p, least;
  int wanted;
};

// A workgroup of THREADS, and what it has in LDS.
template <int THREADS>
struct Sampler {
  static constexpr int kThreads = THREADS, kWaves = kThreads / PARLE_WAVE, kPer = kBuckets / kThreads;
  static constexpr int kList = kThreads;
  static constexpr int kPick = kThreads * 600 / 1024;  // largest top-k by the threads' largest: 600 of 1024 threads hold about 900 classes

  struct Shared {
    uint32_t count[kBuckets], sub_count[kBuckets];
    u64 mass[kBuckets], sub_mass[kBuckets];
    u64 list[kList];
    u64 wave_sum[kWaves];
    uint32_t wave_count[kWaves];
    float wave_max[kWaves];
    double table[kSteps];
    u64 low, high, total;
    // an answer: classes before its last one and with it, their sum, and the last one
    u64 found_mass, found_rank;
    uint32_t found_count, found_bucket, listed;
    // of a row of bf16: how often each value occurs, and the answer that lies among the occurrences of one
    uint32_t times[kValues + 2 + PARLE_WAVE];
    u64 found_before, found_weight;
    uint32_t found_first;
    float found_value;
  };

  // f(x, class) for all classes of a row from the begin-th on, eight neighbours x at a time, in no order; -inf where eight begin with classes that others
  // have, and behind the last.  One load of a thread is on its way, which is enough beside fifteen other wavefronts: four, moved from register to register,
  // took 104 us for 92 (1024 rows of 50001 bf16).  The loop is not unrolled: a row takes few turns, and long code is fetched from memory for each.
  template <typename T, typename F>
  static __device__ __forceinline__ void for_raw(const T *row, int classes, F &&f, int begin = 0) {
    constexpr int kTurn = kThreads * kVec;
    const int last = max(classes - kVec, 0);
    int at = begin + threadIdx.x * kVec;
    Raw8<T> next;
    next.load(row + min(at, last), classes);
  #pragma unroll 1
    for (; at < classes; at += kTurn) {
      Raw8<T> x = next;
      if (classes >= kVec) next.load(row + min(at + kTurn, last), kVec);
      const int first = min(at, last);
      if (at != first || classes < kVec) {
  #pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (!(first + i >= at && first + i < classes)) hide(x, i);
      }
      f(x, first);
    }
  }
  template <typename T, typename F>
  static __device__ __forceinline__ void for_eights(const T *row, int classes, F &&f) {
    for_raw(row, classes, [&](const Raw8<T> &r, int id) {
      float x[kVec];
  #pragma unroll
      for (int i = 0; i < kVec; ++i) x[i] = r.at(i);
      f(x, id);
    });
  }
  // f(x, class) one by one
  template <typename T, typename F>
  static __device__ __forceinline__ void for_row(const T *row, int classes, F &&f) {
    for_eights(row, classes, [&](const float(&x)[kVec], int id) {
  #pragma unroll
      for (int i = 0; i < kVec; ++i) f(x[i], id + i);
    });
  }

  // Sums over the threads up to and with this one.
  static __device__ __forceinline__ void block_scan(Shared &sh, u64 &m, uint32_t &c) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    static_assert(kWaves <= 16, "a row of sixteen lanes adds the wavefronts");
    m = wave_scan(m), c = wave_scan(c);
    if (lane == 63) sh.wave_sum[wave] = m, sh.wave_count[wave] = c;
    __syncthreads();
    const u64 ms = row_scan(sh.wave_sum[lane % kWaves]);
    const uint32_t cs = row_scan(sh.wave_count[lane % kWaves]);
    if (wave > 0) {
      m += (u64)(uint32_t)__builtin_amdgcn_readlane((int)(ms >> 32), wave - 1) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)ms, wave - 1);
      c += (uint32_t)__builtin_amdgcn_readlane((int)cs, wave - 1);
    }
    __syncthreads();
  }
  // Counts and masses of buckets become those up to and with each.
  static __device__ __forceinline__ void scan_buckets(Shared &sh, uint32_t *count, u64 *mass) {
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

  // The first bucket behind which it is reached; `c0` and `m0` lie before the first bucket.  Found by one thread, known to all.
  static __device__ __forceinline__ int find_bucket(Shared &sh, const uint32_t *count, const u64 *mass, uint32_t c0, u64 m0, Ask ask, uint32_t n, double target) {
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

  // The list of `size` ranks in ascending order, one to a thread, ~0 behind them: by exchanges in a network, between lanes where they are near.
  static __device__ __forceinline__ u64 sorted(Shared &sh, uint32_t size) {
    const int tid = threadIdx.x;
    u64 x = tid < (int)size ? sh.list[tid] : ~0ull;
    int span = 64;
    while (span < (int)size) span <<= 1;
    auto keep = [&](u64 y, int j, int k) {
      const bool low = ((tid & j) == 0) == ((tid & k) == 0);  // this one keeps the lower
      x = low == (x < y) ? x : y;
    };
    auto near = [&](auto bit, int k) {
      constexpr int j = decltype(bit)::value;
      if (j < k) keep((u64)across<j>((uint32_t)(x >> 32)) << 32 | across<j>((uint32_t)x), j, k);
    };
  #pragma unroll 1
    for (int k = 2; k <= span; k <<= 1) {
  #pragma unroll 1
      for (int j = k >> 1; j >= 64; j >>= 1) {
        __syncthreads();
        sh.list[tid] = x;
        __syncthreads();
        keep(sh.list[tid ^ j], j, k);
      }
      if (tid < span) {
        near(std::integral_constant<int, 32>{}, k), near(std::integral_constant<int, 16>{}, k), near(std::integral_constant<int, 8>{}, k);
        near(std::integral_constant<int, 4>{}, k), near(std::integral_constant<int, 2>{}, k), near(std::integral_constant<int, 1>{}, k);
      }
    }
    return x;
  }

  // The answer inside step `b` of the row, with found_count, found_mass (from the row's first class on) and found_rank set.
  template <typename T>
  static __device__ void resolve(Shared &sh, const T *row, const Scale &sc, int classes, int b, Ask ask, uint32_t n, double target) {
    const int tid = threadIdx.x;
    uint32_t c0 = b ? sh.count[b - 1] : 0, size = sh.count[b] - c0;
    u64 m0 = b ? sh.mass[b - 1] : 0;
    u64 lo = 0, hi = ~0ull;
    // f(x, class, rank) for the classes of the step whose rank is within lo .. hi.  Logits that are not near it are told apart in fp32, eight at once: its
    // middle, and half its width and a little more.
    const double middle = sc.most - (double)b / kSteps / sc.per, half = 0.5 / kSteps / sc.per;
    const float mid = (float)middle, reach = (float)(half * 1.001 + 1e-6 * fabs(middle)) + 1e-37f;
    auto of_step = [&](auto f) {
      for_eights(row, classes, [&](const float(&x)[kVec], int id) {
        float near = fabsf(x[0] - mid);
  #pragma unroll
        for (int i = 1; i < kVec; ++i) near = fminf(near, fabsf(x[i] - mid));
        if (near <= reach || sc.infinite || !(reach < 3e38f)) {
  #pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (x[i] > -INFINITY && sc.bucket(sc.log_of(x[i])) == b) {
              const u64 r = rank_of(x[i], id + i);
              if (r >= lo && r <= hi) f(x[i], r);
            }
        }
      });
    };
    if (size > kList) {
      if (tid == 0) sh.low = ~0ull, sh.high = 0;
      __syncthreads();
      u64 least = ~0ull, most = 0;
      of_step([&](float, u64 r) { least = r < least ? r : least, most = r > most ? r : most; });
      atomicMin(&sh.low, least), atomicMax(&sh.high, most);
      __syncthreads();
      lo = sh.low, hi = sh.high;
      __syncthreads();
      while (size > kList) {  // ranks differ, so steps of 2^shift end at one rank each
        const int bits = 64 - __clzll((long long)(hi - lo)), shift = bits > 11 ? bits - 11 : 0;
        for (int i = tid; i < kBuckets; i += kThreads) sh.sub_count[i] = 0, sh.sub_mass[i] = 0;
        __syncthreads();
        of_step([&](float x, u64 r) {
          const int at = (int)((r - lo) >> shift);
          atomicAdd(&sh.sub_count[at], 1u);
          atomicAdd(&sh.sub_mass[at], sc.units(sc.log_of(x)));
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
    of_step([&](float, u64 r) { sh.list[atomicAdd(&sh.listed, 1u)] = r; });
    __syncthreads();
    const u64 r = sorted(sh, size);
    const u64 w = tid < (int)size ? sc.units(sc.log_of(value_of(r))) : 0;
    u64 m = w;
    uint32_t c = tid < (int)size;
    block_scan(sh, m, c);
    if (tid < (int)size && reached(ask, n, target, c0 + c, m0 + m) && (tid == 0 || !reached(ask, n, target, c0 + c - 1, m0 + m - w)))
      sh.found_count = c0 + c, sh.found_mass = m0 + m, sh.found_rank = r;
    __syncthreads();
  }

  // A bound that at least `k` threads' values reach, or all threads' least: the upper sixteen bits of the k-th largest value's order, by two counts of
  // eight bits.
  static __device__ float bound_of(Shared &sh, float value, uint32_t k) {
    const int tid = threadIdx.x;
    const uint32_t up = (uint32_t)(~(rank_of(value, 0) >> kIdBits));  // ascends with the value
    uint32_t prefix = 0, left = k;
  #pragma unroll
    for (int round = 0; round < 2; ++round) {
      const int shift = 24 - 8 * round;
      if (tid < 256) sh.sub_count[tid] = 0;
      __syncthreads();
      if (round == 0 || (up >> 24) == prefix >> 24) atomicAdd(&sh.sub_count[255 - ((up >> shift) & 255)], 1u);
      __syncthreads();
      if (tid < 64) {
        uint32_t c[4], sum = 0;
  #pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = sh.sub_count[4 * tid + i], sum += c[i];
        uint32_t before = wave_scan(sum) - sum;
  #pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < left && before + c[i] >= left) sh.found_bucket = 255 - (4 * tid + i), sh.found_count = before;
          before += c[i];
        }
      }
      __syncthreads();
      prefix |= sh.found_bucket << shift, left -= sh.found_count;
      __syncthreads();
    }
    const float bound = __uint_as_float(prefix ^ ((prefix >> 31) ? 0x80000000u : 0xffffffffu));
    return bound == bound ? bound : -INFINITY;  // the order of -inf, cut to sixteen bits, is that of a NaN
  }

  // A row of bf16 by the values that occur in it: 128 to an octave, of which kValues hold the largest ones down to what has no weight, but for a band around zero,
  // whose few classes are listed.  So only values have weights formed, and a rule's answer is how many occurrences of one stay.  False where the band
  // has too many classes.
  static __device__ __forceinline__ bool by_values(Shared &sh, const bf16_t *row, const Scale &sc, int classes, float largest, const Rules &rules, uint32_t &kept, u64 &mass,
                                            u64 &rank) {
    constexpr int kEach = kValues / kThreads;
    const int tid = threadIdx.x;
    // magnitudes as bf16 codes: those of positive values go from the largest logit's down to c0, of negative ones from c0 up to what has no weight and does
    // not reach min-p
    const float none = (float)(sc.most - fmax((double)(sc.bits + 2), rules.least > 0.f ? 1.0 - log2((double)rules.least) : 0.0) / sc.per);
    const int top_p = largest > 0.f ? (int)(__float_as_uint(largest) >> 16) : -1, top_n = none < 0.f ? (int)min(__float_as_uint(-none) >> 16, 0x7f7fu) : -1;
    // Octaves of both sides, 32 together at most, so that places are kValues at most: as deep on one as on the other, but 32 of the larger side where the
    // other has none or none as large, a largest logit just above zero for one, which is of the band then.
    const int op = top_p >> 7, on = top_n >> 7;
    // (zeros are of the band: both are one value)
    const int c0 = max(max((op + on - 30 + 1) >> 1, max(op, on) - 31) * 128, 1);
    const int count_p = top_p >= c0 ? top_p - c0 + 1 : 0, count_n = top_n >= c0 ? top_n - c0 + 1 : 0, shift_n = count_p - c0;
    // Places: the positive values', two for the band, the negative values', and those of what has no weight, a lane's own.  As whole numbers positive
    // values go down to count_p, negative ones, which are their magnitude less 2^15, up.
    const int from_p = max(top_p, 0), low_n = count_p + 1, none_n = count_p + count_n + 2 + (tid & 63), turn_n = 0x8000 + shift_n + 2;
    for (int i = tid; i < kValues + 2 + PARLE_WAVE; i += kThreads) sh.times[i] = 0;
    if (tid == 0) sh.listed = 0, sh.total = 0;
    __syncthreads();
    for_raw(row, classes, [&](const Raw8<bf16_t> &r, int id) {
      const u4 w = __builtin_bit_cast(u4, r.v);
  #pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const int x = i & 1 ? (int)w[i >> 1] >> 16 : (int)(w[i >> 1] << 16) >> 16;
        const int p = min(from_p - x, count_p), n = min(max(x + turn_n, low_n), none_n);
        atomicAdd(&sh.times[x < 0 ? n : p], 1u);
      }
      const us8 size = r.v & (bf16_t)0x7fff;
      if (least_of(size) < c0) {
  #pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (size[i] < c0 && r.at(i) >= none) {
            const uint32_t n = atomicAdd(&sh.listed, 1u);
            if (n < kList) sh.list[n] = rank_of(r.at(i), id + i);
          }
      }
    });
    __syncthreads();
    const uint32_t in_band = sh.listed;
    if (in_band > kList) return false;
    // the band, sorted, and its sums
    const u64 band_rank = sorted(sh, in_band);
    const float band_value = value_of(band_rank);
    const bool banded = tid < (int)in_band;
    const u64 band_w = banded ? sc.units(sc.log_of(band_value)) : 0;
    u64 band_m = band_w;
    uint32_t band_c = banded;
    __syncthreads();
    block_scan(sh, band_m, band_c);
    if (tid == kThreads - 1) sh.total = band_m;
    __syncthreads();
    const u64 band_mass = sh.total;
    // a thread's values: their weights, and counts and masses in front of them
    auto value = [&](int i) {
      const int at = tid * kEach + i;
      return __uint_as_float((uint32_t)(at < count_p ? top_p - at : (at - shift_n) | 0x8000) << 16);
    };
    u64 weight[kEach], before_m = 0;
    uint32_t times[kEach], before_c = 0, stays = 0;
  #pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = tid * kEach + i;
      times[i] = at < count_p ? sh.times[at] : at < count_p + count_n ? sh.times[at + 2] : 0;
      weight[i] = 0;
      if (times[i]) {
        weight[i] = sc.units(sc.log_of(value(i)));
        stays |= (uint32_t)(rules.least > 0.f && sc.at_least(value(i), rules.least)) << i;
      }
      before_m += times[i] * weight[i], before_c += times[i];
    }
    {
      u64 m = before_m;
      uint32_t c = before_c;
      block_scan(sh, m, c);
      before_m = m - before_m, before_c = c - before_c;
    }
    // the band lies behind the positive values
    auto in_front = [&](int i, uint32_t &c, u64 &m) {
      c = before_c, m = before_m;
      for (int j = 0; j < i; ++j) c += times[j], m += times[j] * weight[j];
      if (tid * kEach + i >= count_p) c += in_band, m += band_mass;
    };
    u64 positive_m = 0;
    uint32_t positive_c = 0;
  #pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (tid * kEach + i == (count_p ? count_p - 1 : 0)) {
        uint32_t c;
        u64 m;
        in_front(i, c, m);
        sh.found_count = count_p ? c + times[i] : 0, sh.found_mass = count_p ? m + times[i] * weight[i] : 0;
      }
    if (tid == kThreads - 1) sh.found_first = before_c, sh.found_before = before_m;
    __syncthreads();
    positive_c = sh.found_count, positive_m = sh.found_mass;
    __syncthreads();
    if (tid == kThreads - 1) {
      uint32_t c = before_c + in_band;
      u64 m = before_m + band_mass;
  #pragma unroll
      for (int i = 0; i < kEach; ++i) c += times[i], m += times[i] * weight[i];
      sh.found_count = c, sh.found_mass = m;
    }
    __syncthreads();
    const uint32_t weighted = sh.found_count;
    kept = weighted, mass = sh.found_mass;
    __syncthreads();
    if (weighted < (uint32_t)classes && !(rules.p < 1.f) && !(rules.least > 0.f)) {  // those without weight stay too
      uint32_t above = 0;
      for_row(row, classes, [&](float x, int) { above += x > -INFINITY; });
      u64 unused = 0;
      block_scan(sh, unused, above);
      if (tid == kThreads - 1) sh.found_count = above;
      __syncthreads();
      kept = sh.found_count;
      __syncthreads();
    }
    // the value, or the class of the band, that an answer lies in: sums in front of it and its weight
    auto ask_for = [&](Ask ask, uint32_t n, double target) {
  #pragma unroll
      for (int i = 0; i < kEach; ++i) {
        uint32_t c;
        u64 m;
        in_front(i, c, m);
        if (times[i] && reached(ask, n, target, c + times[i], m + times[i] * weight[i]) && !(c && reached(ask, n, target, c, m)))
          sh.found_first = c, sh.found_before = m, sh.found_weight = weight[i], sh.found_value = value(i), sh.found_rank = ~0ull;
      }
      const uint32_t c = positive_c + band_c - 1;
      const u64 m = positive_m + band_m - band_w;
      if (banded && reached(ask, n, target, c + 1, m + band_w) && !(c && reached(ask, n, target, c, m)))
        sh.found_first = c, sh.found_before = m, sh.found_weight = band_w, sh.found_rank = band_rank;
      __syncthreads();
    };
    // the fewest occurrences, one at least, that reach the target
    auto occurrences = [&](Ask ask, double target) {
      const u64 w = sh.found_weight, m = sh.found_before;
      uint32_t r = w ? (uint32_t)fmin(fmax((target - (double)m) / (double)w, 1.0), 4.2e6) : 1;
      while (r > 1 && reached(ask, 0, target, 0, m + (r - 1) * w)) --r;
      while (w && !reached(ask, 0, target, 0, m + r * w)) ++r;
      return r;
    };
    if (rules.wanted > 0 && (uint32_t)rules.wanted < kept) {
      kept = (uint32_t)rules.wanted;
      if (kept < weighted) {
        ask_for(kCount, kept, 0.0);
        mass = sh.found_before + (kept - sh.found_first) * sh.found_weight;
        __syncthreads();
      }
    }
    if (rules.p < 1.f) {
      const double target = (double)rules.p * (double)mass;
      ask_for(kAtLeast, 0, target);
      const uint32_t r = occurrences(kAtLeast, target);
      kept = sh.found_first + r, mass = sh.found_before + r * sh.found_weight;
      __syncthreads();
    }
    if (rules.least > 0.f) {
      // what stays is a beginning: its last value, or class of the band, knows its sums
      uint32_t most_c = 0;
      u64 most_m = 0;
  #pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (stays >> i & 1) {
          in_front(i, most_c, most_m);
          most_c += times[i], most_m += times[i] * weight[i];
        }
      if (banded && sc.at_least(band_value, rules.least) && positive_c + band_c > most_c) most_c = positive_c + band_c, most_m = positive_m + band_m;
      if (tid == 0) sh.found_count = 1, sh.found_mass = sc.units(0.0);
      __syncthreads();
      const uint32_t c = wave_most(most_c);
      if ((tid & 63) == 63) atomicMax(&sh.found_count, c);
      __syncthreads();
      if (most_c == sh.found_count && most_c > 1) sh.found_mass = most_m;
      __syncthreads();
      if (sh.found_count < kept) kept = sh.found_count, mass = sh.found_mass;
      __syncthreads();
    }
    const double target = (double)rules.u * (double)mass;
    ask_for(kMore, 0, target);
    rank = sh.found_rank;
    if (rank != ~0ull) return true;
    // The class of that occurrence, in the order of classes.  Where more have the value than are listed, it is looked for in one of kValues ranges of
    // them, known by counts, and again in a part of that, until the list holds what is left.
    uint32_t r = occurrences(kMore, target);
    const float v = sh.found_value;
    const bf16_t code = (bf16_t)(__float_as_uint(v) >> 16);
    int from = 0, to = classes;
    __syncthreads();
  #pragma unroll 1
    while (true) {
      if (tid == 0) sh.listed = 0;
      __syncthreads();
      for_raw(row, classes, [&](const Raw8<bf16_t> &x, int id) {
        const us8 other = x.v ^ code;
        if (least_of(other) == 0) {
  #pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (other[i] == 0 && id + i >= from && id + i < to) {
              const uint32_t n = atomicAdd(&sh.listed, 1u);
              if (n < kList) sh.list[n] = rank_of(v, id + i);
            }
        }
      });
      __syncthreads();
      if (sh.listed <= kList) break;
      for (int i = tid; i < kValues; i += kThreads) sh.times[i] = 0;
      __syncthreads();
      const int range = (to - from + kValues - 1) / kValues;
      for_row(row, classes, [&](float x, int id) {
        if (x == v && id >= from && id < to) atomicAdd(&sh.times[(id - from) / range], 1u);
      });
      __syncthreads();
      uint32_t c = 0, each[kEach];
  #pragma unroll
      for (int i = 0; i < kEach; ++i) each[i] = sh.times[tid * kEach + i], c += each[i];
      u64 m = 0;
      uint32_t upto = c;
      block_scan(sh, m, upto);
      upto -= c;
  #pragma unroll
      for (int i = 0; i < kEach; ++i) {
        if (upto < r && upto + each[i] >= r) sh.found_first = upto, sh.found_bucket = tid * kEach + i;
        upto += each[i];
      }
      __syncthreads();
      from += sh.found_bucket * range, to = min(from + range, to), r -= sh.found_first;
      __syncthreads();
    }
    const u64 x = sorted(sh, sh.listed);
    __syncthreads();
    if (tid == (int)r - 1) sh.found_rank = x;
    __syncthreads();
    rank = sh.found_rank;
    return true;
  }

  // A thread's largest logit, and whether it has met a NaN.
  static __device__ __forceinline__ float largest_of(const float *row, int classes, bool &nan) {
    float most = -INFINITY;
    bool odd = false;
    for_row(row, classes, [&](float x, int) { most = fmaxf(most, x), odd |= x != x; });
    nan = odd;
    return most;
  }
  // of bf16 as whole numbers, two at a time: those of positive values ascend with them, of negative ones with their magnitude
  static __device__ __forceinline__ float largest_of(const bf16_t *row, int classes, bool &nan) {
    typedef short s8 __attribute__((ext_vector_type(8)));
    s8 up;
    us8 down, top;
  #pragma unroll
    for (int i = 0; i < kVec; ++i) up[i] = (short)0x8000, down[i] = 0xff80, top[i] = 0;
    auto add = [&](const Raw8<bf16_t> &r, int) {
      const us8 v = r.v;
      up = __builtin_elementwise_max(up, __builtin_bit_cast(s8, v));
      down = __builtin_elementwise_min(down, v), top = __builtin_elementwise_max(top, v);
    };
    // the row comes from memory: several loads of a thread at a time
    constexpr int kAtOnce = 4, kBlock = kAtOnce * kThreads * kVec;
    const int whole = classes / kBlock * kBlock;
  #pragma unroll 1
    for (int at = threadIdx.x * kVec; at < whole; at += kBlock) {
      Raw8<bf16_t> r[kAtOnce];
  #pragma unroll
      for (int j = 0; j < kAtOnce; ++j) r[j].load(row + at + j * kThreads * kVec, kVec);
  #pragma unroll
      for (int j = 0; j < kAtOnce; ++j) add(r[j], 0);
    }
    if (whole < classes) for_raw(row, classes, add, whole);
    int p = up[0];
    uint32_t n = down[0], t = top[0];
  #pragma unroll
    for (int i = 1; i < kVec; ++i) p = max(p, (int)up[i]), n = min(n, (uint32_t)down[i]), t = max(t, (uint32_t)top[i]);
    nan = p > 0x7f80 || t > 0xff80;
    return __uint_as_float((p >= 0 ? (uint32_t)p : n) << 16);
  }

  template <typename T>
  static __device__ __forceinline__ void row_of(Shared &sh, const Args &g) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long at = blockIdx.x;
    const T *row = (const T *)g.logits + at * g.ld;
    const float temperature = g.temperature ? g.temperature[at] : 1.f, p = g.top_p ? g.top_p[at] : 1.f, least = g.min_p ? g.min_p[at] : 0.f;
    const float u = fminf(fmaxf(g.uniform[at], 0.f), 0.99999994f);
    const int wanted = g.top_k ? g.top_k[at] : 0;

    bool nan;
    const float mine = largest_of(row, g.classes, nan);
    float most = wave_max_all(mine);
    if (lane == 0) sh.wave_max[wave] = most;
    if (tid < kSteps) sh.table[tid] = exp2((double)tid / kSteps);
    if (tid == 0) sh.listed = 0, sh.total = 0;
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

    if (!(temperature > 0.f)) {
      if (tid == 0) sh.listed = 0xffffffffu;
      __syncthreads();
      uint32_t first = 0xffffffffu;
      if (mine == most)
        for_row(row, g.classes, [&](float x, int id) { first = x == most ? min(first, (uint32_t)id) : first; });
      if (first != 0xffffffffu) atomicMin(&sh.listed, first);
      __syncthreads();
      if (tid == 0) {
        g.tokens[at] = (int32_t)sh.listed;
        if (g.kept) g.kept[at] = 1;
        if (g.logp) g.logp[at] = 0.f;
      }
      return;
    }

    const Scale sc(most, temperature, g.bits, sh.table);
    uint32_t kept;
    u64 mass, rank = 0;
    auto list = [&](float x, int id) {
      const uint32_t i = atomicAdd(&sh.listed, 1u);
      if (i < kList) sh.list[i] = rank_of(x, id);
    };
    bool done = false;
    if constexpr (sizeof(T) == 2) {
      if (g.classes > kList && most < INFINITY && !(wanted > 0 && wanted <= kPick)) {
        done = by_values(sh, row, sc, g.classes, most, Rules{u, p, least, wanted}, kept, mass, rank);
        if (!done) {  // the list begins anew
          __syncthreads();
          if (tid == 0) sh.listed = 0;
          __syncthreads();
        }
      }
    }
    const bool picks = wanted > 0 && wanted <= kPick, cuts = wanted <= 0 && least > 0.f && most < INFINITY;
    uint32_t size = kList + 1;
    if (done) {
    } else if (g.classes <= kList || picks) {
      const float bound = g.classes <= kList ? -INFINITY : bound_of(sh, mine, wanted);
      if (g.classes <= kList || mine >= bound)
        for_row(row, g.classes, [&](float x, int id) {
          if (x >= bound && x > -INFINITY) list(x, id);
        });
      __syncthreads();
      size = sh.listed;
    } else if (cuts) {
      // what reaches min-p is at or above this logit, and a little more is
      const float from = most + (float)(log((double)least) * (double)temperature) * 1.00001f - 1e-5f * fabsf(most);
      u64 m = 0;
      uint32_t n = 0;
      for_eights(row, g.classes, [&](const float(&x)[kVec], int id) {
        float top = x[0];
  #pragma unroll
        for (int i = 0; i < kVec; ++i) {
          m += sc.raw_units(sc.log_of(x[i])), top = fmaxf(top, x[i]);
          if (i % 4 == 3) asm volatile("" : "+v"(m));  // now: left for later, all of a turn's weights would wait in registers
        }
        n += kVec;
        if (top >= from) {
  #pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (x[i] >= from) list(x[i], id + i);
        }
      });
      atomicAdd(&sh.total, m - n * (u64)__double_as_longlong(Scale::kWhole));
      __syncthreads();
      size = sh.listed;
      if (size == 0) size = kList + 1;  // min-p leaves none: the first stays
    }
    if (done) {
    } else if (size <= kList) {
      const u64 r = sorted(sh, size);
      const u64 w = tid < (int)size ? sc.units(sc.log_of(value_of(r))) : 0;
      u64 m = w;
      uint32_t c = tid < (int)size;
      __syncthreads();
      block_scan(sh, m, c);
      // the sum after top-k; then each rule's count
      kept = wanted > 0 ? min((uint32_t)wanted, size) : size;
      if (tid == (int)kept - 1) sh.found_mass = m;
      if (tid == 0) sh.found_count = 0xffffffffu;
      __syncthreads();
      mass = cuts && g.classes > kList ? sh.total : sh.found_mass;
      const double target = (double)p * (double)mass;
      if (p < 1.f && tid < (int)size && (double)m >= target && (tid == 0 || (double)(m - w) < target)) sh.found_count = tid + 1;
      __syncthreads();
      kept = min(kept, sh.found_count);
      if (least > 0.f) {
        const int stay = __syncthreads_count(tid < (int)size && sc.at_least(value_of(r), least));
        kept = min(kept, (uint32_t)max(stay, 1));
      }
      if (tid == (int)kept - 1) sh.found_mass = m;
      __syncthreads();
      mass = sh.found_mass;
      const double goal = (double)u * (double)mass;
      if ((double)m > goal && (double)(m - w) <= goal) sh.found_rank = r;
      __syncthreads();
      rank = sh.found_rank;
    } else {
      // Steps of the largest weights first: most answers lie there, few classes do, and the sums of the others need no atomics.  All steps where an
      // answer lies behind them.
      for (int last = kNear; !done; last = kBuckets - 1) {
        done = true;
        const bool all = last == kBuckets - 1;
        for (int i = tid; i < kBuckets; i += kThreads) sh.count[i] = 0, sh.mass[i] = 0;
        __syncthreads();
        uint32_t others = 0;
        u64 other_mass = 0;
        for_eights(row, g.classes, [&](const float(&x)[kVec], int) {
  #pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const double t = sc.log_of(x[i]);
            const int b = sc.bucket(t);
            const u64 w = sc.raw_units(t) - (u64)__double_as_longlong(Scale::kWhole);
            const bool near = b < last;
            if (near) atomicAdd(&sh.count[b], 1u), atomicAdd(&sh.mass[b], w);
            others += !near & (x[i] > -INFINITY), other_mass += near ? 0 : w;
            if (i % 4 == 3) asm volatile("" : "+v"(other_mass));
          }
        });
        if (others) atomicAdd(&sh.count[kBuckets - 1], others), atomicAdd(&sh.mass[kBuckets - 1], other_mass);
        __syncthreads();
        scan_buckets(sh, sh.count, sh.mass);

        kept = sh.count[kBuckets - 1], mass = sh.mass[kBuckets - 1];
  #pragma unroll 1
        for (int rule = 0; rule < 3 && done; ++rule) {
          Ask ask = kMore;
          uint32_t n = 0;
          double target = 0.0;
          if (rule == 0) {
            if (wanted <= 0 || (uint32_t)wanted >= kept) continue;
            ask = kCount, n = (uint32_t)wanted;
          } else if (rule == 1) {
            if (!(p < 1.f)) continue;
            ask = kAtLeast, target = (double)p * (double)mass;
          } else {
            if (least > 0.f) {
              const int b = sc.bucket(fmin(log2((double)least), 0.0));
              const uint32_t c0 = b ? sh.count[b - 1] : 0;
              if (c0 < kept && !all && b >= last) {
                done = false;
                break;
              }
              if (c0 < kept) {
                uint32_t c = 0;
                u64 m = 0;
                for_row(row, g.classes, [&](float x, int) {
                  const double t = sc.log_of(x);
                  if (x > -INFINITY && sc.bucket(t) == b && sc.at_least(x, least)) ++c, m += sc.units(t);
                });
                block_scan(sh, m, c);
                if (tid == kThreads - 1) sh.found_count = c0 + c, sh.found_mass = (b ? sh.mass[b - 1] : 0) + m;
                __syncthreads();
                if (sh.found_count < kept) kept = sh.found_count, mass = sh.found_mass;
                if (kept == 0) kept = 1, mass = sc.units(0.0);
                __syncthreads();
              }
            }
            target = (double)u * (double)mass;
          }
          const int b = find_bucket(sh, sh.count, sh.mass, 0, 0, ask, n, target);
          if (!all && b >= last) {
            done = false;
            break;
          }
          if (rule == 0 && (b == kBuckets - 1 || sh.count[b] == n)) {  // the whole step, or classes without weight
            kept = n, mass = sh.mass[b];
            continue;
          }
          resolve(sh, row, sc, g.classes, b, ask, n, target);
          if (rule < 2) kept = sh.found_count, mass = sh.found_mass;
          __syncthreads();
        }
      }
      rank = sh.found_rank;
    }
    if (tid == 0) {
      g.tokens[at] = (int32_t)(rank & ((1u << kIdBits) - 1));
      if (g.kept) g.kept[at] = (int32_t)kept;
      if (g.logp) g.logp[at] = (float)((sc.log_of(value_of(rank)) + g.bits - log2((double)mass)) * 0.69314718055994530942);
    }
  }
};

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void k_sample(Args g) {
  __shared__ typename Sampler<THREADS>::Shared sh;
  Sampler<THREADS>::template row_of<T>(sh, g);
}

}  // namespace

int64_t sample_scratch_bytes(const parle_sample_desc &) { return 0; }

hipError_t launch_sample(hipStream_t st, const parle_sample_desc &d, const void *logits, const float *uniform, const float *temperature,
                         const int32_t *top_k, const float *top_p, const float *min_p, void *, int32_t *tokens, int32_t *kept, float *logp) {
  int bits = 50;
  while (d.classes > 1LL << (62 - bits)) --bits;
  Args g{logits, uniform, temperature, top_k, top_p, min_p, tokens, kept, logp, d.classes, bits, d.ld};
  const int rows = d.n * d.rows;
  // More rows than compute units: workgroups of 512 threads, two to a compute unit, where one's serial steps hide behind the other's passes.  In us, against
  // workgroups of 1024, top-p and min-p without top-k: bf16, 1024 rows of 50001 classes 87 and 104, of 5001 47 and 64, of 1000 41 and 46, 300 of 50001 42 and 52,
  // 257 of 1000 18 and 15; 256 of 50001 32 and 28, 64 of 128000 40 and 34.  fp32, 1024 of 50001 168 and 170, of 1000 24 and 45, 257 of 1000 12 and 15; 256 of
  // 50001 91 and 59; but 300 of 50001 114 and 93, 512 132 and 109, as one long row's passes are most of the time.  With a top-k of 50 the smaller ones win
  // wherever they are taken: 1024 of 50001 46 and 54, 257 of 1000 11 and 14 (fp32 9 and 14), and lose below: 64 of 128000 29 and 22.
  const bool many = rows > 256;
  auto go = [&](auto *kernel, int threads) {
    kernel<<<rows, threads, 0, st>>>(g);
    return hipGetLastError();
  };
  if (d.dtype) return many ? go(k_sample<bf16_t, 512>, 512) : go(k_sample<bf16_t, 1024>, 1024);
  return many ? go(k_sample<float, 512>, 512) : go(k_sample<float, 1024>, 1024);
}
