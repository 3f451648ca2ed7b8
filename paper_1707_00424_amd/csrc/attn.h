// Shared pieces of the attention kernels: fragments of the matrix instructions, tiles in LDS, where a row's sequence lies.
//
// Everything is multiplied in transposed form, S^T = K Q^T and O^T = V^T P^T, so that a lane owns a query (its column of the
// 32 x 32 accumulators: lane l holds column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 in register i).  A row's maximum and sum are then
// register sums and one exchange between the halves of the wavefront, and P^T, as it leaves the accumulators, is the second operand of the
// next product: its eight values of a lane stand for keys 16 t + 8 (j / 4) + 4 (l / 32) + j % 4, and the first operand is read in that order.
#pragma once
#include <type_traits>

#include "igemm_dev.h"
#include "tok.h"

namespace attn {

using tok::u4;
typedef float f16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v lds_s4v;
typedef u4 u4_any __attribute__((aligned(2)));

constexpr int kWaves = 4, kThreads = kWaves * PARLE_WAVE;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Eight elements of a contraction.
template <typename T>
struct Frag {
  u4 v[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Frag<T> zero_frag() {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) f.v[i] = u4{0u, 0u, 0u, 0u};
  return f;
}
template <typename T>
__device__ __forceinline__ Frag<T> load_frag(const T *p) {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) f.v[i] = *(const u4_any *)((const char *)p + 16 * i);
  return f;
}
__device__ __forceinline__ float frag_at(const Frag<float> &f, int j) { return __uint_as_float(f.v[j >> 2][j & 3]); }
__device__ __forceinline__ float frag_at(const Frag<bf16_t> &f, int j) {
  const uint32_t w = f.v[0][j >> 1];
  return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
}
// Eight fp32 values as a fragment: bf16 products take P and dS rounded to nearest even, half a step, 2^-8 of each at most, at random signs.  Matrix instructions
// of fp32 are eight times slower, and two of bf16 for a value and its rest would double the second products.  Against 64 bits results are off by 2.2e-3 of
// their size (gradients 2.4e-3), of which rounding the result itself makes 1.65e-3.
template <typename T>
__device__ __forceinline__ Frag<T> make_frag(const float (&v)[8]);
template <>
__device__ __forceinline__ Frag<float> make_frag<float>(const float (&v)[8]) {
  Frag<float> f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = __float_as_uint(v[j]);
  return f;
}
template <>
__device__ __forceinline__ Frag<bf16_t> make_frag<bf16_t>(const float (&v)[8]) {
  Frag<bf16_t> f;
#pragma unroll
  for (int j = 0; j < 4; ++j) f.v[0][j] = f32x2_to_bf16x2(v[2 * j], v[2 * j + 1]);
  return f;
}

// acc[row of a][column of b] += sum over sixteen contraction values: eight of each half of the wavefront.
__device__ __forceinline__ void mma(const Frag<bf16_t> &a, const Frag<bf16_t> &b, f16v &acc) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a.v[0]), __builtin_bit_cast(bf8, b.v[0]), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(const Frag<float> &a, const Frag<float> &b, f16v &acc) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(frag_at(a, j), frag_at(b, j), acc, 0, 0, 0);
}
__device__ __forceinline__ f16v zero16() {
  f16v z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// A tile of rows in LDS, DP elements each, in 16-byte chunks whose place in the row is XORed with bits of the row, so that neither a chunk of sixteen
// rows nor 32 columns of four rows meet in a bank.
template <typename T, int DP>
struct Tile {
  static constexpr int kPitch = DP == 96 ? 128 : DP;             // elements of a row
  static constexpr int kChunk = 16 / sizeof(T);                  // elements of a chunk
  static constexpr int kRowBytes = kPitch * sizeof(T);
  static __device__ __forceinline__ int turn(int r) {
    if (sizeof(T) == 4) return (((r >> 2) & 1) << 3) | (((r >> 3) & 1) << 2) | (r & 3);
    if (kPitch == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    return ((r & 3) << 2) | ((r >> 2) & 3);
  }
  static __device__ __forceinline__ int at(int r, int chunk) { return r * kRowBytes + ((chunk ^ turn(r)) << 4); }
  // A lane's places in a tile: of elements 16 i + 8 (lane / 32) .. of row lane % 32, and of column 32 d + lane % 32.
  struct Places {
    static constexpr int kRow = sizeof(T) / 2, kCol = sizeof(T) == 2 ? 2 : 4;
    int row[DP / 16][kRow], col[DP / 32][kCol];
    __device__ __forceinline__ void init(int lane) {
      const int h = lane >> 5;
#pragma unroll
      for (int i = 0; i < DP / 16; ++i)
#pragma unroll
        for (int e = 0; e < kRow; ++e) row[i][e] = at(lane & 31, (2 * i + h) * kRow + e);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        if constexpr (sizeof(T) == 4) {
          const int c = 32 * d + (lane & 31);
#pragma unroll
          for (int j = 0; j < 4; ++j) col[d][j] = at(4 * h + j, c >> 2) + 4 * (c & 3);
        } else {
          // a transposing read: lane l of sixteen addresses row l / 4, columns 4 (l % 4) .. + 3 of a 4 x 16 block and receives its column l
          const int r = 4 * h + ((lane & 15) >> 2), c = 32 * d + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          col[d][0] = at(r, c >> 3) + 2 * (c & 7), col[d][1] = at(r + 8, c >> 3) + 2 * (c & 7);
        }
      }
    }
  };
  // elements 16 i + 8 (lane / 32) .. + 7 of row r0 + lane % 32, r0 a multiple of 32
  static __device__ __forceinline__ Frag<T> row(const char *tile, const Places &p, int r0, int i) {
    Frag<T> f;
#pragma unroll
    for (int e = 0; e < Places::kRow; ++e) f.v[e] = *(const u4 *)(tile + p.row[i][e] + r0 * kRowBytes);
    return f;
  }
  // column 32 d + lane % 32 of rows r0 + 8 (j / 4) + 4 (lane / 32) + j % 4, j = 0 .. 7; r0 a multiple of 16
  static __device__ __forceinline__ Frag<T> column(const char *tile, const Places &p, int r0, int d) {
    Frag<T> f;
    if constexpr (sizeof(T) == 4) {
      // the place of a chunk in a row differs by bit 2 of its index between rows 8 apart
#pragma unroll
      for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = *(const uint32_t *)(tile + (p.col[d][j & 3] ^ (j >> 2 ? 64 : 0)) + (r0 + 8 * (j >> 2)) * kRowBytes);
    } else {
      const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(tile + p.col[d][0] + r0 * kRowBytes));
      const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(tile + p.col[d][1] + r0 * kRowBytes));
      f.v[0] = __builtin_bit_cast(u4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    return f;
  }
};

// Rows of a matrix that go into tiles of ROWS rows, by all threads of a workgroup.  With DMA they go straight into LDS, arrive some time later
// (kLoads loads of each wavefront a tile) and are zeros behind the last row; without, they have arrived in front of the next barrier, and the last row
// stands for those behind it.  Columns from `dim` on are zeros.  DMA needs rows of whole 16 bytes, less than 2^31 bytes with those behind the last (`direct`).
template <typename T, int DP, int ROWS, bool DMA>
struct Loader {
  using Tl = Tile<T, DP>;
  static constexpr int kChunks = DP / Tl::kChunk, kTurns = (ROWS * kChunks + kThreads - 1) / kThreads;
  static constexpr int kRowChunks = Tl::kPitch / Tl::kChunk, kLoads = ROWS * Tl::kRowBytes / (kWaves * PARLE_WAVE * 16);
  static_assert(ROWS * Tl::kRowBytes == kLoads * kWaves * PARLE_WAVE * 16, "a tile is whole loads of all wavefronts");
  static constexpr uint32_t kFar = 0x80000000u;  // beyond any buffer, also with a row's offset, less than 2^31, added
  const T *base;
  long long ld;
  int last, dim;
  u4 desc;
  uint32_t off[DMA ? kLoads : 1], mine;  // a lane's places in the matrix, its wavefront's in a tile

  __device__ __forceinline__ void init(long long ld_, int dim_) {
    ld = ld_, dim = dim_;
    if constexpr (DMA) {
      mine = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) * kLoads * 1024);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = ((int)(threadIdx.x >> 6) * kLoads + i) * PARLE_WAVE + (threadIdx.x & 63), r = at / kRowChunks;
        const int c = (at % kRowChunks) ^ Tl::turn(r);
        off[i] = c * Tl::kChunk < dim ? (uint32_t)r * (uint32_t)(ld * sizeof(T)) + c * 16 : kFar;
      }
    }
  }
  // the matrix: rows up to `last` are there
  __device__ __forceinline__ void from(const T *p, int last_) {
    base = p, last = last_;
    if constexpr (DMA) desc = igemm_dev::buffer_desc(p, (uint32_t)(last + 1) * (uint32_t)(ld * sizeof(T)));
  }
  // from row `first` and column `shift` on
  __device__ __forceinline__ void load(char *tile, int first, int shift = 0) const {
    if constexpr (DMA) {
      const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)tile + mine;
      const uint32_t row = (uint32_t)first * (uint32_t)(ld * sizeof(T)) + (uint32_t)(shift * sizeof(T));
#pragma unroll
      for (int i = 0; i < kLoads; ++i) igemm_dev::dma16(__builtin_amdgcn_readfirstlane(lds + i * 1024), desc, off[i] + row, 0);
    } else {
      u4 v[kTurns];
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int at = (int)threadIdx.x + i * kThreads, r = at / kChunks, c = at % kChunks;
        v[i] = u4{0u, 0u, 0u, 0u};
        if ((ROWS * kChunks % kThreads == 0 || r < ROWS) && c * Tl::kChunk < dim)
          v[i] = *(const u4_any *)(base + (long long)min(first + r, last) * ld + shift + c * Tl::kChunk);
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int at = (int)threadIdx.x + i * kThreads, r = at / kChunks, c = at % kChunks;
        if (ROWS * kChunks % kThreads == 0 || r < ROWS) *(u4 *)(tile + Tl::at(r, c)) = v[i];
      }
    }
  }
};
// Whether a matrix can go straight into LDS.  Tiles begin at a row that is there and end up to 126 rows behind the last, by places of less than 2^31 bytes
// as well: beyond that they would come round to the first ones.
constexpr int kRowsBehind = 128;
inline bool direct(int tokens, int64_t ld, int64_t stride, int n, int size) {
  return ld * size % 16 == 0 && (n == 1 || stride * size % 16 == 0) && (tokens + (long long)kRowsBehind) * ld * size < 1LL << 31;
}
// What was loaded into registers is there.  In front of a loop whose loads go to LDS: the compiler, which does not count those, would wait for registers
// loaded before the loop at their first use in it, and so for all that is on its way.
__device__ __forceinline__ void settle() { __builtin_amdgcn_s_waitcnt(0); }
// All but the last N loads have arrived, and every wavefront is here.
template <int N>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The rows [start, end) of the sequence that row i of a replica belongs to; empty where there is none.  offsets NULL: one sequence of all rows.
struct Span {
  int start, end;
};
__device__ __forceinline__ Span span_of(const int32_t *offsets, int sequences, int tokens, int i) {
  if (!offsets) return {0, tokens};
  int lo = 0, hi = sequences;  // the last b in [0, sequences) with offsets[b] <= i, or 0
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= i)
      lo = mid;
    else
      hi = mid;
  }
  const int s = max(offsets[lo], 0), e = min(offsets[lo + 1], tokens);
  if (i < s || i >= e) return {0, 0};
  return {s, e};
}
// The rows that sequences cover: all that lie in one lie in [first, end).
__device__ __forceinline__ Span covered(const int32_t *offsets, int sequences, int tokens) {
  if (!offsets) return {0, tokens};
  return {min(max(offsets[0], 0), tokens), min(max(offsets[sequences], 0), tokens)};
}

// What a query sees: `count` keys from lo on, itself the last of them, and `sinks` from start on.
struct Sight {
  int lo, start;
  uint32_t count, sinks;
  __device__ __forceinline__ bool sees(int j) const { return ((uint32_t)(j - lo) < count) | ((uint32_t)(j - start) < sinks); }
};
__device__ __forceinline__ Sight sight_of(Span s, int i, int window, int sinks) {
  const bool some = s.end > s.start;
  const int lo = window > 0 ? max(s.start, i - min(i, window) + (window <= i ? 1 : 0)) : s.start;
  return {some ? lo : 0x7fffffff, some ? s.start : 0, some ? (uint32_t)(i - lo + 1) : 0u, some ? (uint32_t)min(sinks, i + 1 - s.start) : 0u};
}
// In a tile of sinks, which ends where the window of the first row begins, only sinks count, and only those.
__device__ __forceinline__ Sight only_sinks(const Sight &s, int end) {
  return {s.lo, s.start, 0u, (uint32_t)min((int)s.sinks, max(end - s.start, 0))};
}

// Values of the other half of the wavefront, in both halves.
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ bool non_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }

// Of a fragment's values: the finite ones, zeros for the others; and one for each of the others, zeros for the finite.
template <typename T>
__device__ __forceinline__ void part_finite(const Frag<T> &f, Frag<T> &finite, Frag<T> &others) {
  float a[8], b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = frag_at(f, j);
    const bool bad = non_finite(x);
    a[j] = bad ? 0.f : x, b[j] = bad ? 1.f : 0.f;
  }
  finite = make_frag<T>(a), others = make_frag<T>(b);
}

template <typename T>
__device__ __forceinline__ void store4(T *p, float a, float b, float c, float d);
template <>
__device__ __forceinline__ void store4<float>(float *p, float a, float b, float c, float d) {
  *(tok::f4_any *)p = f4{a, b, c, d};
}
template <>
__device__ __forceinline__ void store4<bf16_t>(bf16_t *p, float a, float b, float c, float d) {
  *(tok::us4_any *)p = f32x4_to_bf16x4(f4{a, b, c, d});
}

// Wavefronts of the kernels of queries that share queries where few take part: of fp32 tiles of 128 elements LDS holds those of two.
inline int most_parts(const parle_attention_desc &d) { return d.dtype || d.dim <= 64 ? 4 : 2; }
// Whether they do.  A workgroup of 128 queries that does not share takes a start and a step for each 64 keys that its queries see; one that shares takes
// 1 / parts of the queries, the same start, and half as long again for its part of the steps, but there may be several rounds of them.  A start is
// worth ten steps of bf16, two of fp32.  Measured, without and with sharing, one sequence: bf16, 64 elements, 4096 tokens of 8 heads 69 and 44 us, of 12 heads
// 70 and 59, of 16 heads 72 and 78; 128 elements, 8192 tokens of 2 heads 157 and 101, 2048 of 12 heads 47 and 56; fp32, 64 elements, 1024 tokens of 16 heads 84
// and 40, with a window of 256 38 and 31, of 24 heads with the window 38 and 45.
inline bool shares_keys(const parle_attention_desc &d) {
  const int parts = most_parts(d), queries = 128 / parts, places = d.dtype && d.dim <= 64 ? 512 : 256;
  const double start = d.dtype ? 10 : 2, length = (double)d.tokens / d.sequences, span = d.window > 0 && d.window < length ? d.window : length;
  const double wgs = (double)tok::ceil_div(d.tokens, queries) * d.heads * d.n, rounds = wgs > places ? wgs / places : 1;
  const double alone = start + (128 + span) / 64, shared = start + (queries + (span < length ? span : span / 2)) / 64 / parts * 1.5;
  return rounds * shared < alone;
}

struct Args {
  const void *q, *k, *v;
  const int32_t *offsets;
  void *out;
  float *lse;
  int n, tokens, sequences, heads, kv_heads, dim, window, sinks, tiles;
  float scale;
  long long ld_q, q_stride, ld_kv, kv_stride, ld_out, out_stride;
};

}  // namespace attn
