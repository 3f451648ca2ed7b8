// Product of 8-bit matrices with power-of-two scales for 128 values: out = a b^T + bias.
//
// The matrix instructions take the scales themselves (one E8M0 byte per row and 32 values of the contraction), so four
// neighbouring blocks of 32 get the same byte and no accumulator is ever multiplied: the inner loop is loads, LDS reads and
// matrix instructions.  Both operands are rows of codes along the contraction, which is the order in which a lane wants them.
//
// The type of the result decides between two kinds of matrix instructions (EXACT below).  The 8-bit ones add groups of eight products,
// cut to 13 binary places below the largest of the group, to fp32 accumulators (measured: next to a product of 2^16, 2^3 is kept
// and 2^2 is not; the same with and without scales).  For normally distributed operands that is about 2e-5 of the result, a hundredth
// of the rounding of a result in bf16.  A result in fp32, such as the gradient of a parameter, is to have fp32 sums: there the codes
// become bf16 numbers times their scale, which is exact, and the bf16 instructions add them without such a cut, at half
// the rate.  (A scale of 2^-127 counts as 0 in that conversion.)
#include "igemm_dev.h"
#include "tok.h"

namespace {

using igemm_dev::buffer_desc;
using igemm_dev::dma16;
using igemm_dev::f16v;
using tok::ceil_div;
using tok::round_up;
using tok::u4;

typedef int i8v __attribute__((ext_vector_type(8)));
typedef int i4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef igemm_dev::bf8 bf8;

constexpr int kThreads = 256;
constexpr int kBlock = 128;            // values of a scale: one step of the contraction
constexpr uint32_t kFar = 0x80000000u;  // an offset beyond every buffer: its 16 bytes arrive as zeros

struct Args {
  const uint8_t *a, *a_scales, *b, *b_scales;
  const float *bias;
  void *out;
  long long ld, out_rs;
  int M, N, K, pitch, s_pitch, steps, b_shift, accumulate;
};

template <typename T>
__device__ __forceinline__ float out_value(const T *p);
template <>
__device__ __forceinline__ float out_value<float>(const float *p) {
  return *p;
}
template <>
__device__ __forceinline__ float out_value<bf16_t>(const bf16_t *p) {
  return bf16_to_f32(*p);
}
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t *p, float v) { *p = f32_to_bf16(v); }

// 64 codes (one row's half step) for a lane: 32 bytes, two of the row's eight 16-byte chunks.  Chunk c of row r lies in slot c ^ (r & 7).
__device__ __forceinline__ i8v fragment(const char *rows, int row, int chunk) {
  const char *p = rows + row * kBlock;
  const i4v lo = *(const i4v *)(p + ((chunk ^ (row & 7)) << 4)), hi = *(const i4v *)(p + (((chunk + 1) ^ (row & 7)) << 4));
  return i8v{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
}

// Eight codes (two dwords) times a power of two, as bf16.
__device__ __forceinline__ bf8 eight_bf16(int lo, int hi, float scale) {
  const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// 2^(byte - 127) of a scale dword's lowest byte
__device__ __forceinline__ float scale_value(int s) { return __uint_as_float(((uint32_t)s & 0xffu) << 23); }

// A tile of BM x BN, WM x WN wavefronts, two steps of the contraction in LDS.
template <typename TO, bool EXACT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN *PARLE_WAVE) void k_fp8_tile(Args g) {
  constexpr int kWaves = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int kStage = (BM + BN) * kBlock;
  constexpr int kLoads = (BM + BN) / 8 / kWaves;  // 1 KiB loads of a wavefront per step: 8 rows each
  __shared__ __attribute__((aligned(1024))) char lds[2 * kStage];
  const int lane = threadIdx.x & (PARLE_WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PARLE_WAVE);
  const int rep = blockIdx.z, m0 = blockIdx.y * BM, n0 = blockIdx.x * BN;
  const uint8_t *a0 = g.a + ((long long)rep * g.M + m0) * g.pitch, *b0 = g.b + ((long long)rep * g.N + n0) * g.pitch;
  const u4 a_desc = buffer_desc(a0, (uint32_t)min((long long)(g.M - m0) * g.pitch, (long long)BM * g.pitch));
  const u4 b_desc = buffer_desc(b0, (uint32_t)min((long long)(g.N - n0) * g.pitch, (long long)BN * g.pitch));
  const int chunk = (lane & 7) ^ (lane >> 3);  // of its row, so that it lands in slot lane & 7
  const uint32_t voff = (uint32_t)(lane >> 3) * (uint32_t)g.pitch + chunk * 16;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

  auto load = [&](int step, int stage) {
    const uint32_t v = step * kBlock + chunk * 16 < g.pitch ? voff : kFar;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = wave * kLoads + i;  // 8 rows of a, then of b
      const bool is_a = piece < BM / 8;
      const uint32_t rows = (is_a ? piece : piece - BM / 8) * 8;
      dma16(__builtin_amdgcn_readfirstlane(lds0 + stage * kStage + piece * 1024), is_a ? a_desc : b_desc, v,
            __builtin_amdgcn_readfirstlane(rows * (uint32_t)g.pitch + step * kBlock));
    }
  };

  const int r = lane & 31, half = lane >> 5;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  const uint8_t *sa[TM], *sb[TN];  // scale rows; those past the end read the last row's and are not stored
#pragma unroll
  for (int t = 0; t < TM; ++t) sa[t] = g.a_scales + ((long long)rep * g.M + min(m0 + wm + t * 32 + r, g.M - 1)) * g.s_pitch;
  const int b_rows = (g.N + (1 << g.b_shift) - 1) >> g.b_shift;
#pragma unroll
  for (int t = 0; t < TN; ++t)
    sb[t] = g.b_scales + ((long long)rep * b_rows + (min(n0 + wn + t * 32 + r, g.N - 1) >> g.b_shift)) * g.s_pitch;

  f16v acc[TM][TN] = {};
  int xa[TM], xb[TN];
  if (g.steps > 0) load(0, 0);
  for (int step = 0; step < g.steps; ++step) {
    if ((step & 3) == 0) {
#pragma unroll
      for (int t = 0; t < TM; ++t) xa[t] = *(const int *)(sa[t] + step);
#pragma unroll
      for (int t = 0; t < TN; ++t) xb[t] = *(const int *)(sb[t] + step);
    }
    igemm_dev::wait_loads<0>();
    __syncthreads();  // this step is in LDS, and everyone has read the step whose place the next one takes
    if (step + 1 < g.steps) load(step + 1, (step + 1) & 1);
    const char *as = lds + (step & 1) * kStage, *bs = as + BM * kBlock;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      i8v fa[TM], fb[TN];
#pragma unroll
      for (int t = 0; t < TM; ++t) fa[t] = fragment(as, wm + t * 32 + r, h * 4 + half * 2);
#pragma unroll
      for (int t = 0; t < TN; ++t) fb[t] = fragment(bs, wn + t * 32 + r, h * 4 + half * 2);
      if (EXACT) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bf8 ea[TM], eb[TN];
#pragma unroll
          for (int t = 0; t < TM; ++t) ea[t] = eight_bf16(fa[t][2 * j], fa[t][2 * j + 1], scale_value(xa[t]));
#pragma unroll
          for (int t = 0; t < TN; ++t) eb[t] = eight_bf16(fb[t][2 * j], fb[t][2 * j + 1], scale_value(xb[t]));
#pragma unroll
          for (int tm = 0; tm < TM; ++tm)
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ea[tm], eb[tn], acc[tm][tn], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
#pragma unroll
          for (int tn = 0; tn < TN; ++tn)
            acc[tm][tn] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa[tm], fb[tn], acc[tm][tn], 0, 0, 0, xa[tm], 0, xb[tn]);
      }
    }
#pragma unroll
    for (int t = 0; t < TM; ++t) xa[t] = (unsigned)xa[t] >> 8;
#pragma unroll
    for (int t = 0; t < TN; ++t) xb[t] = (unsigned)xb[t] >> 8;
  }

  TO *out = (TO *)g.out + rep * g.out_rs;
#pragma unroll
  for (int tn = 0; tn < TN; ++tn) {
    const int n = n0 + wn + tn * 32 + r;
    if (n >= g.N) continue;
    const float bias = g.bias ? g.bias[(long long)rep * g.N + n] : 0.f;
#pragma unroll
    for (int tm = 0; tm < TM; ++tm)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int m = m0 + wm + tm * 32 + 8 * (v >> 2) + 4 * half + (v & 3);
        if (m < g.M) {
          TO *p = out + m * g.ld + n;
          put(p, acc[tm][tn][v] + bias + (g.accumulate ? out_value<TO>(p) : 0.f));
        }
      }
  }
}

template <typename TO>
hipError_t run(hipStream_t st, const parle_fp8_desc &d, const Args &g) {
  const dim3 grid(ceil_div(d.cols, 128), ceil_div(d.rows, 128), d.n);
  k_fp8_tile<TO, sizeof(TO) == 4, 128, 128, 2, 2><<<grid, kThreads, 0, st>>>(g);
  return hipGetLastError();
}

}  // namespace

int64_t fp8_scratch_bytes(const parle_fp8_desc &d) { return 0; }

hipError_t launch_fp8_matmul(hipStream_t st, const parle_fp8_desc &d, const uint8_t *a, const uint8_t *a_scales, const uint8_t *b,
                             const uint8_t *b_scales, const float *bias, float *partial, void *out) {
  Args g;
  g.a = a, g.a_scales = a_scales, g.b = b, g.b_scales = b_scales, g.bias = bias, g.out = out, g.ld = d.ld_out, g.out_rs = d.out_stride;
  g.M = d.rows, g.N = d.cols, g.K = d.depth, g.pitch = (int)round_up(d.depth, 16), g.steps = ceil_div(d.depth, kBlock);
  g.s_pitch = (int)round_up(g.steps, 4), g.b_shift = d.b_block == 1 ? 0 : 7, g.accumulate = d.accumulate;
  return d.out_dtype ? run<bf16_t>(st, d, g) : run<float>(st, d, g);
}
