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
// the rate.  So do the products of up to 16 rows whatever their result, as loads bound them (4 x 8192 x 4096: 10.6 us with the 8-bit
// instructions, 10.9 without).
// (The conversion takes a scale's exponent, 2^-127 too.  Values below 2^-126 become multiples of 2^-133, the smallest bf16 number.)
#include <algorithm>

#include "igemm_dev.h"
#include "tok.h"

namespace {

using igemm_dev::buffer_desc;
using igemm_dev::dma16;
using igemm_dev::dma4;
using igemm_dev::f16v;
using tok::ceil_div;
using tok::round_up;
using tok::u4;

typedef int i8v __attribute__((ext_vector_type(8)));
typedef int i4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef igemm_dev::bf8 bf8;

constexpr int kBlock = 128;            // values of a scale: one step of the contraction
constexpr uint32_t kFar = 0x80000000u;  // an offset beyond every buffer: its 16 bytes arrive as zeros

struct Args {
  const uint8_t *a, *a_scales, *b, *b_scales;
  const float *bias;
  void *out;
  long long ld, out_rs, split_rs;  // split_rs: from the results of one share of the contraction to the next one's
  int M, N, K, pitch, s_pitch, steps, b_shift, accumulate;
  int share;  // steps of a workgroup, a multiple of four where there are more
};

__device__ __forceinline__ float value(const float *p) { return *p; }
__device__ __forceinline__ float value(const bf16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t *p, float v) { *p = f32_to_bf16(v); }

// Eight codes (two dwords) times a power of two, as bf16.
__device__ __forceinline__ bf8 eight_bf16(int lo, int hi, float scale) {
  const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// 2^(byte - 127) of a scale dword's lowest byte, for the conversions: they read the exponent's bits, so that zeros there are 2^-127
__device__ __forceinline__ float scale_value(int s) { return __uint_as_float(((uint32_t)s & 0xffu) << 23); }

// Results of 16 columns from n on, of which the two halves of a wavefront hold four in turn (registers 4 j .. 4 j + 7 of the product):
// the halves exchange, and each lane has eight neighbouring columns, n + 8 half .. + 7.
template <typename TO>
__device__ __forceinline__ void store16(const Args &g, int rep, int m, int n, int half, const f16v *acc, int j, TO *row) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint((*acc)[4 * j + i]), __float_as_uint((*acc)[4 * j + 4 + i]), false, false);
    v[i] = __uint_as_float(x[0]), v[4 + i] = __uint_as_float(x[1]);
  }
  n += 8 * half;
  const int left = g.N - n;
  if (m >= g.M || left <= 0) return;
  if (g.bias) {
    float c[8];
    tok::load8(g.bias + (long long)rep * g.N + n, left, 0.f, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += c[i];
  }
  if (g.accumulate) {
    float o[8];
    tok::load8(row + n, left, 0.f, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += o[i];
  }
  tok::store8(row + n, left, v);
}

// Tile of a workgroup.  Workgroups go to the eight dies in turn, and each die has its own second-level cache: a die gets a
// contiguous share of an order that walks strips of four rows of tiles, column by column, so that the 32 tiles that it works on at a
// time are about four rows by eight columns.
__device__ __forceinline__ void tile_of(int id, int rows, int cols, int &m, int &n) {
  constexpr int kDies = 8, kStrip = 4;
  const int all = rows * cols, share = all / kDies, more = all % kDies, die = id % kDies;
  const int at = die * share + min(die, more) + id / kDies;
  const int strip = at / (kStrip * cols), first = strip * kStrip, height = min(kStrip, rows - first), in = at - first * cols;
  m = first + in % height, n = in / height;
}

// A tile of BM x BN, WM x WN wavefronts.  STAGES steps of the contraction (128 codes of every row) lie in LDS; a wavefront holds the
// fragments of one step in registers, in two halves.  Once all have theirs of step s, half of its products are made, step s + 1 has
// arrived, and one barrier says both: step s + STAGES may be loaded over step s, and the fragments of s + 1 are read while the matrix
// units work on the other half.  Loads, reads and products are interleaved by hand and pinned: left alone, the compiler moves all
// products of a step behind its reads.
// 8192 x 8192 x 4096 (bf16 result): 413 us with tiles of 128 x 128 and no overlap, 302 with 256 x 256 pipelined, 242 with results stored in
// 16 bytes a lane, scales through LDS and two wavefronts on a SIMD, each with 128 x 64 of the tile; 220 on operands that the caches
// hold, 2.5 PFLOP/s: the matrix units are busy 73 % of the time at the 1.6 GHz that the power limit leaves, LDS bank conflicts (reads of
// scales) 3 %.  A fp32 result: 407 us, 1.35 PFLOP/s.  A loop over tiles in one workgroup, its loads running into the next tile, gained nothing: the
// wait for loads waits for the last tile's stores as well.
template <typename TO, bool EXACT, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM *WN *PARLE_WAVE) void k_fp8_tile(Args g) {
  constexpr int kWaves = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int kRows = BM + BN, kStage = kRows * kBlock;
  constexpr int kLoads = (BM + BN) / 8 / kWaves;  // 1 KiB loads of a wavefront per step: 8 rows each
  extern __shared__ __attribute__((aligned(1024))) char lds[];  // the stages, then scales of twice sixteen steps, then what is touched
  const int lane = threadIdx.x & (PARLE_WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PARLE_WAVE);
  int tile_m, tile_n;
  tile_of(blockIdx.x, ceil_div(g.M, BM), ceil_div(g.N, BN), tile_m, tile_n);
  const int rep = blockIdx.z, m0 = tile_m * BM, n0 = tile_n * BN;
  const uint8_t *a0 = g.a + ((long long)rep * g.M + m0) * g.pitch, *b0 = g.b + ((long long)rep * g.N + n0) * g.pitch;
  const u4 a_desc = buffer_desc(a0, (uint32_t)min((long long)(g.M - m0) * g.pitch, (long long)BM * g.pitch));
  const u4 b_desc = buffer_desc(b0, (uint32_t)min((long long)(g.N - n0) * g.pitch, (long long)BN * g.pitch));
  // Chunk c (16 codes) of row r lies in slot c ^ (r / 2 & 7) of the row's 128 bytes: a read of one chunk of 16 neighbouring rows then
  // touches every bank once.  A load brings 8 rows; lane l fills slot l & 7 of row l / 8, in the lower or the upper half of 16 rows.
  const int c_even = (lane & 7) ^ (lane >> 4), c_odd = c_even ^ 4;
  const uint32_t voff = (uint32_t)(lane >> 3) * (uint32_t)g.pitch;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

  // piece i of a wavefront's loads of a step
  auto load = [&](int stage, int step, int i) {
    const int piece = wave * kLoads + i;  // 8 rows of a, then of b
    const int k = step * kBlock, c = (kLoads % 2 ? piece : i) & 1 ? c_odd : c_even;
    const bool is_a = piece < BM / 8;
    const uint32_t rows = (is_a ? piece : piece - BM / 8) * 8;
    dma16(__builtin_amdgcn_readfirstlane(lds0 + stage + piece * 1024), is_a ? a_desc : b_desc,
          k + c * 16 < g.pitch ? voff + c * 16 : kFar, __builtin_amdgcn_readfirstlane(rows * (uint32_t)g.pitch + k));
  };
  // The first workgroup that needs a line waits for memory, longer than a step of 1.2 us takes, and its neighbours with it.  So lines are
  // touched a step before they are loaded, a lane for a line, into 256 bytes per wavefront that nobody reads: of a's rows a quarter by
  // each of four tiles side by side, of b's by each of four one below the other, which run on this die at the same time.  8192 x
  // 8192 x 4096 on operands that no cache holds: 254 -> 228 us (ahead by 2 or 3 steps 230, 231).  Three stages, or the longer steps of an
  // fp32 result, have the time without it, and lose 2 %.
  constexpr int kTouch = kWaves == 8 && STAGES == 2 && !EXACT, kTouchAhead = 1;
  auto touch = [&](int step) {
    if (!kTouch) return;
    const bool is_a = wave < kWaves / 2;
    const int each = (is_a ? BM : BN) / 4 / (kWaves / 2), first = ((is_a ? tile_n : tile_m) & 3) * ((is_a ? BM : BN) / 4) + wave % (kWaves / 2) * each;
    dma4(__builtin_amdgcn_readfirstlane(lds0 + STAGES * kStage + 32 * kRows + wave * 256), is_a ? a_desc : b_desc,
         lane < each && step < g.steps ? (uint32_t)(first + lane) * (uint32_t)g.pitch + step * kBlock : kFar);
  };
  // Scales of sixteen steps, 16 bytes per row of the tile: 64 rows for a wavefront's load, in turn.
  constexpr int kScaleLoads = kRows / PARLE_WAVE;
  const int b_rows = (g.N + (1 << g.b_shift) - 1) >> g.b_shift, b_row0 = n0 >> g.b_shift;
  const u4 sa_desc = buffer_desc(g.a_scales + ((long long)rep * g.M + m0) * g.s_pitch, (uint32_t)(min(BM, g.M - m0) * g.s_pitch));
  const u4 sb_desc =
      buffer_desc(g.b_scales + ((long long)rep * b_rows + b_row0) * g.s_pitch, (uint32_t)(min(BN, b_rows - b_row0) * g.s_pitch));
  auto load_scales = [&](int first) {
#pragma unroll
    for (int i = 0; i < (kScaleLoads + kWaves - 1) / kWaves; ++i) {
      const int p = (i * kWaves + wave) % kScaleLoads;
      const bool is_a = p < BM / PARLE_WAVE;
      const int row = (is_a ? p : p - BM / PARLE_WAVE) * PARLE_WAVE + lane;
      const int at = is_a ? row : ((n0 + row) >> g.b_shift) - b_row0;
      dma16(__builtin_amdgcn_readfirstlane(lds0 + STAGES * kStage + (first & 16) * kRows + p * PARLE_WAVE * 16), is_a ? sa_desc : sb_desc,
            first < g.s_pitch ? (uint32_t)(at * g.s_pitch + first) : kFar, 0);
    }
  };
  static_assert((BM + BN) % (8 * kWaves) == 0 && BM % 16 == 0, "whole pieces for every wavefront, that alternate between halves of 16 rows");

  const int r = lane & 31, half = lane >> 5;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
  f16v acc[TM][TN] = {};
  int xa[TM], xb[TN];  // scales of the step, in the lowest byte
  auto take_scales = [&](int first) {
    const int *p = (const int *)(lds + STAGES * kStage + (first & 16) * kRows) + r * 4 + (first >> 2 & 3);
#pragma unroll
    for (int t = 0; t < TM; ++t) xa[t] = p[(wm + t * 32) * 4];
#pragma unroll
    for (int t = 0; t < TN; ++t) xb[t] = p[(BM + wn + t * 32) * 4];
  };

  // 64 codes of a row for two lanes: chunks 4 h + 2 half and the one behind it
  i8v fa[2][TM], fb[2][TN];
  const int slot = (half * 2) ^ ((r >> 1) & 7);
  // fragment t of a half step: of a, then of b
  auto read = [&](int stage, int h, int t) {
    const char *q = lds + stage + (r + (t < TM ? wm + t * 32 : BM + wn + (t - TM) * 32)) * kBlock;
    const int lo = (slot ^ (h * 4)) * 16, hi = lo ^ 16;
    const i4v x = *(const i4v *)(q + lo), y = *(const i4v *)(q + hi);
    (t < TM ? fa[h][t] : fb[h][t - TM]) = i8v{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  };
  // the products of a half step; between(i) is issued behind product i
  auto multiply = [&](int h, const auto &between) {
    if (EXACT) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf8 ea[TM], eb[TN];
#pragma unroll
        for (int t = 0; t < TM; ++t) ea[t] = eight_bf16(fa[h][t][2 * j], fa[h][t][2 * j + 1], scale_value(xa[t]));
#pragma unroll
        for (int t = 0; t < TN; ++t) eb[t] = eight_bf16(fb[h][t][2 * j], fb[h][t][2 * j + 1], scale_value(xb[t]));
#pragma unroll
        for (int tm = 0; tm < TM; ++tm)
#pragma unroll
          for (int tn = 0; tn < TN; ++tn) {
            acc[tm][tn] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eb[tn], ea[tm], acc[tm][tn], 0, 0, 0);
            if (j == 0) between(tm * TN + tn);
          }
      }
    } else {
#pragma unroll
      for (int tm = 0; tm < TM; ++tm)
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) {
          acc[tm][tn] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[h][tn], fa[h][tm], acc[tm][tn], 0, 0, 0, xb[tn], 0, xa[tm]);
          __builtin_amdgcn_sched_barrier(0);
          between(tm * TN + tn);
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  };
  constexpr int kProducts = TM * TN, kFrags = TM + TN;
  // share i of n pieces of work among the products of a half step, done by `last` products
  auto share = [&](int i, int n, int last, const auto &work) {
#pragma unroll
    for (int w = 0; w < n; ++w)
      if (w * last / n == i) work(w);
  };

  // Loads and reads past the last step bring zeros that nothing uses: the loop's body has no branch that the products could be moved
  // across.
  const int from = blockIdx.y * g.share, to = min(from + g.share, g.steps);
  load_scales(from & ~15);
#pragma unroll
  for (int p = 0; p < STAGES; ++p)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(p * kStage, from + p, i);
  touch(from + STAGES);
  igemm_dev::wait_loads<(STAGES - 1) * kLoads + kTouch>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int t = 0; t < kFrags; ++t) read(0, 0, t);
  int here = 0;  // the step's stage
  for (int first = from; first < to; first += 4) {
    take_scales(first);
    if (first == from || (first & 15) == 0) load_scales((first & ~15) + 16);  // over those of the sixteen before, which everyone has taken
    const int last = min(first + 4, to);
    for (int step = first; step < last; ++step) {
      const int next = here == (STAGES - 1) * kStage ? 0 : here + kStage;
      multiply(0, [&](int i) { share(i, kFrags, kProducts / 2, [&](int t) { read(here, 1, t); }); });
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * (kLoads + kTouch) + kTouch) : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      multiply(1, [&](int i) {
        share(i, kFrags, kProducts, [&](int t) { read(next, 0, t); });
        share(i, kLoads, kProducts, [&](int p) { load(here, step + STAGES, p); });
        if (i == kProducts - 1) touch(step + STAGES + kTouchAhead);
      });
      __builtin_amdgcn_sched_barrier(0);
      here = next;
#pragma unroll
      for (int t = 0; t < TM; ++t) xa[t] = (unsigned)xa[t] >> 8;
#pragma unroll
      for (int t = 0; t < TN; ++t) xb[t] = (unsigned)xb[t] >> 8;
    }
  }
  igemm_dev::wait_loads<0>();

  // A lane has row m = its r of a 32 x 32 product, columns 8 j + 4 half .. + 3 in registers 4 j .. 4 j + 3.
  TO *out = (TO *)g.out + rep * g.out_rs + blockIdx.y * g.split_rs;
#pragma unroll
  for (int tm = 0; tm < TM; ++tm) {
    const int m = m0 + wm + tm * 32 + r;
    TO *row = out + m * g.ld;
#pragma unroll
    for (int tn = 0; tn < TN; ++tn)
#pragma unroll
      for (int j = 0; j < 4; j += 2) store16<TO>(g, rep, m, n0 + wn + tn * 32 + j * 8, half, &acc[tm][tn], j, row);
  }
}

// Up to 16 rows of a: what counts is reading b once, at the rate of memory (4 x 8192 x 4096: 9.6 us, 3.5 TB/s; a tile of 128 rows took 30).  A wavefront multiplies 16 rows of b with all of a over its
// share of the contraction, straight from memory into fragments and with no barrier; SPLIT wavefronts of a workgroup share a group of 16
// rows of b and add their parts in LDS, in order.
constexpr int kRowsWaves = 8;

template <typename TO, int SPLIT>
__global__ __launch_bounds__(kRowsWaves *PARLE_WAVE) void k_fp8_rows(Args g) {
  constexpr int kAhead = 4;  // steps whose loads are on their way together
  __shared__ f4 part[kRowsWaves][PARLE_WAVE];
  const int lane = threadIdx.x & (PARLE_WAVE - 1), r = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PARLE_WAVE), share = wave % SPLIT;
  const int rep = blockIdx.y, n0 = (blockIdx.x * (kRowsWaves / SPLIT) + wave / SPLIT) * 16;
  const int b_rows = (g.N + (1 << g.b_shift) - 1) >> g.b_shift, n = min(n0 + r, g.N - 1);  // rows past the end are not stored
  const uint8_t *b = g.b + ((long long)rep * g.N + n) * g.pitch, *sb = g.b_scales + ((long long)rep * b_rows + (n >> g.b_shift)) * g.s_pitch;
  const long long m = (long long)rep * g.M + min(r, g.M - 1);
  const uint8_t *a = g.a + m * g.pitch, *sa = g.a_scales + m * g.s_pitch;
  // 32 of a step's 128 codes of a row: chunks `quarter` and `quarter` + 4, so that four lanes read 64 bytes side by side
  const auto codes = [&](const uint8_t *p, int k) {
    const int at = k + quarter * 16;
    const i4v zero = {0, 0, 0, 0}, x = at < g.pitch ? *(const i4v *)(p + at) : zero, y = at + 64 < g.pitch ? *(const i4v *)(p + at + 64) : zero;
    return i8v{x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  };
  f4 acc = {0.f, 0.f, 0.f, 0.f};
  const int each = (g.steps + SPLIT - 1) / SPLIT, last = min((share + 1) * each, g.steps);
  for (int step = share * each; step < last; step += kAhead) {
    i8v fb[kAhead], fa[kAhead];
    int xb[kAhead], xa[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (step + u >= last) break;
      fb[u] = codes(b, (step + u) * kBlock), xb[u] = sb[step + u];
      fa[u] = codes(a, (step + u) * kBlock), xa[u] = sa[step + u];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (step + u >= last) break;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(eight_bf16(fb[u][2 * j], fb[u][2 * j + 1], scale_value(xb[u])),
                                                      eight_bf16(fa[u][2 * j], fa[u][2 * j + 1], scale_value(xa[u])), acc, 0, 0, 0);
    }
  }
  if (SPLIT > 1) {
    part[wave][lane] = acc;
    __syncthreads();
    if (share != 0) return;
#pragma unroll
    for (int w = 1; w < SPLIT; ++w) acc += part[wave + w][lane];
  }
  // a lane has row m = lane & 15 of a, columns 4 (lane / 16) .. + 3 of the group
  if (r >= g.M) return;
  TO *out = (TO *)g.out + rep * g.out_rs + r * g.ld;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int col = n0 + quarter * 4 + i;
    if (col < g.N) put(out + col, acc[i] + (g.bias ? g.bias[(long long)rep * g.N + col] : 0.f) + (g.accumulate ? value(out + col) : 0.f));
  }
}

// Adds the shares of the contraction, in order: out = their sum + bias (+ out).  grid: (vectors of a row's, rows, replicas)
template <typename TO>
__global__ __launch_bounds__(256) void k_fp8_join(const float *part, int splits, Args g) {
  const int n = (blockIdx.x * 256 + threadIdx.x) * tok::kVec, left = g.N - n, rep = blockIdx.z;
  if (left <= 0) return;
  for (int m = blockIdx.y; m < g.M; m += gridDim.y) {
    float v[tok::kVec] = {};
    if (g.bias) tok::load8(g.bias + (long long)rep * g.N + n, left, 0.f, v);
    const float *p = part + ((long long)rep * g.M + m) * g.N + n;
    const long long step = (long long)gridDim.z * g.M * g.N;
    for (int s = 0; s < splits; s += 2) {  // an even number of shares
      tok::Raw8<float> u, w;
      u.load(p + s * step, left), w.load(p + (s + 1) * step, left);
#pragma unroll
      for (int i = 0; i < tok::kVec; ++i) v[i] = (v[i] + u.at(i)) + w.at(i);
    }
    TO *to = (TO *)g.out + rep * g.out_rs + m * g.ld + n;
    if (g.accumulate) {
      float o[tok::kVec];
      tok::load8(to, left, 0.f, o);
#pragma unroll
      for (int i = 0; i < tok::kVec; ++i) v[i] += o[i];
    }
    tok::store8(to, left, v);
  }
}

template <typename TO, bool EXACT, int BM, int BN, int WM, int WN, int STAGES>
hipError_t run_tile(hipStream_t st, const Args &g, int replicas, int splits = 1) {
  constexpr int kLds = (BM + BN) * (STAGES * kBlock + 2 * 16) + WM * WN * 256;
  static const hipError_t lds_ok =
      hipFuncSetAttribute((const void *)k_fp8_tile<TO, EXACT, BM, BN, WM, WN, STAGES>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  if (lds_ok != hipSuccess) return lds_ok;
  const dim3 grid(ceil_div(g.N, BN) * ceil_div(g.M, BM), splits, replicas);
  k_fp8_tile<TO, EXACT, BM, BN, WM, WN, STAGES><<<grid, WM * WN * PARLE_WAVE, kLds, st>>>(g);
  return hipGetLastError();
}

template <typename TO, int SPLIT>
hipError_t run_rows(hipStream_t st, const Args &g, int replicas) {
  const dim3 grid(ceil_div(g.N, 16 * (kRowsWaves / SPLIT)), replicas);
  k_fp8_rows<TO, SPLIT><<<grid, kRowsWaves * PARLE_WAVE, 0, st>>>(g);
  return hipGetLastError();
}

// What a tiling takes, in microseconds: the start and end of a tile, and a step of it with one or two tiles on a compute unit (two: 0
// where one fills it).  Measured at 8192 x 8192 x 4096, 2050 x 4000 x 1024, 2050 x 1024 x 4000, 4000 x 1024 x 2050 (three replicas) and
// 128 x 8192 x 4096: what decides is how many rounds of tiles there are and how full the last one is.  bf16 and fp32 results.
struct Tiling {
  int bm, bn;
  float start, one[2], two[2];
  float cost(const parle_fp8_desc &d, int splits) const {
    const int steps = ceil_div(d.depth, kBlock), share = splits > 1 ? (int)round_up(ceil_div(steps, splits), 4) : steps, wide = d.out_dtype ? 0 : 1;
    const long long tiles = (long long)ceil_div(d.rows, bm) * ceil_div(d.cols, bn) * d.n * splits, each = (tiles + 255) / 256;
    const float single = start + one[wide] * (float)share, pair = start + two[wide] * (float)share;
    const float join = splits > 1 ? 3.f + (float)d.n * d.rows * d.cols * (8.f * splits + 4.f) / 4e6f : 0.f;
    return join + (two[0] == 0.f ? (float)each * single : (float)(each / 2) * pair + (float)(each % 2) * single);
  }
};
constexpr Tiling kTilings[] = {{256, 256, 5.5f, {1.5f, 3.2f}, {0.f, 0.f}},
                               {192, 256, 5.5f, {1.3f, 2.7f}, {0.f, 0.f}},
                               {128, 256, 5.5f, {0.95f, 1.75f}, {0.f, 0.f}},
                               {128, 128, 4.f, {0.65f, 1.f}, {1.1f, 1.7f}},
                               {64, 64, 3.f, {0.25f, 0.4f}, {0.5f, 0.65f}}};
constexpr int kSmallest = 4;

constexpr int kFewRows = 16;

struct Plan {
  int tiling, splits;
};
// The tiling that takes least; the contraction of the smallest one may be shared, where the whole product is a few tiles.
Plan plan_of(const parle_fp8_desc &d) {
  Plan best = {0, 1};
  float least = kTilings[0].cost(d, 1);
  const auto consider = [&](int tiling, int splits) {
    const float c = kTilings[tiling].cost(d, splits);
    if (c < least) least = c, best = Plan{tiling, splits};
  };
  for (int i = 1; i <= kSmallest; ++i) consider(i, 1);
  for (int splits = 2; splits <= 8; splits *= 2)
    if (ceil_div(d.depth, kBlock) >= 4 * splits) consider(kSmallest, splits);
  return best;
}

template <typename TO>
hipError_t run(hipStream_t st, const parle_fp8_desc &d, Args g, float *partial) {
  constexpr bool kExact = sizeof(TO) == 4;
  if (g.M <= kFewRows) {
    // four steps at least for a wavefront, and no fewer wavefronts than eight for 16 rows of b
    if (g.steps >= 32) return run_rows<TO, 8>(st, g, d.n);
    if (g.steps >= 16) return run_rows<TO, 4>(st, g, d.n);
    if (g.steps >= 8) return run_rows<TO, 2>(st, g, d.n);
    return run_rows<TO, 1>(st, g, d.n);
  }
  const Plan p = plan_of(d);
  if (p.splits > 1) {
    Args part = g;
    part.out = partial, part.ld = g.N, part.out_rs = (long long)g.M * g.N, part.split_rs = part.out_rs * d.n;
    part.bias = nullptr, part.accumulate = 0, part.share = (int)round_up(ceil_div(g.steps, p.splits), 4);
    const hipError_t e = run_tile<float, kExact, 64, 64, 2, 2, 4>(st, part, d.n, p.splits);
    if (e != hipSuccess) return e;
    k_fp8_join<TO><<<dim3(ceil_div(g.N, 256 * tok::kVec), std::min(g.M, 1024), d.n), 256, 0, st>>>(partial, p.splits, g);
    return hipGetLastError();
  }
  switch (p.tiling) {
    case 0: return run_tile<TO, kExact, 256, 256, 2, 4, 2>(st, g, d.n);
    case 1: return run_tile<TO, kExact, 192, 256, 2, 4, 2>(st, g, d.n);
    case 2: return run_tile<TO, kExact, 128, 256, 2, 4, 3>(st, g, d.n);
    case 3: return run_tile<TO, kExact, 128, 128, 2, 2, 2>(st, g, d.n);
    default: return run_tile<TO, kExact, 64, 64, 2, 2, 4>(st, g, d.n);
  }
}

}  // namespace

int64_t fp8_scratch_bytes(const parle_fp8_desc &d) {
  if (d.rows <= kFewRows) return 0;
  const int splits = plan_of(d).splits;
  return splits > 1 ? (int64_t)splits * d.n * d.rows * d.cols * 4 : 0;
}

hipError_t launch_fp8_matmul(hipStream_t st, const parle_fp8_desc &d, const uint8_t *a, const uint8_t *a_scales, const uint8_t *b,
                             const uint8_t *b_scales, const float *bias, float *partial, void *out) {
  Args g;
  g.a = a, g.a_scales = a_scales, g.b = b, g.b_scales = b_scales, g.bias = bias, g.out = out, g.ld = d.ld_out, g.out_rs = d.out_stride;
  g.M = d.rows, g.N = d.cols, g.K = d.depth, g.pitch = (int)round_up(d.depth, 16), g.steps = ceil_div(d.depth, kBlock);
  g.s_pitch = (int)round_up(g.steps, 4), g.b_shift = d.b_block == 1 ? 0 : 7, g.accumulate = d.accumulate, g.share = g.steps, g.split_rs = 0;
  return d.out_dtype ? run<bf16_t>(st, d, g, partial) : run<float>(st, d, g, partial);
}
