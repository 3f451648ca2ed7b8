// 8-bit codes and power-of-two scales of a matrix and of its transpose, from one read.
//
// A workgroup takes a 128 x 128 tile: it is what shares a scale (block 128), or holds whole scale blocks in both directions
// (block 1: 128 values of a row, and 128 of a column for the transpose).  A thread holds 8 x 8 neighbouring values in registers: largest
// magnitudes go over lanes and through a little LDS, rows of codes are written from where they are, and columns pass through LDS as
// bytes, eight rows of a column at a time, so that a tile takes 17 KiB and rows of both results leave in whole lines of 128 bytes.
// The vector unit is what bounds it, so bf16 values stay in pairs: magnitudes are compared as 16-bit integers, two at a time, and the
// conversion takes pairs and the scale.  Tiles that hold NaN, infinities or magnitudes below 2^-118 go value by value through memory
// instead, in as little code as it takes: a workgroup runs through the kernel once, and waits for what it has to fetch of it.
// Both orders of 3 x 2050 x 4000 bf16 (98 MB): 58 us with fp32 in LDS, 42 with bytes, 35 with pairs, 29 with short code, 3.4 TB/s; of
// 3 x 4000 x 1024 fp32 parameters: 17 us, 4.3 TB/s.  What is left is a tile's chain of loads, exchange, codes, exchange and stores.
#include "tok.h"

namespace {

using namespace tok;

constexpr int kThreads = 256, kWaves = kThreads / PARLE_WAVE, kTile = 128;
constexpr int kPitch = kTile + 8;  // bytes of a column of codes in LDS: eight lanes apart, columns begin 16 banks apart

struct Args {
  uint8_t *q, *scales, *qt, *scales_t;
  long long ld, stride;
  int rows, cols;
  int pitch, s_pitch, pitch_t, s_pitch_t;  // of codes and scales, and of the transpose's
};

// The 8 x 8 values of a thread.
template <typename T>
struct Values;

template <>
struct Values<float> {
  float v[kVec][kVec];
  __device__ __forceinline__ void load(int j, const float *p) { load8(p, kVec, 0.f, v[j]); }
  __device__ __forceinline__ void load(int j, const float *p, int count) { load8(p, count, 0.f, v[j]); }
  // Row j without its first `skip` values, zeros behind.
  __device__ __forceinline__ void shift(int j, int skip) {
#pragma unroll
    for (int s = 1; s <= kVec; s *= 2)
      if (skip & s || (s == kVec && skip > s)) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[j][i] = i + s < kVec ? v[j][i + s] : 0.f;
      }
  }
  __device__ __forceinline__ float at(int j, int i) const { return v[j][i]; }
  // Bits of the largest magnitudes, of row j and of the columns.
  __device__ __forceinline__ uint32_t row_most(int j) const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = max(m, __float_as_uint(v[j][i]) & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ void col_most(uint32_t (&m)[kVec]) const {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      m[i] = 0;
#pragma unroll
      for (int j = 0; j < kVec; ++j) m[i] = max(m[i], __float_as_uint(v[j][i]) & 0x7fffffffu);
    }
  }
  __device__ __forceinline__ u2 row_codes(int j, float s) const {
    return u2{codes4_of(v[j][0], v[j][1], v[j][2], v[j][3], s), codes4_of(v[j][4], v[j][5], v[j][6], v[j][7], s)};
  }
  __device__ __forceinline__ u2 col_codes(int i, float s) const {
    return u2{codes4_of(v[0][i], v[1][i], v[2][i], v[3][i], s), codes4_of(v[4][i], v[5][i], v[6][i], v[7][i], s)};
  }
};

template <>
struct Values<bf16_t> {
  typedef unsigned short us2 __attribute__((ext_vector_type(2)));
  u4 row[kVec];  // pairs of columns
  __device__ __forceinline__ void load(int j, const bf16_t *p) { row[j] = __builtin_bit_cast(u4, (us8)*(const us8_any *)p); }
  __device__ __forceinline__ void load(int j, const bf16_t *p, int count) {
    us8 x;
#pragma unroll
    for (int i = 0; i < kVec; ++i) x[i] = i < count ? p[i] : (bf16_t)0;
    row[j] = __builtin_bit_cast(u4, x);
  }
  __device__ __forceinline__ void shift(int j, int skip) {
    if (skip & 1) row[j] = u4{row[j][0] >> 16 | row[j][1] << 16, row[j][1] >> 16 | row[j][2] << 16, row[j][2] >> 16 | row[j][3] << 16, row[j][3] >> 16};
    if (skip & 2) row[j] = u4{row[j][1], row[j][2], row[j][3], 0};
    if (skip & 4) row[j] = u4{row[j][2], row[j][3], 0, 0};
    if (skip >= kVec) row[j] = u4{0, 0, 0, 0};
  }
  __device__ __forceinline__ float at(int j, int i) const { return __uint_as_float(i & 1 ? row[j][i / 2] & 0xffff0000u : row[j][i / 2] << 16); }
  static __device__ __forceinline__ uint32_t most2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
  }
  __device__ __forceinline__ uint32_t pair(int j, int k) const { return row[j][k] & 0x7fff7fffu; }
  __device__ __forceinline__ uint32_t row_most(int j) const {
    const uint32_t m = most2(most2(pair(j, 0), pair(j, 1)), most2(pair(j, 2), pair(j, 3)));
    return max(m << 16, m & 0xffff0000u);
  }
  __device__ __forceinline__ void col_most(uint32_t (&m)[kVec]) const {
#pragma unroll
    for (int k = 0; k < kVec / 2; ++k) {
      uint32_t x = pair(0, k);
#pragma unroll
      for (int j = 1; j < kVec; ++j) x = most2(x, pair(j, k));
      m[2 * k] = x << 16, m[2 * k + 1] = x & 0xffff0000u;
    }
  }
  __device__ __forceinline__ u2 row_codes(int j, float s) const { return u2{codes4_of(row[j][0], row[j][1], s), codes4_of(row[j][2], row[j][3], s)}; }
  __device__ __forceinline__ uint32_t down(int j, int i) const {  // column i of rows j, j + 1
    return __builtin_amdgcn_perm(row[j + 1][i / 2], row[j][i / 2], i & 1 ? 0x07060302 : 0x05040100);
  }
  __device__ __forceinline__ u2 col_codes(int i, float s) const { return u2{codes4_of(down(0, i), down(2, i), s), codes4_of(down(4, i), down(6, i), s)}; }
};

// Block `at` of a row of scales; the last of `blocks` also clears the row's padding.
__device__ __forceinline__ void put_scale(uint8_t *row, int at, int blocks, int pitch, uint32_t byte) {
  row[at] = (uint8_t)byte;
  if (at == blocks - 1)
#pragma unroll 1
    for (int k = blocks; k < pitch; ++k) row[k] = 0;
}

__device__ __forceinline__ float element(const float *p) { return *p; }
__device__ __forceinline__ float element(const bf16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ uint8_t code_of(float v, float inv) { return (uint8_t)(codes4(scaled(v, inv), 0.f, 0.f, 0.f) & 0xff); }

// A tile with special magnitudes: lines of the tile (rows, then columns) one to a thread, value by value from memory.  from: the tile's
// first value; rows, cols: what the tile holds.
template <typename T, bool ROWS>
__device__ __forceinline__ void slow_tile(const T *from, const Args &a, int rep, int rows, int cols, uint32_t *most_of) {
  const int r0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile;
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {  // the rows of q, the rows of qt
    const int lines = turn ? cols : rows, len = turn ? rows : cols, t = threadIdx.x;
    const long long line_step = turn ? 1 : a.ld, step = turn ? a.ld : 1;
    uint32_t most = 0;
    if (t < lines)
#pragma unroll 1
      for (int i = 0; i < len; ++i) most = max(most, finite_bits(element(from + t * line_step + i * step)));
    if (!ROWS) {
      __syncthreads();
      if (t < kTile) most_of[t] = most;
      __syncthreads();
#pragma unroll 1
      for (int i = 0; i < kTile; ++i) most = max(most, most_of[i]);
    }
    uint8_t *codes = turn ? a.qt : a.q, *scales = turn ? a.scales_t : a.scales;
    const int pitch = turn ? a.pitch_t : a.pitch, s_pitch = turn ? a.s_pitch_t : a.s_pitch;
    const int first = turn ? c0 : r0, at = turn ? r0 : c0, all = turn ? a.cols : a.rows;
    const int block = turn ? blockIdx.y : blockIdx.x, blocks = turn ? gridDim.y : gridDim.x, line_blocks = turn ? gridDim.x : gridDim.y;
    if (!codes || t >= lines) continue;
    const uint32_t byte = scale_byte(most);
    uint8_t *to = codes + ((long long)rep * all + first + t) * pitch + at;
#pragma unroll 1
    for (int i = 0; i < min(kTile, pitch - at); ++i)
      to[i] = i < len ? code_of(element(from + t * line_step + i * step), scale_inverse(byte)) : 0;
    if (ROWS)
      put_scale(scales + ((long long)rep * all + first + t) * s_pitch, block, blocks, s_pitch, byte);
    else if (t == 0)
      put_scale(scales + ((long long)rep * line_blocks + first / kTile) * s_pitch, block, blocks, s_pitch, byte);
  }
}

// grid: (column tiles, row tiles, n).  Thread: columns 8 lane16 .. + 7, rows 8 group .. + 7 of the tile.
template <typename T, bool ROWS>
__global__ __launch_bounds__(kThreads) void k_fp8_quantize(const T *src, Args a) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[kTile * kPitch];
  __shared__ uint32_t most_of[kWaves][kTile];
  const int r0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile, rep = blockIdx.z;
  const int lane16 = threadIdx.x & 15, group = threadIdx.x >> 4, wave = threadIdx.x / PARLE_WAVE;
  const int c = c0 + lane16 * kVec, r = r0 + group * kVec;
  Values<T> x;
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const T *row = src + rep * a.stride + (long long)min(r + j, a.rows - 1) * a.ld;
    if (a.cols >= kVec)
      x.load(j, row + min(c, a.cols - kVec));
    else
      x.load(j, row, c == 0 ? a.cols : 0);
  }
  // Behind the matrix are zeros.  Whatever loads got there is put right afterwards: a guard splits the wavefront, and each load waits
  // for the one before.
  const int skip = a.cols >= kVec ? max(0, c - (a.cols - kVec)) : 0;
  if (skip > 0) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) x.shift(j, skip);
  }
  if (r + kVec > a.rows) {
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      if (r + j >= a.rows) x.shift(j, kVec);
  }
  // largest magnitudes: of rows over 16 lanes, of columns over the groups of a wavefront, then over wavefronts
  uint32_t row_most[kVec], col_most[kVec], tile_most = 0;
  bool special = false;
#pragma unroll
  for (int j = 0; j < kVec; ++j) row_most[j] = x.row_most(j);
  if (ROWS) {
    x.col_most(col_most);
#pragma unroll
    for (int j = 0; j < kVec; ++j) row_most[j] = row_max16(row_most[j]), special |= special_most(row_most[j]);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      uint32_t m = col_most[i];
      m = max(m, (uint32_t)__shfl_xor((int)m, 16, PARLE_WAVE));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32, PARLE_WAVE));
      if ((threadIdx.x & 48) == 0) most_of[wave][lane16 * kVec + i] = m;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = max(m, most_of[w][lane16 * kVec + i]);
      col_most[i] = m;
      special |= special_most(m);
    }
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kVec; ++j) m = max(m, row_most[j]);
    m = row_max16(m);
    if (lane16 == 0) most_of[0][group] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 16; ++w) m = max(m, most_of[0][w]);
    tile_most = m, special = special_most(m);
  }
  if (__syncthreads_or(special)) {
    slow_tile<T, ROWS>(src + rep * a.stride + r0 * a.ld + c0, a, rep, min(kTile, a.rows - r0), min(kTile, a.cols - c0), most_of[0]);
    return;
  }
  const uint32_t byte = scale_byte(tile_most);  // of the whole tile
  if (a.q && c < a.pitch) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      if (r + j >= a.rows) break;
      const uint32_t sb = ROWS ? scale_byte(row_most[j]) : byte;
      *(u2 *)(a.q + ((long long)rep * a.rows + r + j) * a.pitch + c) = x.row_codes(j, scale_float(sb));
    }
  }
  if (ROWS && a.q) {  // lane j of 16 writes row j's scale
    uint32_t m = row_most[0];
#pragma unroll
    for (int j = 1; j < kVec; ++j) m = lane16 == j ? row_most[j] : m;
    if (lane16 < kVec && r + lane16 < a.rows)
      put_scale(a.scales + ((long long)rep * a.rows + r + lane16) * a.s_pitch, blockIdx.x, gridDim.x, a.s_pitch, scale_byte(m));
  }
  if (!ROWS && a.q && threadIdx.x == 0)
    put_scale(a.scales + ((long long)rep * gridDim.y + blockIdx.y) * a.s_pitch, blockIdx.x, gridDim.x, a.s_pitch, byte);
  if (!a.qt) return;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const uint32_t sb = ROWS ? scale_byte(col_most[i]) : byte;
    *(u2 *)(turned + (lane16 * kVec + i) * kPitch + group * kVec) = x.col_codes(i, scale_float(sb));
  }
  if (ROWS) {
    const int t = threadIdx.x;
    if (t < kTile && c0 + t < a.cols) {
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = max(m, most_of[w][t]);
      put_scale(a.scales_t + ((long long)rep * a.cols + c0 + t) * a.s_pitch_t, blockIdx.y, gridDim.y, a.s_pitch_t, scale_byte(m));
    }
  } else if (threadIdx.x == 0) {
    put_scale(a.scales_t + ((long long)rep * gridDim.x + blockIdx.x) * a.s_pitch_t, blockIdx.y, gridDim.y, a.s_pitch_t, byte);
  }
  __syncthreads();
  // eight lanes write the 128 bytes of a row of the transpose
  const int piece = (threadIdx.x & 7) * 16;
#pragma unroll
  for (int j = 0; j < kTile / 32; ++j) {
    const int row = j * 32 + (threadIdx.x >> 3);
    if (c0 + row >= a.cols || r0 + piece >= a.pitch_t) continue;
    const u2 lo = *(const u2 *)(turned + row * kPitch + piece), hi = *(const u2 *)(turned + row * kPitch + piece + 8);
    *(u4 *)(a.qt + ((long long)rep * a.cols + c0 + row) * a.pitch_t + r0 + piece) = u4{lo.x, lo.y, hi.x, hi.y};
  }
}

template <typename T, bool ROWS>
void run(hipStream_t st, dim3 grid, const void *src, const Args &a) {
  k_fp8_quantize<T, ROWS><<<grid, kThreads, 0, st>>>((const T *)src, a);
}

}  // namespace

hipError_t launch_fp8_quantize(hipStream_t st, const parle_quant_desc &d, const void *src, uint8_t *q, uint8_t *scales, uint8_t *qt,
                               uint8_t *scales_t) {
  Args a;
  a.q = q, a.scales = scales, a.qt = qt, a.scales_t = scales_t, a.ld = d.ld, a.stride = d.stride;
  a.rows = d.rows, a.cols = d.cols;
  const int rb = ceil_div(d.rows, kTile), cb = ceil_div(d.cols, kTile);
  a.pitch = (int)round_up(d.cols, 16), a.s_pitch = (int)round_up(cb, 4);
  a.pitch_t = (int)round_up(d.rows, 16), a.s_pitch_t = (int)round_up(rb, 4);
  const dim3 grid(cb, rb, d.n);
  if (d.dtype)
    d.block == 1 ? run<bf16_t, true>(st, grid, src, a) : run<bf16_t, false>(st, grid, src, a);
  else
    d.block == 1 ? run<float, true>(st, grid, src, a) : run<float, false>(st, grid, src, a);
  return hipGetLastError();
}
