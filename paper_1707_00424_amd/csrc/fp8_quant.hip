// 8-bit codes and power-of-two scales of a matrix and of its transpose, from one read.
//
// A workgroup takes a 128 x 128 tile: it is what shares a scale (block 128), or holds whole scale blocks in both directions
// (block 1: 128 values of a row, and 128 of a column for the transpose).  A thread holds 8 x 8 neighbouring values in registers: largest
// magnitudes go over lanes and through a little LDS, rows of codes are written from where they are, and columns pass through LDS as
// bytes, eight rows of a column at a time, so that a tile takes 17 KiB and rows of both results leave in whole lines of 128 bytes.
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

// Codes of eight values under one scale.
__device__ __forceinline__ u2 codes8(const float (&v)[kVec], float inv) {
  return u2{codes4(scaled(v[0], inv), scaled(v[1], inv), scaled(v[2], inv), scaled(v[3], inv)),
            codes4(scaled(v[4], inv), scaled(v[5], inv), scaled(v[6], inv), scaled(v[7], inv))};
}
// Block `at` of a row of scales; the last of `blocks` also clears the row's padding.
__device__ __forceinline__ void put_scale(uint8_t *row, int at, int blocks, int pitch, uint32_t byte) {
  row[at] = (uint8_t)byte;
  if (at == blocks - 1)
    for (int k = blocks; k < pitch; ++k) row[k] = 0;
}

// grid: (column tiles, row tiles, n).  Thread: columns 8 lane16 .. + 7, rows 8 group .. + 7 of the tile.
template <typename T, bool ROWS>
__global__ __launch_bounds__(kThreads) void k_fp8_quantize(const T *src, Args a) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[kTile * kPitch];
  __shared__ uint32_t most_of[kWaves][kTile];
  const int r0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile, rep = blockIdx.z;
  const int lane16 = threadIdx.x & 15, group = threadIdx.x >> 4, wave = threadIdx.x / PARLE_WAVE;
  const int c = c0 + lane16 * kVec, r = r0 + group * kVec, left = a.cols - c;
  const T *from = src + rep * a.stride + c;
  float v[kVec][kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) load8(from + (long long)min(r + j, a.rows - 1) * a.ld, r + j < a.rows ? left : 0, 0.f, v[j]);
  // largest magnitudes: of rows over 16 lanes, of columns over the groups of a wavefront, then over wavefronts
  uint32_t row_most[kVec], col_most[kVec] = {};
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    row_most[j] = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const uint32_t b = finite_bits(v[j][i]);
      row_most[j] = max(row_most[j], b), col_most[i] = max(col_most[i], b);
    }
  }
  uint32_t byte = 0;  // of the whole tile
  if (ROWS) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) row_most[j] = row_max16(row_most[j]);
    if (a.qt) {
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
      }
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
    byte = scale_byte(m);
  }
  const float tile_inv = scale_inverse(byte);
  if (a.q && c < a.pitch) {
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      if (r + j >= a.rows) break;
      const uint32_t sb = ROWS ? scale_byte(row_most[j]) : byte;
      *(u2 *)(a.q + ((long long)rep * a.rows + r + j) * a.pitch + c) = codes8(v[j], ROWS ? scale_inverse(sb) : tile_inv);
      if (ROWS && lane16 == 0)
        put_scale(a.scales + ((long long)rep * a.rows + r + j) * a.s_pitch, blockIdx.x, gridDim.x, a.s_pitch, sb);
    }
  }
  if (!ROWS && a.q && threadIdx.x == 0)
    put_scale(a.scales + ((long long)rep * gridDim.y + blockIdx.y) * a.s_pitch, blockIdx.x, gridDim.x, a.s_pitch, byte);
  if (!a.qt) return;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const float inv = ROWS ? scale_inverse(scale_byte(col_most[i])) : tile_inv;
    const float u[kVec] = {v[0][i], v[1][i], v[2][i], v[3][i], v[4][i], v[5][i], v[6][i], v[7][i]};
    *(u2 *)(turned + (lane16 * kVec + i) * kPitch + group * kVec) = codes8(u, inv);
  }
  if (ROWS) {
    if (group == 0) {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (i < left) put_scale(a.scales_t + ((long long)rep * a.cols + c + i) * a.s_pitch_t, blockIdx.y, gridDim.y, a.s_pitch_t, scale_byte(col_most[i]));
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

template <typename T>
void run(hipStream_t st, dim3 grid, const void *src, const Args &a, bool rows) {
  if (rows)
    k_fp8_quantize<T, true><<<grid, kThreads, 0, st>>>((const T *)src, a);
  else
    k_fp8_quantize<T, false><<<grid, kThreads, 0, st>>>((const T *)src, a);
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
    run<bf16_t>(st, grid, src, a, d.block == 1);
  else
    run<float>(st, grid, src, a, d.block == 1);
  return hipGetLastError();
}
