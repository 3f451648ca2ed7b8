// 8-bit codes and power-of-two scales of a matrix and of its transpose, from one read.
//
// A workgroup takes a 128 x 128 tile: it is what shares a scale (block 128), or holds whole scale blocks in both directions
// (block 1: 128 values of a row, and 128 of a column for the transpose).  The tile passes through LDS in fp32; rows
// are written from the registers that loaded them, columns are read back from LDS.
#include "tok.h"

namespace {

using namespace tok;

constexpr int kThreads = 256, kTile = 128;
constexpr int kPitch = kTile + 1;  // fp32: columns are read without bank conflicts

struct Args {
  uint8_t *q, *scales, *qt, *scales_t;
  long long ld, stride;
  int rows, cols, block;
  int pitch, s_pitch, pitch_t, s_pitch_t;  // of codes and scales, and of the transpose's
};

// grid: (row tiles, column tiles, n)
template <typename T>
__global__ __launch_bounds__(kThreads) void k_fp8_quantize(const T *src, Args a) {
  __shared__ float tile[kTile * kPitch];
  __shared__ uint32_t most_of[kTile * 2 + 8];
  const int r0 = blockIdx.x * kTile, c0 = blockIdx.y * kTile, rep = blockIdx.z;
  const int lane16 = threadIdx.x & 15, group = threadIdx.x >> 4;
  const T *from = src + rep * a.stride + c0 + lane16 * kVec;
  const int left = a.cols - c0 - lane16 * kVec;
  float v[kTile / 16][kVec];
#pragma unroll
  for (int j = 0; j < kTile / 16; ++j) {
    const int r = r0 + j * 16 + group;
    load8(from + (long long)min(r, a.rows - 1) * a.ld, r < a.rows ? left : 0, 0.f, v[j]);
  }
  uint32_t all = 0;
  uint32_t most[kTile / 16];
#pragma unroll
  for (int j = 0; j < kTile / 16; ++j) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = max(m, finite_bits(v[j][i]));
    most[j] = row_max16(m);
    all = max(all, most[j]);
  }
  if (a.qt) {
#pragma unroll
    for (int j = 0; j < kTile / 16; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) tile[(j * 16 + group) * kPitch + lane16 * kVec + i] = v[j][i];
  }
  if (a.block != 1) {
    if (lane16 == 0) most_of[group] = all;
  }
  __syncthreads();
  if (a.block != 1) {
    for (int g = 0; g < 16; ++g) all = max(all, most_of[g]);
  }
  const int kb = blockIdx.y, rb = blockIdx.x;  // block columns of q, of qt
  if (a.q) {
#pragma unroll
    for (int j = 0; j < kTile / 16; ++j) {
      const int r = r0 + j * 16 + group;
      if (r >= a.rows) continue;
      const uint32_t sb = scale_byte(a.block == 1 ? most[j] : all);
      const float inv = scale_inverse(sb);
      const int c = c0 + lane16 * kVec;
      if (c < a.pitch) {
        const float *u = v[j];
        *(u2 *)(a.q + ((long long)rep * a.rows + r) * a.pitch + c) =
            u2{codes4(scaled(u[0], inv), scaled(u[1], inv), scaled(u[2], inv), scaled(u[3], inv)),
               codes4(scaled(u[4], inv), scaled(u[5], inv), scaled(u[6], inv), scaled(u[7], inv))};
      }
      if (a.block == 1 && lane16 == 0) {
        uint8_t *s = a.scales + ((long long)rep * a.rows + r) * a.s_pitch;
        s[kb] = (uint8_t)sb;
        if (kb == (int)gridDim.y - 1)
          for (int k = kb + 1; k < a.s_pitch; ++k) s[k] = 0;
      }
    }
    if (a.block != 1 && threadIdx.x == 0) {
      uint8_t *s = a.scales + ((long long)rep * gridDim.x + rb) * a.s_pitch;
      s[kb] = (uint8_t)scale_byte(all);
      if (kb == (int)gridDim.y - 1)
        for (int k = kb + 1; k < a.s_pitch; ++k) s[k] = 0;
    }
  }
  if (!a.qt) return;
  // a column of the tile is half a thread pair's: rows 64 h .. 64 h + 63
  const int c = threadIdx.x & (kTile - 1), h = threadIdx.x >> 7;
  uint32_t sb;
  if (a.block == 1) {
    uint32_t m = 0;
    for (int r = 0; r < kTile / 2; ++r) m = max(m, finite_bits(tile[(h * 64 + r) * kPitch + c]));
    most_of[h * kTile + c] = m;
    __syncthreads();
    sb = scale_byte(max(most_of[c], most_of[kTile + c]));
  } else {
    sb = scale_byte(all);
  }
  if (c0 + c >= a.cols) return;
  const float inv = scale_inverse(sb);
  uint8_t *out = a.qt + ((long long)rep * a.cols + c0 + c) * a.pitch_t + r0 + h * 64;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if (r0 + h * 64 + g * 16 >= a.pitch_t) break;
    u4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float *t = &tile[(h * 64 + g * 16 + k * 4) * kPitch + c];
      w[k] = codes4(scaled(t[0], inv), scaled(t[kPitch], inv), scaled(t[2 * kPitch], inv), scaled(t[3 * kPitch], inv));
    }
    *(u4 *)(out + g * 16) = w;
  }
  if (h == 0 && (a.block == 1 || c == 0)) {
    const long long srow = a.block == 1 ? (long long)rep * a.cols + c0 + c : (long long)rep * gridDim.y + kb;
    uint8_t *s = a.scales_t + srow * a.s_pitch_t;
    s[rb] = (uint8_t)sb;
    if (rb == (int)gridDim.x - 1)
      for (int k = rb + 1; k < a.s_pitch_t; ++k) s[k] = 0;
  }
}

}  // namespace

hipError_t launch_fp8_quantize(hipStream_t st, const parle_quant_desc &d, const void *src, uint8_t *q, uint8_t *scales, uint8_t *qt,
                               uint8_t *scales_t) {
  Args a;
  a.q = q, a.scales = scales, a.qt = qt, a.scales_t = scales_t, a.ld = d.ld, a.stride = d.stride;
  a.rows = d.rows, a.cols = d.cols, a.block = d.block;
  const int rb = ceil_div(d.rows, kTile), cb = ceil_div(d.cols, kTile);
  a.pitch = (int)round_up(d.cols, 16), a.s_pitch = (int)round_up(cb, 4);
  a.pitch_t = (int)round_up(d.rows, 16), a.s_pitch_t = (int)round_up(rb, 4);
  const dim3 grid(rb, cb, d.n);
  if (d.dtype)
    k_fp8_quantize<bf16_t><<<grid, kThreads, 0, st>>>((const bf16_t *)src, a);
  else
    k_fp8_quantize<float><<<grid, kThreads, 0, st>>>((const float *)src, a);
  return hipGetLastError();
}
