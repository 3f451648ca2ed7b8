// Shared pieces of the token-model operators: loads of rows that need no alignment, 8-bit conversion, launchers.
#pragma once
#include "common.h"

namespace tok {

typedef unsigned int u2 __attribute__((ext_vector_type(2)));
typedef unsigned int u4 __attribute__((ext_vector_type(4)));
// Vectors at element alignment: a row of odd width begins anywhere, and global memory takes wide accesses at any address.
typedef us8 us8_any __attribute__((aligned(2)));
typedef us4 us4_any __attribute__((aligned(2)));
typedef f4 f4_any __attribute__((aligned(4)));
typedef u4 u4_any __attribute__((aligned(4)));

constexpr int kVec = 8;  // elements that a thread takes at a time

constexpr int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
constexpr long long round_up(long long a, long long b) { return (a + b - 1) / b * b; }

// Eight elements as fp32; `count` of them exist (a row's last group), the others read as `fill`.
__device__ __forceinline__ void load8(const float *p, int count, float fill, float (&v)[kVec]) {
  if (count >= kVec) {
    const f4 a = *(const f4_any *)p, b = *(const f4_any *)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i < count ? p[i] : fill;
  }
}
__device__ __forceinline__ void load8(const bf16_t *p, int count, float fill, float (&v)[kVec]) {
  if (count >= kVec) {
    const us8 a = *(const us8_any *)p;
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = bf16_to_f32(a[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i < count ? bf16_to_f32(p[i]) : fill;
  }
}
__device__ __forceinline__ void store8(float *p, int count, const float (&v)[kVec]) {
  if (count >= kVec) {
    *(f4_any *)p = f4{v[0], v[1], v[2], v[3]};
    *(f4_any *)(p + 4) = f4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < count) p[i] = v[i];
  }
}
__device__ __forceinline__ void store8(bf16_t *p, int count, const float (&v)[kVec]) {
  if (count >= kVec) {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
    *(us8_any *)p = __builtin_bit_cast(us8, r);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < count) p[i] = f32_to_bf16(v[i]);
  }
}

// Eight elements as they came, to be widened when they are used; zeros past `count`.
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16_t> {
  us8 v;
  __device__ __forceinline__ void load(const bf16_t *p, int count) {
    if (count >= kVec) {
      v = *(const us8_any *)p;
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = i < count ? p[i] : (bf16_t)0;
    }
  }
  __device__ __forceinline__ float at(int i) const { return bf16_to_f32(v[i]); }
};
template <>
struct Raw8<float> {
  f4 a, b;
  __device__ __forceinline__ void load(const float *p, int count) {
    if (count >= kVec) {
      a = *(const f4_any *)p, b = *(const f4_any *)(p + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = i < count ? p[i] : 0.f, b[i] = 4 + i < count ? p[4 + i] : 0.f;
    }
  }
  __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};

// The value as it is stored in type T.
template <typename T>
__device__ __forceinline__ float stored(float v);
template <>
__device__ __forceinline__ float stored<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ float stored<bf16_t>(float v) {
  return bf16_to_f32(f32_to_bf16(v));
}

// ---- 8-bit: e4m3 codes under E8M0 scales ----
// Magnitude that counts for a block's scale: NaN and infinities do not.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// Scale byte of a block from the bits of its largest magnitude 1.m * 2^(E-127): the smallest e with that <= 448 * 2^e =
// 1.75 * 2^(e+8) is E - 135, one more where 1.m > 1.75; 1 for a block of zeros.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  const int e = (int)(most >> 23) - 135 + ((most & 0x7fffffu) > 0x600000u);
  return most == 0 ? 127u : (uint32_t)(max(e, -127) + 127);
}
// Magnitudes that the plain conversions below do not take: NaN and infinities, and what would need a scale of 2^-127.
__device__ __forceinline__ bool special_most(uint32_t most) { return most >= 0x7f800000u || (most != 0 && scale_byte(most) == 0); }
// Two values divided by 2^(byte-127), as codes in the lower or the upper half of a dword; not for special ones.
typedef short s2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf2_hw __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float scale_float(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ uint32_t codes4_of(float a, float b, float c, float d, float scale) {
  s2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true));
}
__device__ __forceinline__ uint32_t codes4_of(uint32_t ab, uint32_t cd, float scale) {  // pairs in bf16
  s2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf2_hw, ab), scale, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf2_hw, cd), scale, true));
}
// 2^-(byte-127): e is at most 120, so the result is a normal number.
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// Codes of four values that are already divided by their scale; infinity becomes NaN in front of the conversion.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
__device__ __forceinline__ float scaled(float v, float inv) {
  return (__float_as_uint(v) & 0x7fffffffu) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : v * inv;
}

// Sums and maxima over lanes, in all of them.  Neighbours, quads, halves and rows of 16 lanes exchange inside the vector unit; the
// four rows of a wavefront meet as scalars.
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float from_lane(float v) {
  return __uint_as_float(from_lane<CTRL>(__float_as_uint(v)));
}
constexpr int kLaneXor1 = 0xb1, kLaneXor2 = 0x4e, kHalfMirror = 0x141, kRowMirror = 0x140;

__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

__device__ __forceinline__ float row_sum8(float v) {
  v += from_lane<kLaneXor1>(v);
  v += from_lane<kLaneXor2>(v);
  return v + from_lane<kHalfMirror>(v);
}
__device__ __forceinline__ float row_sum16(float v) {
  v = row_sum8(v);
  return v + from_lane<kRowMirror>(v);
}
__device__ __forceinline__ float wave_sum_all(float v) {
  v = row_sum16(v);
  return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ __forceinline__ float wave_max_all(float v) {
  v = fmaxf(v, from_lane<kLaneXor1>(v));
  v = fmaxf(v, from_lane<kLaneXor2>(v));
  v = fmaxf(v, from_lane<kHalfMirror>(v));
  v = fmaxf(v, from_lane<kRowMirror>(v));
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
__device__ __forceinline__ uint32_t row_max16(uint32_t v) {
  v = max(v, from_lane<kLaneXor1>(v));
  v = max(v, from_lane<kLaneXor2>(v));
  v = max(v, from_lane<kHalfMirror>(v));
  return max(v, from_lane<kRowMirror>(v));
}

}  // namespace tok

hipError_t launch_embed_fwd(hipStream_t st, const parle_embed_desc &d, const void *table, const int32_t *tokens, void *out);
int64_t embed_scratch_bytes(const parle_embed_desc &d);
hipError_t launch_embed_bwd(hipStream_t st, const parle_embed_desc &d, const int32_t *tokens, const void *dout, void *scratch,
                            float *dtable);

hipError_t launch_rmsnorm_fwd(hipStream_t st, const parle_norm_desc &d, const void *x, const void *resid, const void *w, void *h,
                              void *y, uint8_t *q, uint8_t *scales, float *rstd);
int64_t rmsnorm_scratch_bytes(const parle_norm_desc &d);
hipError_t launch_rmsnorm_bwd(hipStream_t st, const parle_norm_desc &d, const void *h, const void *w, const float *rstd,
                              const void *dout, const void *dresid, float *partial, void *dx, float *dw);

hipError_t launch_fp8_quantize(hipStream_t st, const parle_quant_desc &d, const void *src, uint8_t *q, uint8_t *scales, uint8_t *qt,
                               uint8_t *scales_t);
int64_t fp8_scratch_bytes(const parle_fp8_desc &d);
hipError_t launch_fp8_matmul(hipStream_t st, const parle_fp8_desc &d, const uint8_t *a, const uint8_t *a_scales, const uint8_t *b,
                             const uint8_t *b_scales, const float *bias, float *partial, void *out);

int64_t logprob_scratch_bytes(const parle_logprob_desc &d);
hipError_t launch_logprob_fwd(hipStream_t st, const parle_logprob_desc &d, const void *logits, const int32_t *labels, void *scratch,
                              float *logp, float *entropy, float *lse, int32_t *top_ids, float *top_logp);
hipError_t launch_logprob_bwd(hipStream_t st, const parle_logprob_desc &d, const void *logits, const int32_t *labels, const float *lse,
                              const float *entropy, const float *dlogp, const float *dentropy, void *dlogits);
