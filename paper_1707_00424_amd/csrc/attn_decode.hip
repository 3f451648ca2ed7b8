// Attention of one new token of every sequence over its cache, and what puts a prompt's keys and values there.
//
// A cache is read once and nothing else matters, so its tokens are shared out over enough workgroups to keep memory busy, and their maxima, sums
// and partial results are joined behind.  The query heads of a key head, up to sixteen at a time, are the sixteen columns of a matrix instruction:
// S^T = K Q^T and O^T = V^T P^T as in the forward pass, in tiles of 16 keys.  A wavefront has the next 32 keys and values on their way in registers while
// it multiplies: 64 sequences of up to 8192 tokens, 32 heads on 8 of keys of 128 elements, bf16: 1.63 GB in 299 us, 5.4 TB/s (a plain read of as much 5.9); 4 sequences of 1028
// tokens 11.5 us, of which 8.3 are the shares and 3 to join them.
#include "attn.h"

namespace {

using namespace attn;
typedef float f4v __attribute__((ext_vector_type(4)));

constexpr int kStep = 32;   // keys of a wavefront at a time
constexpr int kCols = 16;   // query heads of a workgroup
constexpr int kLeast = 128; // keys that a share has at least: one step of each of four wavefronts

struct DecodeArgs {
  const void *q, *k, *v;
  const int32_t *lengths;
  void *k_cache, *v_cache, *out;
  float *part, *stats;  // of a share: o [sequences][heads][splits][dim]; m and l [sequences][heads][splits][2]
  int sequences, capacity, heads, kv_heads, dim, window, sinks, splits, groups;
  float scale;
  long long ld_q, ld_kv, ld_out;
};

// acc[row of a][column of b]: lane l holds column l % 16, rows 4 (l / 16) + i; a and b have eight values of row or column l % 16 at l / 16.
__device__ __forceinline__ void mma16(const Frag<bf16_t> &a, const Frag<bf16_t> &b, f4v &acc) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a.v[0]), __builtin_bit_cast(bf8, b.v[0]), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma16(const Frag<float> &a, const Frag<float> &b, f4v &acc) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(frag_at(a, j), frag_at(b, j), acc, 0, 0, 0);
}

// Which tokens of a sequence are seen: the first `first`, then those from `lo` on; `seen` of them.
struct Seen {
  int first, lo, seen;
};
__device__ __forceinline__ Seen seen_of(int length, int window, int sinks, int capacity) {
  const int ring = capacity - sinks, w = window > 0 ? min(window, ring) : ring;
  const int first = min(sinks, length), lo = max(first, length - w);
  return {first, lo, first + length - lo};
}
__device__ __forceinline__ int slot_of(int p, int sinks, int capacity) { return p < sinks ? p : sinks + (p - sinks) % (capacity - sinks); }

// Values of lanes l % 16 alike, over the four quarters.
__device__ __forceinline__ float quarters_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return half_max(v);
}
__device__ __forceinline__ float quarters_sum(float v) {
  v += __shfl_xor(v, 16);
  return half_sum(v);
}

template <typename T, int DP, int WAVES>
__global__ __launch_bounds__(WAVES *PARLE_WAVE) void k_decode(DecodeArgs g) {
  using Tl = Tile<T, DP>;
  constexpr int kWaves = WAVES, kThreads = WAVES * PARLE_WAVE;
  constexpr int NS = DP / 32, ND = DP / 16;
  constexpr int kChunks = DP / Tl::kChunk, kTurns = kStep * kChunks / PARLE_WAVE;  // 16-byte pieces of a step's values, of a lane
  constexpr int kTileBytes = kStep * Tl::kRowBytes;
  __shared__ __attribute__((aligned(1024))) char lds[kWaves][kTileBytes];
  __shared__ float stat[kWaves][2][kCols];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
  const int split = blockIdx.x, kvh = blockIdx.y / g.groups, group = blockIdx.y % g.groups, seq = blockIdx.z;
  const int share = g.heads / g.kv_heads, g0 = group * kCols, cols = min(kCols, share - g0), head0 = kvh * share + g0;
  const int length = g.lengths[seq];
  T *out = (T *)g.out + (long long)seq * g.ld_out + (long long)head0 * g.dim;
  float *part = g.part + ((long long)seq * g.heads + head0) * g.splits * g.dim;
  float *stats = g.stats + ((long long)seq * g.heads + head0) * g.splits * 2;
  T *kc = (T *)g.k_cache + ((long long)seq * g.kv_heads + kvh) * g.capacity * g.dim;
  T *vc = (T *)g.v_cache + ((long long)seq * g.kv_heads + kvh) * g.capacity * g.dim;

  if (length <= 0) {
    if (split == 0)
      for (int i = tid; i < cols * g.dim; i += kThreads) out[i] = 0;
    return;
  }
  const Seen s = seen_of(length, g.window, g.sinks, g.capacity);
  // this share of the tokens seen: [from, to)
  const int each = (int)tok::round_up(((long long)s.seen + g.splits - 1) / g.splits, kStep);
  const int from = min((long long)split * each, (long long)s.seen), to = min((long long)from + each, (long long)s.seen);

  if (g.k && to == s.seen && from < to) {
    // the new token's rows; what this workgroup reads of the caches comes behind the barrier
    const int slot = slot_of(length - 1, g.sinks, g.capacity);
    const T *kn = (const T *)g.k + (long long)seq * g.ld_kv + (long long)kvh * g.dim, *vn = (const T *)g.v + (long long)seq * g.ld_kv + (long long)kvh * g.dim;
    if (tid < g.dim) kc[(long long)slot * g.dim + tid] = kn[tid];
    if (tid >= 128 && tid - 128 < g.dim) vc[(long long)slot * g.dim + tid - 128] = vn[tid - 128];
    __syncthreads();
  }

  Frag<T> qf[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    qf[i] = zero_frag<T>();
    const int at = 32 * i + 8 * quarter;
    if (col < cols && at < g.dim) qf[i] = load_frag((const T *)g.q + (long long)seq * g.ld_q + (long long)(head0 + col) * g.dim + at);
  }

  // slot of the u-th token seen
  const int ring = g.capacity - g.sinks, turn = s.lo >= g.sinks ? (s.lo - g.sinks) % ring : 0;
  auto slot = [&](int u) {
    if (u < s.first) return u;
    const int r = turn + (u - s.first);
    return g.sinks + (r < ring ? r : r - ring);
  };
  Frag<T> kf[2][NS];
  u4 vr[kTurns];
  auto fetch = [&](int u0) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const T *p = kc + (long long)slot(min(u0 + 16 * b + col, to - 1)) * g.dim;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        kf[b][i] = zero_frag<T>();
        const int at = 32 * i + 8 * quarter;
        if (at < g.dim) kf[b][i] = load_frag(p + at);
      }
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int at = lane + i * PARLE_WAVE, r = at / kChunks, c = at % kChunks;
      vr[i] = u4{0u, 0u, 0u, 0u};
      if (c * Tl::kChunk < g.dim) vr[i] = *(const u4 *)(vc + (long long)slot(min(u0 + r, to - 1)) * g.dim + c * Tl::kChunk);
    }
  };

  const float c = g.scale * kLog2e;
  f4v o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = f4v{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  char *vt = lds[wave];
  int u0 = from + wave * kStep;
  if (u0 < to) fetch(u0);
  for (; u0 < to; u0 += kWaves * kStep) {
    f4v sc[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      sc[b] = f4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NS; ++i) mma16(kf[b][i], qf[i], sc[b]);
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
      const int at = lane + i * PARLE_WAVE, r = at / kChunks, cc = at % kChunks;
      *(u4 *)(vt + Tl::at(r, cc)) = vr[i];
    }
    // the tile is this wavefront's own, written and read in order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (u0 + kWaves * kStep < to) fetch(u0 + kWaves * kStep);
    if (u0 + kStep > to) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sc[b][i] = u0 + 16 * b + 4 * quarter + i >= to ? -INFINITY : sc[b][i];
    }
    float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])), fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
    top = quarters_max(top) * c;
    if (__any(top > m + 8.f)) {  // as in the forward pass
      const float now = fmaxf(m, top), f = now == m ? 1.f : __builtin_amdgcn_exp2f(m - now);
      m = now, l *= f;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= f;
    }
    const float mu = m == -INFINITY ? 0.f : m;
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j >> 2][j & 3], c, -mu));
    l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    const Frag<T> pf = make_frag<T>(p);
    // contraction value j of quarter h is key 16 (j / 4) + 4 h + j % 4
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      Frag<T> f;
      if constexpr (sizeof(T) == 4) {
        const int e = 16 * d + col;
#pragma unroll
        for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = *(const uint32_t *)(vt + Tl::at(16 * (j >> 2) + 4 * quarter + (j & 3), e >> 2) + 4 * (e & 3));
      } else {
        const int r = 4 * quarter + (col >> 2), e = 16 * d + 4 * (col & 3);
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(vt + Tl::at(r, e >> 3) + 2 * (e & 7)));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(vt + Tl::at(r + 16, e >> 3) + 2 * (e & 7)));
        f.v[0] = __builtin_bit_cast(u4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
      mma16(f, pf, o[d]);
    }
  }
  l = quarters_sum(l);

  // the wavefronts' results meet at the largest of their maxima
  if (lane < kCols) stat[wave][0][col] = m, stat[wave][1][col] = l;
  __syncthreads();  // the tiles of values are dead as well
  float most = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) most = fmaxf(most, stat[w][0][col]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += stat[w][1][col] * (stat[w][0][col] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat[w][0][col] - most));
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - most);
  constexpr int kPitch = DP + 4;
  float *red = (float *)&lds[0][0];                         // [wave][column][d], over the tiles of values
  constexpr int kAtOnce = sizeof(T) == 2 ? kWaves / 2 : kWaves;  // wavefronts that find room there
  static_assert(kAtOnce * kCols * kPitch * 4 <= kWaves * kTileBytes, "");
  constexpr int kSums = (kCols * DP + kThreads - 1) / kThreads;
  float total[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) total[i] = 0.f;
#pragma unroll
  for (int w0 = 0; w0 < kWaves; w0 += kAtOnce) {
    if (wave >= w0 && wave < w0 + kAtOnce) {
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[((wave - w0) * kCols + col) * kPitch + 16 * d + 4 * quarter + i] = o[d][i] * f;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSums; ++i) {
      const int at = tid + i * kThreads;
      for (int w = 0; w < kAtOnce; ++w) total[i] += red[(w * kCols + at / DP) * kPitch + at % DP];
    }
    __syncthreads();
  }
  if (wave == 0 && lane < kCols) stat[0][0][col] = most, stat[0][1][col] = sum;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSums; ++i) {
    const int at = tid + i * kThreads, cl = at / DP, d = at % DP;
    if (cl >= cols || d >= g.dim) continue;
    if (g.splits == 1) {
      const float v = total[i] / stat[0][1][cl];
      if constexpr (sizeof(T) == 4)
        out[(long long)cl * g.dim + d] = v;
      else
        out[(long long)cl * g.dim + d] = f32_to_bf16(v);
    } else {
      part[((long long)cl * g.splits + split) * g.dim + d] = total[i];
      if (d == 0) *(f2 *)(stats + ((long long)cl * g.splits + split) * 2) = f2{stat[0][0][cl], stat[0][1][cl]};
    }
  }
}

// The shares of a head joined: a workgroup for a head, a wavefront for every fourth share, four columns to a lane.  All loads are on their way at once.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_decode_join(DecodeArgs g) {
  constexpr int kMost = 256 / PARLE_WAVE;  // shares of a lane
  __shared__ float factor[256];
  __shared__ f4 sums[kWaves][32];
  const int head = blockIdx.x, seq = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (g.lengths[seq] <= 0) return;
  const float *stats = g.stats + ((long long)seq * g.heads + head) * g.splits * 2;
  const float *part = g.part + ((long long)seq * g.heads + head) * g.splits * g.dim;
  float m[kMost], l[kMost], most = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int at = lane + i * PARLE_WAVE;
    const f2 v = at < g.splits ? *(const f2 *)(stats + 2 * at) : f2{-INFINITY, 0.f};
    m[i] = v.x, l[i] = v.y, most = fmaxf(most, v.x);
  }
  most = tok::wave_max_all(most);
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const float f = m[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[i] - most);
    sum += f * l[i];
    if (wave == 0) factor[lane + i * PARLE_WAVE] = f;
  }
  sum = tok::wave_sum_all(sum);
  __syncthreads();
  const int at = (lane & 31) * 4, half = lane >> 5;
  f4 o = {0.f, 0.f, 0.f, 0.f};
  if (at < g.dim) {
#pragma unroll 4
    for (int i = 2 * wave + half; i < g.splits; i += 2 * kWaves) o += factor[i] * *(const f4 *)(part + (long long)i * g.dim + at);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
  if (half == 0) sums[wave][lane] = o;
  __syncthreads();
  if (threadIdx.x < 32 && at < g.dim) {
    o = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
    const float inv = 1.f / sum;
    store4((T *)g.out + (long long)seq * g.ld_out + (long long)head * g.dim + at, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  }
}

int visible(const parle_cache_desc &d) {
  const long long ring = (long long)d.capacity - d.sinks;
  return (int)(d.sinks + (d.window > 0 && d.window < ring ? d.window : ring));
}
// Few tokens of many sequences, or so few that there is nothing to share, go through one workgroup of eight wavefronts for a key head: a share for each of
// several workgroups costs a second launch to join them.  1028 tokens, 8 key heads: 4 sequences take 15 us in one and 11.5 in shares, 32 sequences
// 28 and 34.
bool in_one(const parle_cache_desc &d) {
  const long long wgs = (long long)d.sequences * d.kv_heads * tok::ceil_div(d.heads / d.kv_heads, kCols);
  return visible(d) <= (wgs >= 128 ? 1536 : 512);
}
// Shares of a cache: as many as make two workgroups for a compute unit, of kLeast tokens at least; 16384 tokens of one sequence, 8 key heads, take
// 17.7 us in 64 shares, 21.4 in 128.
int splits_of(const parle_cache_desc &d) {
  if (d.sequences == 0 || in_one(d)) return 1;
  const long long wgs = (long long)d.sequences * d.kv_heads * tok::ceil_div(d.heads / d.kv_heads, kCols);
  long long n = (512 + wgs - 1) / wgs;
  const long long most = tok::ceil_div(visible(d), kLeast);
  n = n < most ? n : most;
  return (int)(n < 1 ? 1 : n > 256 ? 256 : n);
}

// ---- a prompt's rows into the caches: a wavefront takes a row, whose sequence and slot it looks up once, and a lane eight elements of a head.
// Memory bounds it: 16384 rows of 8 heads of 128 elements, bf16, 14 us, 6.0 TB/s for what is kept ----
struct StoreArgs {
  const void *k, *v;
  const int32_t *offsets, *lengths;
  void *k_cache, *v_cache;
  int tokens, sequences, capacity, kv_heads, dim, sinks;
  long long ld_kv;
};
template <typename T>
__global__ __launch_bounds__(kThreads) void k_store(StoreArgs g) {
  const int lane = threadIdx.x & 63, row = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
  if (row >= g.tokens) return;
  int lo = 0, hi = g.sequences;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (g.offsets[mid] <= row)
      lo = mid;
    else
      hi = mid;
  }
  const int begin = g.offsets[lo], end = g.offsets[lo + 1], length = g.lengths[lo];
  const long long p = (long long)length - end + row;
  if (row < begin || row >= end || p < 0 || !(p < g.sinks || p >= (long long)length - (g.capacity - g.sinks))) return;
  const int slot = slot_of((int)p, g.sinks, g.capacity);
  const long long head_step = (long long)g.capacity * g.dim, first = ((long long)lo * g.kv_heads * g.capacity + slot) * g.dim;
  const int per = g.dim / 8, items = g.kv_heads * per;
  const T *k = (const T *)g.k + row * g.ld_kv, *v = (const T *)g.v + row * g.ld_kv;
  for (int it = lane; it < items; it += PARLE_WAVE) {
    const int head = it / per, e = (it - head * per) * 8;
    const Frag<T> fk = load_frag(k + it * 8), fv = load_frag(v + it * 8);  // a row's heads lie one behind the other
    const long long at = first + head * head_step + e;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      *(u4 *)((char *)((T *)g.k_cache + at) + 16 * i) = fk.v[i];
      *(u4 *)((char *)((T *)g.v_cache + at) + 16 * i) = fv.v[i];
    }
  }
}

}  // namespace

int64_t decode_scratch_bytes(const parle_cache_desc &d) {
  const int s = splits_of(d);
  return s == 1 ? 0 : (int64_t)d.sequences * d.heads * s * (d.dim + 2) * 4;  // dim is a multiple of 8, so both parts are aligned
}

hipError_t launch_attention_decode(hipStream_t st, const parle_cache_desc &d, const void *q, const void *k, const void *v, const int32_t *lengths,
                                   void *scratch, void *k_cache, void *v_cache, void *out) {
  const int groups = tok::ceil_div(d.heads / d.kv_heads, kCols), splits = splits_of(d);
  DecodeArgs g{q,         k,       v,       lengths, k_cache, v_cache, out,    (float *)scratch, (float *)scratch + (int64_t)d.sequences * d.heads * splits * d.dim, d.sequences, d.capacity, d.heads, d.kv_heads, d.dim,
               d.window, d.sinks, splits, groups,  d.scale, d.ld_q,  d.ld_kv, d.ld_out};
  // fp32 rows of 128 elements leave no registers for eight wavefronts: 32 sequences of 512 tokens, 8 key heads, 37 us with eight, 30 with four
  const bool eight = in_one(d) && (d.dtype || d.dim <= 64);
  auto go = [&](auto *kernel, auto *join) {
    kernel<<<dim3(splits, d.kv_heads * groups, d.sequences), (eight ? 8 : 4) * PARLE_WAVE, 0, st>>>(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    join<<<dim3(d.heads, d.sequences), kThreads, 0, st>>>(g);
    return hipGetLastError();
  };
#define PARLE_GO(T, DP) (eight ? go(k_decode<T, DP, 8>, k_decode_join<T>) : go(k_decode<T, DP, 4>, k_decode_join<T>))
  if (d.dtype) return d.dim <= 64 ? PARLE_GO(bf16_t, 64) : PARLE_GO(bf16_t, 128);
  return d.dim <= 64 ? PARLE_GO(float, 64) : go(k_decode<float, 128, 4>, k_decode_join<float>);
#undef PARLE_GO
}

hipError_t launch_attention_store(hipStream_t st, const parle_cache_desc &d, int tokens, const void *k, const void *v, const int32_t *offsets,
                                  const int32_t *lengths, void *k_cache, void *v_cache) {
  StoreArgs g{k, v, offsets, lengths, k_cache, v_cache, tokens, d.sequences, d.capacity, d.kv_heads, d.dim, d.sinks, d.ld_kv};
  const int grid = tok::ceil_div(tokens, kWaves);
  if (d.dtype)
    k_store<bf16_t><<<grid, kThreads, 0, st>>>(g);
  else
    k_store<float><<<grid, kThreads, 0, st>>>(g);
  return hipGetLastError();
}
