// Attention of one new token of every sequence over its cache, and what puts a prompt's keys and values there.
//
// A cache is read once and nothing else matters, so its tokens are shared out over enough workgroups to keep memory busy, and their maxima, sums
// and partial results are joined behind.  The query heads of a key head, up to sixteen at a time, are the sixteen columns of a matrix instruction:
// S^T = K Q^T and O^T = V^T P^T as in the forward pass, in tiles of 16 keys.
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
  float *part;  // [sequences][heads][splits][dim + 2]: o, m, l
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

template <typename T, int DP>
__global__ __launch_bounds__(kThreads) void k_decode(DecodeArgs g) {
  using Tl = Tile<T, DP>;
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
  float *part = g.part + ((long long)seq * g.heads + head0) * g.splits * (g.dim + 2);
  T *kc = (T *)g.k_cache + ((long long)seq * g.kv_heads + kvh) * g.capacity * g.dim;
  T *vc = (T *)g.v_cache + ((long long)seq * g.kv_heads + kvh) * g.capacity * g.dim;

  if (length <= 0) {
    if (split == 0)
      for (int i = tid; i < cols * g.dim; i += kThreads) out[i] = 0;
    if (g.splits > 1)
      for (int i = tid; i < cols; i += kThreads) part[((long long)i * g.splits + split) * (g.dim + 2) + g.dim + 1] = 0.f;
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
  }
  __syncthreads();

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
  float *red = (float *)&lds[0][0];                // [wave][column][d], over the tiles of values
  constexpr int kAtOnce = sizeof(T) == 2 ? 2 : 4;  // wavefronts that find room there
  static_assert(kAtOnce * kCols * kPitch * 4 <= kWaves * kTileBytes, "");
  float total[(kCols * DP + kThreads - 1) / kThreads];
#pragma unroll
  for (int i = 0; i < (int)(sizeof(total) / 4); ++i) total[i] = 0.f;
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
    for (int i = 0; i < (int)(sizeof(total) / 4); ++i) {
      const int at = tid + i * kThreads;
      for (int w = 0; w < kAtOnce; ++w) total[i] += red[(w * kCols + at / DP) * kPitch + at % DP];
    }
    __syncthreads();
  }
  if (wave == 0 && lane < kCols) stat[0][0][col] = most, stat[0][1][col] = sum;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < (int)(sizeof(total) / 4); ++i) {
    const int at = tid + i * kThreads, cl = at / DP, d = at % DP;
    if (cl >= cols || d >= g.dim) continue;
    if (g.splits == 1) {
      const float v = total[i] / stat[0][1][cl];
      if constexpr (sizeof(T) == 4)
        out[(long long)cl * g.dim + d] = v;
      else
        out[(long long)cl * g.dim + d] = f32_to_bf16(v);
    } else {
      float *p = part + ((long long)cl * g.splits + split) * (g.dim + 2);
      p[d] = total[i];
      if (d == 0) p[g.dim] = stat[0][0][cl], p[g.dim + 1] = stat[0][1][cl];
    }
  }
}

// The shares of a head joined: one workgroup for a head, a thread for a column.
template <typename T>
__global__ __launch_bounds__(128) void k_decode_join(DecodeArgs g) {
  const int head = blockIdx.x, seq = blockIdx.y, d = threadIdx.x;
  if (g.lengths[seq] <= 0 || d >= g.dim) return;
  const float *p = g.part + ((long long)seq * g.heads + head) * g.splits * (g.dim + 2);
  float most = -INFINITY;
  for (int i = 0; i < g.splits; ++i) most = fmaxf(most, p[(long long)i * (g.dim + 2) + g.dim]);
  float sum = 0.f, o = 0.f;
  for (int i = 0; i < g.splits; ++i) {
    const float *x = p + (long long)i * (g.dim + 2);
    const float f = x[g.dim] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[g.dim] - most);
    sum += f * x[g.dim + 1], o += f * x[d];
  }
  T *out = (T *)g.out + (long long)seq * g.ld_out + (long long)head * g.dim;
  if constexpr (sizeof(T) == 4)
    out[d] = o / sum;
  else
    out[d] = f32_to_bf16(o / sum);
}

int visible(const parle_cache_desc &d) {
  const long long ring = (long long)d.capacity - d.sinks;
  return (int)(d.sinks + (d.window > 0 && d.window < ring ? d.window : ring));
}
// Shares of a cache: as many as fill the chip four workgroups to a compute unit, of kLeast tokens at least.
int splits_of(const parle_cache_desc &d) {
  if (d.sequences == 0) return 1;
  const long long groups = tok::ceil_div(d.heads / d.kv_heads, kCols), wgs = (long long)d.sequences * d.kv_heads * groups;
  long long n = (1024 + wgs - 1) / wgs;
  const long long most = tok::ceil_div(visible(d), kLeast);
  n = n < most ? n : most;
  return (int)(n < 1 ? 1 : n > 256 ? 256 : n);
}

// ---- a prompt's rows into the caches: a thread takes eight elements of a token's head, of k or of v ----
struct StoreArgs {
  const void *k, *v;
  const int32_t *offsets, *lengths;
  void *k_cache, *v_cache;
  int tokens, sequences, capacity, kv_heads, dim, sinks;
  long long ld_kv, items;
};
template <typename T>
__global__ __launch_bounds__(256) void k_store(StoreArgs g) {
  const int per = g.dim / 8, row_items = 2 * g.kv_heads * per;
  for (long long it = (long long)blockIdx.x * 256 + threadIdx.x; it < g.items; it += (long long)gridDim.x * 256) {
    const int row = (int)(it / row_items), rest = (int)(it - (long long)row * row_items);
    const int which = rest / (g.kv_heads * per), head = rest / per - which * g.kv_heads, e = (rest % per) * 8;
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
    if (row < begin || row >= end || p < 0 || !(p < g.sinks || p >= (long long)length - (g.capacity - g.sinks))) continue;
    const int slot = slot_of((int)p, g.sinks, g.capacity);
    const T *src = (const T *)(which ? g.v : g.k) + (long long)row * g.ld_kv + (long long)head * g.dim + e;
    T *dst = (T *)(which ? g.v_cache : g.k_cache) + (((long long)lo * g.kv_heads + head) * g.capacity + slot) * g.dim + e;
    const Frag<T> f = load_frag(src);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(u4 *)((char *)dst + 16 * i) = f.v[i];
  }
}

}  // namespace

int64_t decode_scratch_bytes(const parle_cache_desc &d) {
  const int s = splits_of(d);
  return s == 1 ? 0 : (int64_t)d.sequences * d.heads * s * (d.dim + 2) * 4;
}

hipError_t launch_attention_decode(hipStream_t st, const parle_cache_desc &d, const void *q, const void *k, const void *v, const int32_t *lengths,
                                   void *scratch, void *k_cache, void *v_cache, void *out) {
  const int groups = tok::ceil_div(d.heads / d.kv_heads, kCols), splits = splits_of(d);
  DecodeArgs g{q,         k,       v,       lengths, k_cache, v_cache, out,    (float *)scratch, d.sequences, d.capacity, d.heads, d.kv_heads, d.dim,
               d.window, d.sinks, splits, groups,  d.scale, d.ld_q,  d.ld_kv, d.ld_out};
  auto go = [&](auto *kernel, auto *join) {
    kernel<<<dim3(splits, d.kv_heads * groups, d.sequences), kThreads, 0, st>>>(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    join<<<dim3(d.heads, d.sequences), 128, 0, st>>>(g);
    return hipGetLastError();
  };
  if (d.dtype) return d.dim <= 64 ? go(k_decode<bf16_t, 64>, k_decode_join<bf16_t>) : go(k_decode<bf16_t, 128>, k_decode_join<bf16_t>);
  return d.dim <= 64 ? go(k_decode<float, 64>, k_decode_join<float>) : go(k_decode<float, 128>, k_decode_join<float>);
}

hipError_t launch_attention_store(hipStream_t st, const parle_cache_desc &d, int tokens, const void *k, const void *v, const int32_t *offsets,
                                  const int32_t *lengths, void *k_cache, void *v_cache) {
  const long long items = (long long)tokens * d.kv_heads * (d.dim / 8) * 2;
  StoreArgs g{k, v, offsets, lengths, k_cache, v_cache, tokens, d.sequences, d.capacity, d.kv_heads, d.dim, d.sinks, d.ld_kv, items};
  const long long wgs = (items + 255) / 256;
  const int grid = (int)(wgs < 16384 ? wgs : 16384);
  if (d.dtype)
    k_store<bf16_t><<<grid, 256, 0, st>>>(g);
  else
    k_store<float><<<grid, 256, 0, st>>>(g);
  return hipGetLastError();
}
