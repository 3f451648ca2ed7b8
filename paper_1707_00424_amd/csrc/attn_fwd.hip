// Attention over packed sequences, forward: one pass over the keys that a tile of queries sees, with the running maximum and sum of the softmax:
// m = max s, l = sum e^(s - m), o = sum e^(s - m) v over the keys so far; where m grows, l and o are multiplied by e^(m before - m).
//
// A wavefront has 32 queries, whose Q stays in registers; tiles of 64 keys and values go from memory straight into LDS, the next one while one is
// multiplied.  Per tile that is as much work for the matrix unit (of 128 elements: 32 instructions of 32 cycles) as for the vector unit (exponentials, maxima
// and conversions), and half of that for LDS, where the values' transposing reads go at a quarter of the rate of rows.  Two wavefronts of a SIMD overlap
// them in part: 8192 tokens of 32 heads of 128 elements in bf16, 534 us, are 1.03 PFLOP/s, the units 55 and 51 % of the time busy.  With a window of 1024 (16
// heads) it is 0.66 PFLOP/s, 83 us: a third of what a wavefront multiplies lies outside of its window's edges, and starts are a larger part.
// 64 queries to a wavefront, which would halve the reads of LDS, need more registers than there are.
#include "attn.h"

namespace {

using namespace attn;

constexpr int kRows = 32 * kWaves;  // queries of a workgroup, 32 to a wavefront

// PARTS wavefronts share queries: they take the tiles of keys in turn, and their maxima, sums and results meet in LDS, so that few queries still
// make enough workgroups.
template <typename T, int DP, int PARTS, bool DMA>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 4 && DP == 128) || (PARTS > 1 && (sizeof(T) == 4 || DP > 64)) ? 1 : 2) void k_attn_fwd(Args g) {
  using Tl = Tile<T, DP>;
  constexpr int BN = sizeof(T) == 2 && PARTS == 1 ? 64 : 32, NB = BN / 32, ND = DP / 32, NS = DP / 16, kQueries = kRows / PARTS;
  constexpr int kTileBytes = BN * Tl::kRowBytes;
  __shared__ __attribute__((aligned(1024))) char lds[2][PARTS][2][kTileBytes];  // of keys and values, for each part, of two steps

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, part = wave % PARTS;
  const int hx = blockIdx.x % g.heads, kvh = hx % g.kv_heads, head = kvh * (g.heads / g.kv_heads) + hx / g.kv_heads;
  const int tile = g.tiles - 1 - blockIdx.x / g.heads, rep = blockIdx.y;
  const int32_t *offsets = g.offsets ? g.offsets + (long long)rep * (g.sequences + 1) : nullptr;
  const T *q = (const T *)g.q + rep * g.q_stride + (long long)head * g.dim;
  const T *k = (const T *)g.k + rep * g.kv_stride + (long long)kvh * g.dim;
  const T *v = (const T *)g.v + rep * g.kv_stride + (long long)kvh * g.dim;

  const int r0 = tile * kQueries, w0 = r0 + wave / PARTS * 32, row = w0 + (lane & 31);
  const Span cov = covered(offsets, g.sequences, g.tokens);
  Sight s = sight_of({0, 0}, 0, 0, 0);
  if (row < g.tokens) s = sight_of(span_of(offsets, g.sequences, g.tokens, row), row, g.window, g.sinks);
  const int rv0 = max(r0, cov.start), rv1 = min(r0 + kQueries, cov.end) - 1;

  // Keys: [s0, s1) of the sinks in front of the window of the first row, then [klo, khi).  A sequence that begins inside the tile has its
  // sinks in the second part.
  int klo = 0, khi = 0, s0 = 0, s1 = 0;
  if (rv0 <= rv1) {
    const Sight f = sight_of(span_of(offsets, g.sequences, g.tokens, rv0), rv0, g.window, g.sinks);
    if (f.count) klo = f.lo, khi = rv1 + 1, s0 = f.start, s1 = min(f.start + (int)f.sinks, f.lo);
  }
  klo = __builtin_amdgcn_readfirstlane(klo), khi = __builtin_amdgcn_readfirstlane(khi);
  s0 = __builtin_amdgcn_readfirstlane(s0), s1 = __builtin_amdgcn_readfirstlane(s1);
  const int nS = s1 > s0 ? (s1 - s0 + BN - 1) / BN : 0, total = nS + (khi - klo + BN - 1) / BN;
  // of this wavefront's rows: whether all lie in sequences, the first key of the first and of the last one's window, the first one's sinks
  const bool all_in = w0 >= cov.start && w0 + 31 < cov.end;
  const int lo_first = __builtin_amdgcn_readlane(s.lo, 0), lo_last = __builtin_amdgcn_readlane(s.lo, 31);
  const int sink_first = __builtin_amdgcn_readlane(s.start, 0) + g.sinks;

  Frag<T> qf[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    qf[i] = zero_frag<T>();
    if (16 * i + 8 * h < g.dim) qf[i] = load_frag(q + (long long)min(row, g.tokens - 1) * g.ld_q + 16 * i + 8 * h);
  }

  Loader<T, DP, BN, DMA> kl, vl;
  kl.init(g.ld_kv, g.dim), vl.init(g.ld_kv, g.dim);
  kl.from(k, khi - 1), vl.from(v, khi - 1);
  typename Tl::Places at;
  at.init(lane);

  settle();
  const float c = g.scale * kLog2e;
  f16v o[ND];
  float m, l;
  // Masked tiles multiply the values of keys that a row does not see by zero, which is no zero where they are infinite or NaN.  That is looked
  // for in the result, and only then is all done again with such values taken out of those tiles and their rows noted.
  auto pass = [&](auto safe) {
    constexpr bool SAFE = decltype(safe)::value;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = zero16();
    m = -INFINITY, l = 0.f;
    auto base_of = [&](int t) { return t < nS ? s0 + t * BN : klo + (t - nS) * BN; };
    auto fetch = [&](int step) {  // tiles behind the last have no rows that are seen
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        const int at = base_of(step * PARTS + i);
        kl.load(lds[step & 1][i][0], at), vl.load(lds[step & 1][i][1], at);
      }
    };
    const int steps = (total + PARTS - 1) / PARTS;
    if (steps > 0) fetch(0);
    for (int step = 0; step < steps; ++step) {
      arrive<0>();
      if (step + 1 < steps) fetch(step + 1);
      const int t = step * PARTS + part, kb = base_of(t);
      const char *kt = lds[step & 1][part][0], *vt = lds[step & 1][part][1];
      const bool none = kb > w0 + 31 || (all_in && t >= nS && kb + BN - 1 < lo_first && kb >= sink_first);
      if (!none) {
        f16v sc[NB];
        Frag<T> kf[NB][NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) kf[0][i] = Tl::row(kt, at, 0, i);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if (b + 1 < NB) {
#pragma unroll
            for (int i = 0; i < NS; ++i) kf[b + 1][i] = Tl::row(kt, at, 32 * (b + 1), i);
          }
          sc[b] = zero16();
#pragma unroll
          for (int i = 0; i < NS; ++i) mma(kf[b][i], qf[i], sc[b]);
        }
        const bool whole = all_in && t >= nS && kb + BN - 1 <= w0 && kb >= lo_last;
        uint32_t seen[NB];
        if (!whole) {
          const Sight now = t < nS ? only_sinks(s, s1) : s;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if (SAFE) seen[b] = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const bool ok = now.sees(kb + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3));
              if (SAFE) seen[b] |= (uint32_t)ok << i;
              sc[b][i] = ok ? sc[b][i] : -INFINITY;
            }
          }
        }
        // Everything is relative to m, the largest of scale log2(e) s so far or up to eight below it: as one number m is the same for all
        // terms of a row, so its own rounding cancels, and o need not be scaled again for each small step of the maximum.
        float top = sc[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[b][i]);
        top = half_max(top) * c;
        if (__any(top > m + 8.f)) {
          const float now = fmaxf(m, top), f = now == m ? 1.f : __builtin_amdgcn_exp2f(m - now);
          m = now, l *= f;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float mu = m == -INFINITY ? 0.f : m;
        Frag<T> pf[2 * NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][8 * u + j], c, -mu));
            l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
            pf[2 * b + u] = make_frag<T>(p);
          }
        if (!SAFE || whole) {
#pragma unroll
          for (int u = 0; u < 2 * NB; ++u)
#pragma unroll
            for (int d = 0; d < ND; ++d) mma(Tl::column(vt, at, 16 * u, d), pf[u], o[d]);
        } else {
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            f16v bad = zero16();
#pragma unroll
            for (int u = 0; u < 2 * NB; ++u) {
              Frag<T> fin, oth;
              part_finite(Tl::column(vt, at, 16 * u, d), fin, oth);
              float ones[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) ones[j] = (seen[u >> 1] >> (8 * (u & 1) + j)) & 1u ? 1.f : 0.f;
              mma(fin, pf[u], o[d]);
              mma(oth, make_frag<T>(ones), bad);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
              o[d][i] = bad[i] > 0.f ? NAN : o[d][i];
          }
        }
      }
    }
    bool odd = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= non_finite(o[d][i]);
    return odd;
  };
  if (__syncthreads_or(pass(std::false_type{}))) pass(std::true_type{});

  l = half_sum(l);
  if constexpr (PARTS > 1) {
    // at the largest of the parts' maxima; the first part sums, in order, a block of 32 elements at a time
    float *red = (float *)&lds[0][0][0][0];
    static_assert(kWaves * 16 * PARLE_WAVE * 4 <= (int)sizeof(lds), "");
    __syncthreads();
    red[wave * PARLE_WAVE + lane] = m;
    __syncthreads();
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) most = fmaxf(most, red[(wave - part + i) * PARLE_WAVE + lane]);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - most);
    l *= f, m = most;
    __syncthreads();
    red[wave * PARLE_WAVE + lane] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) l += red[(wave - part + i) * PARLE_WAVE + lane];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 16; ++i) red[(wave * 16 + i) * PARLE_WAVE + lane] = o[d][i] * f;
      __syncthreads();
      if (part == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          o[d][i] *= f;
#pragma unroll
          for (int j = 1; j < PARTS; ++j) o[d][i] += red[((wave + j) * 16 + i) * PARLE_WAVE + lane];
        }
      }
    }
    if (part) return;
  }
  if (row >= g.tokens) return;
  // no sum: a row outside of every sequence, or one that sees scores of -inf only, whose softmax is not a number
  const float inv = l == 0.f ? (s.count ? NAN : 0.f) : 1.f / l;
  T *out = (T *)g.out + rep * g.out_stride + (long long)row * g.ld_out + (long long)head * g.dim;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int e = 32 * d + 8 * b + 4 * h;
      if (e < g.dim) store4(out + e, o[d][4 * b] * inv, o[d][4 * b + 1] * inv, o[d][4 * b + 2] * inv, o[d][4 * b + 3] * inv);
    }
  if (g.lse && h == 0) g.lse[((long long)rep * g.heads + head) * g.tokens + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace

hipError_t launch_attention_fwd(hipStream_t st, const parle_attention_desc &d, const void *q, const void *k, const void *v,
                                const int32_t *offsets, void *out, float *lse) {
  Args g{q,       k,      v,          offsets, out,        lse,     d.n,     d.tokens, d.sequences, d.heads, d.kv_heads,
         d.dim,   d.window, d.sinks, tok::ceil_div(d.tokens, kRows), d.scale, d.ld_q,  d.q_stride, d.ld_kv, d.kv_stride, d.ld_out, d.out_stride};
  const bool dma = direct(d.tokens, d.ld_kv, d.kv_stride, d.n, d.dtype ? 2 : 4);
  const bool few = shares_keys(d);
  if (few) g.tiles = tok::ceil_div(d.tokens, kRows / most_parts(d));
  auto go = [&](auto *kernel) {
    kernel<<<dim3(g.tiles * d.heads, d.n), kThreads, 0, st>>>(g);
    return hipGetLastError();
  };
#define PARLE_GO(T, DP, MOST) \
  (dma ? (few ? go(k_attn_fwd<T, DP, MOST, true>) : go(k_attn_fwd<T, DP, 1, true>)) : (few ? go(k_attn_fwd<T, DP, MOST, false>) : go(k_attn_fwd<T, DP, 1, false>)))
  if (d.dtype) return d.dim <= 64 ? PARLE_GO(bf16_t, 64, 4) : d.dim <= 96 ? PARLE_GO(bf16_t, 96, 4) : PARLE_GO(bf16_t, 128, 4);
  return d.dim <= 64 ? PARLE_GO(float, 64, 4) : PARLE_GO(float, 128, 2);
#undef PARLE_GO
}
