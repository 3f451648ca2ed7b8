// Attention over packed sequences, backward.  With P = e^(scale s - lse) and dS = P * (dP - delta), dP = dO V^T, delta = rowsum(dO * O):
// dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
//
// Two kernels make the probabilities each for themselves: one owns rows of queries and walks over the keys they see (dQ, and delta on the
// way), one owns keys and walks over the queries that see them (dK, dV), of all query heads that share the keys.  So no sum crosses
// workgroups, nothing is added atomically, and results are the same every time; seven products instead of the five that one pass would take.
// Sinks behind a window are seen by far more queries than other keys.  What chunks of kChunk queries beyond the reach of a sink's tile add to it is summed
// by workgroups of their own, in front, into scratch.
#include "attn.h"

namespace {

using namespace attn;

constexpr int kRows = 32 * kWaves;  // queries, or keys, of a workgroup
constexpr int kChunk = 512;

struct BwdArgs {
  Args a;
  const void *dout;
  float *delta;    // [n][heads][tokens]
  float *far;      // [n][kv_heads][chunks][sinks][2][dim]: dK / scale and dV of the sinks of the sequence that a chunk begins in
  void *dq, *dk, *dv;
  int chunks;
};

// The first query that the workgroup of key tile `t` leaves to the chunks, for sinks.
__host__ __device__ __forceinline__ int reach(int t, int window, int tokens) {
  const long long e = ((long long)(t + 1) * kRows - 1 + window + kChunk - 1) / kChunk * kChunk;
  return (int)(e < tokens ? e : tokens);
}

template <typename T, int DP>
__global__ __launch_bounds__(kThreads, 2) void k_attn_dq(BwdArgs b) {
  const Args &g = b.a;
  using Tl = Tile<T, DP>;
  constexpr int BN = sizeof(T) == 2 ? 64 : 32, NB = BN / 32, ND = DP / 32, NS = DP / 16;
  constexpr int kTileBytes = BN * Tl::kRowBytes;
  __shared__ __attribute__((aligned(1024))) char lds[2][2][kTileBytes];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
  const int hx = blockIdx.x % g.heads, kvh = hx % g.kv_heads, head = kvh * (g.heads / g.kv_heads) + hx / g.kv_heads;
  const int tile = g.tiles - 1 - blockIdx.x / g.heads, rep = blockIdx.y;
  const int32_t *offsets = g.offsets ? g.offsets + (long long)rep * (g.sequences + 1) : nullptr;
  const T *k = (const T *)g.k + rep * g.kv_stride + (long long)kvh * g.dim;
  const T *v = (const T *)g.v + rep * g.kv_stride + (long long)kvh * g.dim;

  const int r0 = tile * kRows, w0 = r0 + wave * 32, row = w0 + (lane & 31), rowc = min(row, g.tokens - 1);
  const Span cov = covered(offsets, g.sequences, g.tokens);
  Sight s = sight_of({0, 0}, 0, 0, 0);
  if (row < g.tokens) s = sight_of(span_of(offsets, g.sequences, g.tokens, row), row, g.window, g.sinks);
  const int rv0 = max(r0, cov.start), rv1 = min(r0 + kRows, cov.end) - 1;
  int klo = 0, khi = 0, s0 = 0, s1 = 0;  // as in the forward pass
  if (rv0 <= rv1) {
    const Sight f = sight_of(span_of(offsets, g.sequences, g.tokens, rv0), rv0, g.window, g.sinks);
    if (f.count) klo = f.lo, khi = rv1 + 1, s0 = f.start, s1 = min(f.start + (int)f.sinks, f.lo);
  }
  klo = __builtin_amdgcn_readfirstlane(klo), khi = __builtin_amdgcn_readfirstlane(khi);
  s0 = __builtin_amdgcn_readfirstlane(s0), s1 = __builtin_amdgcn_readfirstlane(s1);
  const int nS = s1 > s0 ? (s1 - s0 + BN - 1) / BN : 0, total = nS + (khi - klo + BN - 1) / BN;
  const bool all_in = w0 >= cov.start && w0 + 31 < cov.end;
  const int lo_first = __builtin_amdgcn_readlane(s.lo, 0), lo_last = __builtin_amdgcn_readlane(s.lo, 31);
  const int sink_first = __builtin_amdgcn_readlane(s.start, 0) + g.sinks;

  const T *qrow = (const T *)g.q + rep * g.q_stride + (long long)head * g.dim + (long long)rowc * g.ld_q;
  const T *drow = (const T *)b.dout + rep * g.out_stride + (long long)head * g.dim + (long long)rowc * g.ld_out;
  const T *orow = (const T *)g.out + rep * g.out_stride + (long long)head * g.dim + (long long)rowc * g.ld_out;
  Frag<T> qf[NS], df[NS];
  float delta = 0.f;
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    qf[i] = zero_frag<T>(), df[i] = zero_frag<T>();
    const int at = 16 * i + 8 * h;
    if (at < g.dim) {
      qf[i] = load_frag(qrow + at), df[i] = load_frag(drow + at);
      const Frag<T> of = load_frag(orow + at);
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = __builtin_fmaf(frag_at(df[i], j), frag_at(of, j), delta);
    }
  }
  delta = half_sum(delta);
  const long long stat = ((long long)rep * g.heads + head) * g.tokens + rowc;
  const float lse2 = g.lse[stat] * kLog2e;
  if (row < g.tokens && h == 0) b.delta[stat] = delta;

  const float c = g.scale * kLog2e;
  f16v dq[ND];
  for (int safe = 0;; ++safe) {  // as in the forward pass, for infinite and NaN keys
#pragma unroll
    for (int d = 0; d < ND; ++d) dq[d] = zero16();
    Rows<T, DP, BN> kr, vr;
    auto base_of = [&](int t) { return t < nS ? s0 + t * BN : klo + (t - nS) * BN; };
    auto fetch = [&](int t) {
      const int at = base_of(t), last = (t < nS ? s1 : khi) - 1;
      kr.load(k, g.ld_kv, at, last, g.dim, tid);
      vr.load(v, g.ld_kv, at, last, g.dim, tid);
    };
    if (total > 0) {
      fetch(0);
      kr.store(lds[0][0], tid), vr.store(lds[0][1], tid);
    }
    __syncthreads();
    for (int t = 0; t < total; ++t) {
      if (t + 1 < total) fetch(t + 1);
      const int kb = base_of(t);
      const char *kt = lds[t & 1][0], *vt = lds[t & 1][1];
      const bool none = kb > w0 + 31 || (all_in && t >= nS && kb + BN - 1 < lo_first && kb >= sink_first);
      if (!none) {
        const bool whole = all_in && t >= nS && kb + BN - 1 <= w0 && kb >= lo_last;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          f16v sc = zero16(), dp = zero16();
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            mma(Tl::row(kt, 32 * n + (lane & 31), 2 * i + h), qf[i], sc);
            mma(Tl::row(vt, 32 * n + (lane & 31), 2 * i + h), df[i], dp);
          }
          float ds[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) ds[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], c, -lse2)) * (dp[i] - delta);
          uint32_t seen = 0;
          if (!whole) {
            const Sight now = t < nS ? only_sinks(s, s1) : s;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const bool ok = now.sees(kb + 32 * n + 8 * (i >> 2) + 4 * h + (i & 3));
              seen |= (uint32_t)ok << i;
              ds[i] = ok ? ds[i] : 0.f;
            }
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = ds[8 * u + j];
            const Frag<T> pf = make_frag<T>(p);
            if (!(safe && !whole)) {
#pragma unroll
              for (int d = 0; d < ND; ++d) mma(Tl::column(kt, 32 * n + 16 * u, d, lane), pf, dq[d]);
            } else {
              float ones[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) ones[j] = (seen >> (8 * u + j)) & 1u ? 1.f : 0.f;
              const Frag<T> see = make_frag<T>(ones);
#pragma unroll
              for (int d = 0; d < ND; ++d) {
                Frag<T> fin, oth;
                part_finite(Tl::column(kt, 32 * n + 16 * u, d, lane), fin, oth);
                f16v bad = zero16();
                mma(fin, pf, dq[d]);
                mma(oth, see, bad);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  dq[d][i] = bad[i] > 0.f ? NAN : dq[d][i];
              }
            }
          }
        }
      }
      if (t + 1 < total) kr.store(lds[(t + 1) & 1][0], tid), vr.store(lds[(t + 1) & 1][1], tid);
      __syncthreads();
    }
    bool odd = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= non_finite(dq[d][i]);
    if (safe || !__syncthreads_or(odd)) break;
  }
  if (row >= g.tokens) return;
  T *out = (T *)b.dq + rep * g.q_stride + (long long)row * g.ld_q + (long long)head * g.dim;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int at = 32 * d + 8 * n + 4 * h;
      if (at < g.dim)
        store4(out + at, dq[d][4 * n] * g.scale, dq[d][4 * n + 1] * g.scale, dq[d][4 * n + 2] * g.scale, dq[d][4 * n + 3] * g.scale);
    }
}

// FAR: the keys are the sinks of the sequence that a chunk of queries begins in.
template <typename T, int DP, bool FAR>
__global__ __launch_bounds__(kThreads, 1) void k_attn_dkv(BwdArgs b) {
  const Args &g = b.a;
  using Tl = Tile<T, DP>;
  constexpr int BQ = 32, ND = DP / 32, NS = DP / 16;
  constexpr int kTileBytes = BQ * Tl::kRowBytes;
  __shared__ __attribute__((aligned(1024))) char lds[2][2][kTileBytes];
  __shared__ __attribute__((aligned(16))) float stats[2][2][BQ];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
  const int kvh = blockIdx.x % g.kv_heads, tile = blockIdx.x / g.kv_heads, rep = blockIdx.y, group = g.heads / g.kv_heads;
  const int32_t *offsets = g.offsets ? g.offsets + (long long)rep * (g.sequences + 1) : nullptr;
  const T *k = (const T *)g.k + rep * g.kv_stride + (long long)kvh * g.dim;
  const T *v = (const T *)g.v + rep * g.kv_stride + (long long)kvh * g.dim;
  const Span cov = covered(offsets, g.sequences, g.tokens);

  // This lane's key, and the queries that see it: key .. hi.  Queries of the workgroup: [qlo, qhi).
  int key, hi = -1, qlo = 0, qhi = 0, sink = 0x7fffffff, end = 0;
  bool all_in;
  if constexpr (FAR) {
    const int c0 = tile * kChunk;
    const Span s = span_of(offsets, g.sequences, g.tokens, c0);
    key = s.start + wave * 32 + (lane & 31);
    if (key < s.start + g.sinks && key < s.end && c0 >= reach(key / kRows, g.window, g.tokens)) hi = s.end - 1;
    // the first sink's tile has the least reach
    if (s.end > s.start && c0 >= reach(s.start / kRows, g.window, g.tokens)) qlo = c0, qhi = min(c0 + kChunk, s.end);
    all_in = __all(hi >= 0);
  } else {
    const int k0 = tile * kRows;
    key = k0 + wave * 32 + (lane & 31);
    Span s = {0, 0};
    if (key < g.tokens) s = span_of(offsets, g.sequences, g.tokens, key);
    if (s.end > s.start) {
      end = s.end;
      hi = g.window > 0 && key - s.start >= g.sinks ? (int)min((long long)s.end, (long long)key + g.window) - 1 : s.end - 1;
      if (g.window > 0 && key - s.start < g.sinks) sink = key - s.start, hi = min(hi, max(reach(tile, g.window, g.tokens), key + 1) - 1);
    }
    const int kv0 = max(k0, cov.start), kv1 = min(k0 + kRows, cov.end) - 1;
    if (kv0 <= kv1) {
      const Span f = span_of(offsets, g.sequences, g.tokens, kv1);
      qlo = kv0;
      qhi = g.window > 0 ? (int)min((long long)f.end, (long long)kv1 + g.window) : f.end;
      if (g.window > 0 && max(f.start, kv0) - f.start < g.sinks) qhi = max(qhi, min(f.end, reach(tile, g.window, g.tokens)));
    }
    all_in = key - (lane & 31) >= cov.start && key - (lane & 31) + 31 < cov.end;
  }
  qlo = __builtin_amdgcn_readfirstlane(qlo), qhi = __builtin_amdgcn_readfirstlane(qhi);
  int hi_least = hi, hi_most = hi, key_last = key;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) hi_least = min(hi_least, __shfl_xor(hi_least, o)), hi_most = max(hi_most, __shfl_xor(hi_most, o));
  hi_least = __builtin_amdgcn_readfirstlane(hi_least), hi_most = __builtin_amdgcn_readfirstlane(hi_most);
  key_last = __builtin_amdgcn_readlane(key, 31);
  const int key_first = __builtin_amdgcn_readfirstlane(key);

  const int keyc = min(key, g.tokens - 1);
  Frag<T> kf[NS], vf[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    kf[i] = zero_frag<T>(), vf[i] = zero_frag<T>();
    const int at = 16 * i + 8 * h;
    if (at < g.dim) kf[i] = load_frag(k + (long long)keyc * g.ld_kv + at), vf[i] = load_frag(v + (long long)keyc * g.ld_kv + at);
  }

  const float c = g.scale * kLog2e;
  const int each = (max(qhi - qlo, 0) + BQ - 1) / BQ, total = each * group;
  f16v dk[ND], dv[ND];
  for (int safe = 0;; ++safe) {  // as in the forward pass, for infinite and NaN rows of q and dout
#pragma unroll
    for (int d = 0; d < ND; ++d) dk[d] = zero16(), dv[d] = zero16();
    Rows<T, DP, BQ> qr, dr;
    float st = 0.f;
    auto fetch = [&](int t) {
      const int head = kvh * group + t / each, at = qlo + t % each * BQ;
      qr.load((const T *)g.q + rep * g.q_stride + (long long)head * g.dim, g.ld_q, at, qhi - 1, g.dim, tid);
      dr.load((const T *)b.dout + rep * g.out_stride + (long long)head * g.dim, g.ld_out, at, qhi - 1, g.dim, tid);
      if (tid < 2 * BQ) {
        const long long i = ((long long)rep * g.heads + head) * g.tokens + min(at + (tid & (BQ - 1)), qhi - 1);
        st = tid < BQ ? g.lse[i] * kLog2e : b.delta[i];
      }
    };
    auto put = [&](int buf) {
      qr.store(lds[buf][0], tid), dr.store(lds[buf][1], tid);
      if (tid < 2 * BQ) stats[buf][tid / BQ][tid & (BQ - 1)] = st;
    };
    if (total > 0) fetch(0), put(0);
    __syncthreads();
    for (int t = 0; t < total; ++t) {
      if (t + 1 < total) fetch(t + 1);
      const int qb = qlo + t % each * BQ;
      const char *qt = lds[t & 1][0], *dt = lds[t & 1][1];
      if (qb + BQ > key_first && qb <= hi_most) {
        f16v sc = zero16(), dp = zero16();
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          mma(Tl::row(qt, lane & 31, 2 * i + h), kf[i], sc);
          mma(Tl::row(dt, lane & 31, 2 * i + h), vf[i], dp);
        }
        float p[16], ds[16];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const f4 ls = *(const f4 *)&stats[t & 1][0][8 * n + 4 * h], de = *(const f4 *)&stats[t & 1][1][8 * n + 4 * h];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[4 * n + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * n + i], c, -ls[i]));
            ds[4 * n + i] = p[4 * n + i] * (dp[4 * n + i] - de[i]);
          }
        }
        const bool whole = all_in && qb >= key_last && qb + BQ - 1 <= hi_least;
        uint32_t seen = 0;
        if (!whole) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = qb + 8 * (i >> 2) + 4 * h + (i & 3);
            const bool ok = (row >= key) & (row <= hi);
            seen |= (uint32_t)ok << i;
            p[i] = ok ? p[i] : 0.f, ds[i] = ok ? ds[i] : 0.f;
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float x[8], y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = p[8 * u + j], y[j] = ds[8 * u + j];
          const Frag<T> pf = make_frag<T>(x), sf = make_frag<T>(y);
          if (!(safe && !whole)) {
#pragma unroll
            for (int d = 0; d < ND; ++d) {
              mma(Tl::column(dt, 16 * u, d, lane), pf, dv[d]);
              mma(Tl::column(qt, 16 * u, d, lane), sf, dk[d]);
            }
          } else {
            float ones[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) ones[j] = (seen >> (8 * u + j)) & 1u ? 1.f : 0.f;
            const Frag<T> see = make_frag<T>(ones);
            auto add = [&](const char *tile, const Frag<T> &f, f16v &acc, int d) {
              Frag<T> fin, oth;
              part_finite(Tl::column(tile, 16 * u, d, lane), fin, oth);
              f16v bad = zero16();
              mma(fin, f, acc);
              mma(oth, see, bad);
#pragma unroll
              for (int i = 0; i < 16; ++i)
                acc[i] = bad[i] > 0.f ? NAN : acc[i];
            };
#pragma unroll
            for (int d = 0; d < ND; ++d) add(dt, pf, dv[d], d), add(qt, sf, dk[d], d);
          }
        }
      }
      if (t + 1 < total) put((t + 1) & 1);
      __syncthreads();
    }
    bool odd = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= non_finite(dk[d][i]) | non_finite(dv[d][i]);
    if (safe || !__syncthreads_or(odd)) break;
  }

  // [2][dim] of a sink, of chunk 0
  float *far = b.far ? b.far + ((long long)rep * g.kv_heads + kvh) * b.chunks * g.sinks * 2 * g.dim : nullptr;
  const long long far_chunk = (long long)g.sinks * 2 * g.dim;
  if constexpr (FAR) {
    if (hi < 0) return;
    far += tile * far_chunk + (long long)(wave * 32 + (lane & 31)) * 2 * g.dim;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int at = 32 * d + 8 * n + 4 * h;
        if (at < g.dim) {
          *(f4 *)(far + at) = f4{dk[d][4 * n], dk[d][4 * n + 1], dk[d][4 * n + 2], dk[d][4 * n + 3]};
          *(f4 *)(far + g.dim + at) = f4{dv[d][4 * n], dv[d][4 * n + 1], dv[d][4 * n + 2], dv[d][4 * n + 3]};
        }
      }
  } else {
    if (key >= g.tokens) return;
    const int first = sink < g.sinks ? (reach(tile, g.window, g.tokens) + kChunk - 1) / kChunk : 0x7fffffff;
    T *dkr = (T *)b.dk + rep * g.kv_stride + (long long)key * g.ld_kv + (long long)kvh * g.dim;
    T *dvr = (T *)b.dv + rep * g.kv_stride + (long long)key * g.ld_kv + (long long)kvh * g.dim;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int at = 32 * d + 8 * n + 4 * h;
        if (at < g.dim) {
          f4 x = {dk[d][4 * n], dk[d][4 * n + 1], dk[d][4 * n + 2], dk[d][4 * n + 3]};
          f4 y = {dv[d][4 * n], dv[d][4 * n + 1], dv[d][4 * n + 2], dv[d][4 * n + 3]};
          for (long long ch = first; ch * kChunk < end; ++ch) {
            x += *(const f4 *)(far + ch * far_chunk + (long long)sink * 2 * g.dim + at);
            y += *(const f4 *)(far + ch * far_chunk + (long long)sink * 2 * g.dim + g.dim + at);
          }
          store4(dkr + at, x[0] * g.scale, x[1] * g.scale, x[2] * g.scale, x[3] * g.scale);
          store4(dvr + at, y[0], y[1], y[2], y[3]);
        }
      }
  }
}

bool has_far(const parle_attention_desc &d) { return d.window > 0 && d.sinks > 0 && reach(0, d.window, d.tokens) < d.tokens; }
int64_t delta_bytes(const parle_attention_desc &d) { return tok::round_up((long long)d.n * d.heads * d.tokens * 4, 256); }

}  // namespace

int64_t attention_scratch_bytes(const parle_attention_desc &d) {
  if (d.tokens == 0) return 0;
  const int64_t far = has_far(d) ? (int64_t)d.n * d.kv_heads * tok::ceil_div(d.tokens, kChunk) * d.sinks * 2 * d.dim * 4 : 0;
  return delta_bytes(d) + far;
}

hipError_t launch_attention_bwd(hipStream_t st, const parle_attention_desc &d, const void *q, const void *k, const void *v,
                                const int32_t *offsets, const void *out, const float *lse, const void *dout, void *scratch, void *dq, void *dk,
                                void *dv) {
  const int tiles = tok::ceil_div(d.tokens, kRows), chunks = tok::ceil_div(d.tokens, kChunk);
  const bool far = has_far(d);
  BwdArgs b{{q, k, v, offsets, (void *)out, (float *)lse, d.n, d.tokens, d.sequences, d.heads, d.kv_heads, d.dim, d.window, d.sinks, tiles, d.scale,
             d.ld_q, d.q_stride, d.ld_kv, d.kv_stride, d.ld_out, d.out_stride},
            dout, (float *)scratch, far ? (float *)((char *)scratch + delta_bytes(d)) : nullptr, dq, dk, dv, chunks};
  auto go = [&](auto *of_queries, auto *of_sinks, auto *of_keys) {
    of_queries<<<dim3(tiles * d.heads, d.n), kThreads, 0, st>>>(b);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && far) {
      of_sinks<<<dim3(chunks * d.kv_heads, d.n), kThreads, 0, st>>>(b);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    of_keys<<<dim3(tiles * d.kv_heads, d.n), kThreads, 0, st>>>(b);
    return hipGetLastError();
  };
#define PARLE_GO(T, DP) go(k_attn_dq<T, DP>, k_attn_dkv<T, DP, true>, k_attn_dkv<T, DP, false>)
  if (d.dtype) return d.dim <= 64 ? PARLE_GO(bf16_t, 64) : d.dim <= 96 ? PARLE_GO(bf16_t, 96) : PARLE_GO(bf16_t, 128);
  return d.dim <= 64 ? PARLE_GO(float, 64) : PARLE_GO(float, 128);
#undef PARLE_GO
}
