// Attention over packed sequences, backward.  With P = e^(scale s - lse) and dS = P * (dP - delta), dP = dO V^T, delta = rowsum(dO * O):
// dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
//
// Two kernels make the probabilities each for themselves: one owns rows of queries and walks over the keys they see (dQ, and delta on the
// way), one owns keys and walks over the queries that see them (dK, dV), of all query heads that share the keys.  So no sum crosses
// workgroups, nothing is added atomically, and results are the same every time; seven products instead of the five that one pass would take.
// Sinks behind a window are seen by far more queries than other keys.  What the queries beyond the reach of a sink's tile add to it is summed in chunks by
// workgroups of their own, into scratch, and joined behind.
//
// Measured, bf16: three replicas of 4096 tokens, 16 heads of 64 elements on 4 of keys, a window of 1024 and 4 sinks: 247 us, 0.51 PFLOP/s of the seven
// products, of which dQ takes 42 %, dK and dV 55 %, the sinks 3; 4099 tokens of 16 heads of 128 elements without a window 386 us, 0.63 PFLOP/s, 41 and 59 %.
// What bounds them is that matrix unit (30 and 27 to 47 % of the time), vector unit (24 to 45 %) and LDS (15 to 24 %) wait for one another: dK and dV of 128
// elements leave room for one wavefront on a SIMD, the others for two.  With one, the scalar operations in front of a step's loads count as well (1000 of
// 3900 cycles before all heads of a group shared a descriptor).
#include "attn.h"

namespace {

using namespace attn;

constexpr int kRows = 32 * kWaves;  // queries of a workgroup

struct BwdArgs {
  Args a;
  const void *dout;
  float *stats;  // [n][heads][2][tokens]: -lse log2(e), -delta
  // dK / scale and dV of sinks, [2][dim] each: of the queries of a chunk, for the sequence that the chunk begins in; and of the queries in front of a
  // sequence's first such chunk, by that chunk.  [n][kv_heads][chunks][sinks].
  float *far, *near;
  void *dq, *dk, *dv;
  int chunk, chunks;  // rows of a chunk, a multiple of kRows
};

// The first query that the workgroup of a key leaves to the chunks, for sinks.
__host__ __device__ __forceinline__ int reach(int key, int window, int chunk, int tokens) {
  const long long e = ((long long)(key / kRows + 1) * kRows - 1 + window + chunk - 1) / chunk * chunk;
  return (int)(e < tokens ? e : tokens);
}

// PARTS: as in the forward pass.
template <typename T, int DP, int PARTS, bool DMA>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 4 && DP == 128) || (PARTS > 1 && (sizeof(T) == 4 || DP > 64)) ? 1 : 2) void k_attn_dq(BwdArgs b) {
  const Args &g = b.a;
  using Tl = Tile<T, DP>;
  constexpr int BN = sizeof(T) == 2 && PARTS == 1 ? 64 : 32, NB = BN / 32, ND = DP / 32, NS = DP / 16, kQueries = kRows / PARTS;
  constexpr int kTileBytes = BN * Tl::kRowBytes;
  __shared__ __attribute__((aligned(1024))) char lds[2][PARTS][2][kTileBytes];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, part = wave % PARTS;
  const int hx = blockIdx.x % g.heads, kvh = hx % g.kv_heads, head = kvh * (g.heads / g.kv_heads) + hx / g.kv_heads;
  const int tile = g.tiles - 1 - blockIdx.x / g.heads, rep = blockIdx.y;
  const int32_t *offsets = g.offsets ? g.offsets + (long long)rep * (g.sequences + 1) : nullptr;
  const T *k = (const T *)g.k + rep * g.kv_stride + (long long)kvh * g.dim;
  const T *v = (const T *)g.v + rep * g.kv_stride + (long long)kvh * g.dim;

  const int r0 = tile * kQueries, w0 = r0 + wave / PARTS * 32, row = w0 + (lane & 31), rowc = min(row, g.tokens - 1);
  const Span cov = covered(offsets, g.sequences, g.tokens);
  Sight s = sight_of({0, 0}, 0, 0, 0);
  if (row < g.tokens) s = sight_of(span_of(offsets, g.sequences, g.tokens, row), row, g.window, g.sinks);
  const int rv0 = max(r0, cov.start), rv1 = min(r0 + kQueries, cov.end) - 1;
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
  if (row < g.tokens && h == 0 && part == 0) {
    float *to = b.stats + 2 * (stat - rowc) + rowc;
    to[0] = -lse2, to[g.tokens] = -delta;
  }

  Loader<T, DP, BN, DMA> kl, vl;
  kl.init(g.ld_kv, g.dim), vl.init(g.ld_kv, g.dim);
  kl.from(k, khi - 1), vl.from(v, khi - 1);
  typename Tl::Places pl;
  pl.init(lane);

  settle();
  const float c = g.scale * kLog2e;
  f16v dq[ND];
  auto pass = [&](auto safe) {  // as in the forward pass, for infinite and NaN keys
    constexpr bool SAFE = decltype(safe)::value;
#pragma unroll
    for (int d = 0; d < ND; ++d) dq[d] = zero16();
    auto base_of = [&](int t) { return t < nS ? s0 + t * BN : klo + (t - nS) * BN; };
    auto fetch = [&](int step) {
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
        const bool whole = all_in && t >= nS && kb + BN - 1 <= w0 && kb >= lo_last;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          f16v sc = zero16(), dp = zero16();
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            mma(Tl::row(kt, pl, 32 * n, i), qf[i], sc);
            mma(Tl::row(vt, pl, 32 * n, i), df[i], dp);
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
              if (SAFE) seen |= (uint32_t)ok << i;
              ds[i] = ok ? ds[i] : 0.f;
            }
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = ds[8 * u + j];
            const Frag<T> pf = make_frag<T>(p);
            if (!SAFE || whole) {
#pragma unroll
              for (int d = 0; d < ND; ++d) mma(Tl::column(kt, pl, 32 * n + 16 * u, d), pf, dq[d]);
            } else {
              float ones[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) ones[j] = (seen >> (8 * u + j)) & 1u ? 1.f : 0.f;
              const Frag<T> see = make_frag<T>(ones);
#pragma unroll
              for (int d = 0; d < ND; ++d) {
                Frag<T> fin, oth;
                part_finite(Tl::column(kt, pl, 32 * n + 16 * u, d), fin, oth);
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
    }
    bool odd = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= non_finite(dq[d][i]);
    return odd;
  };
  if (__syncthreads_or(pass(std::false_type{}))) pass(std::true_type{});
  if constexpr (PARTS > 1) {  // the parts' sums meet, in order
    float *red = (float *)&lds[0][0][0][0];
    static_assert(kWaves * 16 * PARLE_WAVE * 4 <= (int)sizeof(lds), "");
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 16; ++i) red[(wave * 16 + i) * PARLE_WAVE + lane] = dq[d][i];
      __syncthreads();
      if (part == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int j = 1; j < PARTS; ++j) dq[d][i] += red[((wave + j) * 16 + i) * PARLE_WAVE + lane];
      }
    }
    if (part) return;
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

// A wavefront owns 32 keys: K and V are fragments in registers, dK and dV accumulators, and 32 queries a step come through LDS, read as rows for
// S = Q K^T and dP = dO V^T and as columns for dV and dK.  PARTS wavefronts share keys: they take the steps in turn and their sums meet in LDS, so
// that a few keys, or few heads of keys, still make enough workgroups.  Behind the workgroups of keys come those of the sinks' chunks.
template <typename T, int DP, int PARTS, bool DMA>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 && DP == 64) ? 2 : 1) void k_attn_dkv(BwdArgs b) {
  const Args &g = b.a;
  using Tl = Tile<T, DP>;
  constexpr int BQ = 32, ND = DP / 32, NS = DP / 16, kKeys = kRows / PARTS;
  // Stages in LDS, of a tile for each part: one that is multiplied and kAhead on their way.
  constexpr int kTileBytes = BQ * Tl::kRowBytes, kStageBytes = PARTS * 2 * kTileBytes;
  constexpr int kRoom = (sizeof(T) == 2 && DP == 64 ? 72 : 136) << 10;  // two workgroups to a compute unit, or one
  constexpr int kBufs = !DMA || 3 * kStageBytes > kRoom ? 2 : 4 * kStageBytes > kRoom ? 3 : 4, kAhead = kBufs - 1;
  __shared__ __attribute__((aligned(1024))) char lds[kBufs][PARTS][2][kTileBytes];
  __shared__ __attribute__((aligned(16))) float stats[kBufs][kWaves][2][BQ];  // of each wavefront its own: -lse log2(e), -delta

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, part = wave % PARTS;
  const int kvh = blockIdx.x % g.kv_heads, rep = blockIdx.y, group = g.heads / g.kv_heads, key_tiles = g.tiles;
  const bool far = (int)(blockIdx.x / g.kv_heads) >= key_tiles;
  const int tile = blockIdx.x / g.kv_heads - (far ? key_tiles : 0);
  const int32_t *offsets = g.offsets ? g.offsets + (long long)rep * (g.sequences + 1) : nullptr;
  const T *k = (const T *)g.k + rep * g.kv_stride + (long long)kvh * g.dim;
  const T *v = (const T *)g.v + rep * g.kv_stride + (long long)kvh * g.dim;
  const Span cov = covered(offsets, g.sequences, g.tokens);

  // This lane's key, and the queries that see it: key .. hi.  Queries of the workgroup: [qlo, qhi).  slot: where sums of a sink go, or -1.
  int key = wave / PARTS * 32 + (lane & 31), hi = -1, qlo = 0, qhi = 0;
  long long slot = -1;
  bool all_in;
  if (far) {
    // workgroups of a chunk, one for kKeys sinks each
    const int blocks = (g.sinks + kKeys - 1) / kKeys, ch = tile / blocks, first = tile % blocks * kKeys, c0 = ch * b.chunk;
    const Span s = span_of(offsets, g.sequences, g.tokens, c0);
    const int sink = first + key;
    key = s.start + sink;
    if (sink < g.sinks && key < s.end && c0 >= reach(key, g.window, b.chunk, g.tokens)) {
      hi = s.end - 1;
      slot = (((long long)rep * g.kv_heads + kvh) * b.chunks + ch) * g.sinks + sink;
    }
    // the first sink has the least reach
    if (s.end > s.start && c0 >= reach(s.start + first, g.window, b.chunk, g.tokens)) qlo = c0, qhi = min(c0 + b.chunk, s.end);
    all_in = __all(hi >= 0);
  } else {
    const int k0 = tile * kKeys;
    key += k0;
    Span s = {0, 0};
    if (key < g.tokens) s = span_of(offsets, g.sequences, g.tokens, key);
    if (s.end > s.start) {
      hi = g.window > 0 && key - s.start >= g.sinks ? (int)min((long long)s.end, (long long)key + g.window) - 1 : s.end - 1;
      if (g.window > 0 && key - s.start < g.sinks) {
        const int r = reach(key, g.window, b.chunk, g.tokens), ch = (r + b.chunk - 1) / b.chunk;
        hi = min(hi, r - 1);
        if ((long long)ch * b.chunk < s.end) slot = (((long long)rep * g.kv_heads + kvh) * b.chunks + ch) * g.sinks + key - s.start;
      }
    }
    const int kv0 = max(k0, cov.start), kv1 = min(k0 + kKeys, cov.end) - 1;
    if (kv0 <= kv1) {
      const Span f = span_of(offsets, g.sequences, g.tokens, kv1);
      qlo = kv0;
      qhi = g.window > 0 ? (int)min((long long)f.end, (long long)kv1 + g.window) : f.end;
      if (g.window > 0 && max(f.start, kv0) - f.start < g.sinks) qhi = max(qhi, min(f.end, reach(kv1, g.window, b.chunk, g.tokens)));
    }
    all_in = key - (lane & 31) >= cov.start && key - (lane & 31) + 31 < cov.end;
  }
  qlo = __builtin_amdgcn_readfirstlane(qlo), qhi = __builtin_amdgcn_readfirstlane(qhi);
  int hi_least = hi, hi_most = hi;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) hi_least = min(hi_least, __shfl_xor(hi_least, o)), hi_most = max(hi_most, __shfl_xor(hi_most, o));
  hi_least = __builtin_amdgcn_readfirstlane(hi_least), hi_most = __builtin_amdgcn_readfirstlane(hi_most);
  const int key_first = __builtin_amdgcn_readfirstlane(key), key_last = key_first + 31;

  const int keyc = min(key, g.tokens - 1);
  Frag<T> kf[NS], vf[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    kf[i] = zero_frag<T>(), vf[i] = zero_frag<T>();
    const int at = 16 * i + 8 * h;
    if (at < g.dim) kf[i] = load_frag(k + (long long)keyc * g.ld_kv + at), vf[i] = load_frag(v + (long long)keyc * g.ld_kv + at);
  }

  settle();
  const float c = g.scale * kLog2e;
  const int each = (max(qhi - qlo, 0) + BQ - 1) / BQ, total = each * group;
  f16v dk[ND], dv[ND];
  Loader<T, DP, BQ, DMA> ql, dl;
  ql.init(g.ld_q, g.dim), dl.init(g.ld_out, g.dim);
  // the rows of all query heads that share the keys: a head is a column to begin at
  ql.from((const T *)g.q + rep * g.q_stride + (long long)kvh * group * g.dim, qhi - 1);
  dl.from((const T *)b.dout + rep * g.out_stride + (long long)kvh * group * g.dim, qhi - 1);
  constexpr int kLoads = PARTS * 2 * Loader<T, DP, BQ, DMA>::kLoads + 1;
  typename Tl::Places pl;
  pl.init(lane);

  // One step: 32 queries from `qb` on.  SAFE: infinite and NaN values of q and dout are taken out of masked tiles, as in the forward pass.
  auto add = [&](auto masked, auto safe, const char *qt, const char *dt, const float *st, int qb) {
    constexpr bool MASKED = decltype(masked)::value, SAFE = decltype(safe)::value;
    // Loads from LDS are put in front of what hides them: fragments of rows first, those of the first half's columns beside the products of rows,
    // those of the second half's beside the first half's products.
    f16v sc = zero16(), dp;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const f4 de = *(const f4 *)&st[BQ + 8 * n + 4 * h];
#pragma unroll
      for (int i = 0; i < 4; ++i) dp[4 * n + i] = de[i];
    }
    constexpr bool AHEAD = !(sizeof(T) == 4 && DP == 128);  // there is no room for them, and the instructions of fp32 are slow
    Frag<T> qr[NS], dr[NS], qc[2][ND], dc[2][ND];
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < NS; ++i) qr[i] = Tl::row(qt, pl, 0, i), dr[i] = Tl::row(dt, pl, 0, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    auto columns = [&](int u) {
#pragma unroll
      for (int d = 0; d < ND; ++d) dc[u][d] = Tl::column(dt, pl, 16 * u, d), qc[u][d] = Tl::column(qt, pl, 16 * u, d);
    };
    if constexpr (AHEAD) columns(0);
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      if constexpr (!AHEAD) {
        qr[i] = Tl::row(qt, pl, 0, i), dr[i] = Tl::row(dt, pl, 0, i);
        if (i % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
      mma(qr[i], kf[i], sc);
      mma(dr[i], vf[i], dp);
    }
    __builtin_amdgcn_sched_barrier(0);
    uint32_t seen = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float x[8], y[8];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const f4 ls = *(const f4 *)&st[8 * (2 * u + n) + 4 * h];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 4 * n + i, r = 8 * u + j;
          float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[r], c, ls[i])), ds = p * dp[r];
          if constexpr (MASKED) {
            const int row = qb + 8 * (r >> 2) + 4 * h + (r & 3);
            const bool ok = (row >= key) & (row <= hi);
            if (SAFE) seen |= (uint32_t)ok << r;
            p = ok ? p : 0.f, ds = ok ? ds : 0.f;
          }
          x[j] = p, y[j] = ds;
        }
      }
      const Frag<T> pf = make_frag<T>(x), sf = make_frag<T>(y);
      if (AHEAD && u == 0) columns(1);
      if constexpr (!(SAFE && MASKED)) {
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          if constexpr (!AHEAD) {
            dc[u][d] = Tl::column(dt, pl, 16 * u, d), qc[u][d] = Tl::column(qt, pl, 16 * u, d);
            __builtin_amdgcn_sched_barrier(0);
          }
          mma(dc[u][d], pf, dv[d]);
          mma(qc[u][d], sf, dk[d]);
        }
      } else {
        float ones[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) ones[j] = (seen >> (8 * u + j)) & 1u ? 1.f : 0.f;
        const Frag<T> see = make_frag<T>(ones);
        auto finite = [&](const Frag<T> &column, const Frag<T> &f, f16v &acc) {
          Frag<T> fin, oth;
          part_finite(column, fin, oth);
          f16v bad = zero16();
          mma(fin, f, acc);
          mma(oth, see, bad);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[i] = bad[i] > 0.f ? NAN : acc[i];
        };
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          if constexpr (!AHEAD) dc[u][d] = Tl::column(dt, pl, 16 * u, d), qc[u][d] = Tl::column(qt, pl, 16 * u, d);
          finite(dc[u][d], pf, dv[d]), finite(qc[u][d], sf, dk[d]);
        }
      }
    }
  };
  auto pass = [&](auto safe) {
#pragma unroll
    for (int d = 0; d < ND; ++d) dk[d] = zero16(), dv[d] = zero16();
    // the tile that is fetched next: query head of the group, first query; and this part's that is added next
    int fetch_head = -1, fetch_at = qhi, at = qlo + part * BQ;
    const float *sp = b.stats + (((long long)rep * g.heads + kvh * group) - 1) * 2 * g.tokens;
    auto fetch = [&](int buf) {
#pragma unroll
      for (int i = 0; i < PARTS; ++i) {
        if (fetch_at >= qhi) {
          if (fetch_head + 1 < group) ++fetch_head, sp += 2LL * g.tokens;  // behind the last tile, the last head's again, so that loads keep their count
          fetch_at = qlo;
        }
        ql.load(lds[buf][i][0], fetch_at, fetch_head * g.dim), dl.load(lds[buf][i][1], fetch_at, fetch_head * g.dim);
        if (i == part) {
          if constexpr (DMA)
            igemm_dev::dma4(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)&stats[buf][wave][0][0]),
                            igemm_dev::buffer_desc(sp, (uint32_t)g.tokens * 8u), (uint32_t)((lane >> 5) * g.tokens + fetch_at + (lane & 31)) * 4u);
          else
            stats[buf][wave][lane >> 5][lane & 31] = sp[(long long)(lane >> 5) * g.tokens + min(fetch_at + (lane & 31), qhi - 1)];
        }
        fetch_at += BQ;
      }
    };
    if (total > 0)
      for (int i = 0; i < kAhead; ++i) fetch(i);
    int buf = 0;
    // a part's tiles of a head follow on those of the head before without a gap, so it steps over heads' ends by itself
    for (int t = part; t < total + part; t += PARTS) {
      while (at >= qhi) at -= each * BQ;
      arrive<DMA ? (kAhead - 1) * kLoads : 0>();
      fetch(buf == 0 ? kBufs - 1 : buf - 1);
      if ((t < total) & (at + BQ > key_first) & (at <= hi_most)) {
        const char *qt = lds[buf][part][0], *dt = lds[buf][part][1];
        const float *st = &stats[buf][wave][0][0];
        if (all_in & (at >= key_last) & (at + BQ - 1 <= hi_least))
          add(std::false_type{}, safe, qt, dt, st, at);
        else
          add(std::true_type{}, safe, qt, dt, st, at);
      }
      at += PARTS * BQ;
      buf = buf + 1 < kBufs ? buf + 1 : 0;
    }
    arrive<0>();  // nothing lands in LDS later
    bool odd = false;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= non_finite(dk[d][i]) | non_finite(dv[d][i]);
    return odd;
  };
  if (__syncthreads_or(pass(std::false_type{}))) pass(std::true_type{});

  // the parts' sums meet in the first part's registers, in order, a block of 32 elements at a time
  if constexpr (PARTS > 1) {
    float *red = (float *)&lds[0][0][0][0] + wave / PARTS * (2 * 16 * PARLE_WAVE);
    static_assert(kWaves / PARTS * 2 * 16 * PARLE_WAVE * 4 <= (int)sizeof(lds), "");
#pragma unroll
    for (int d = 0; d < ND; ++d)
      for (int from = 1; from < PARTS; ++from) {
        __syncthreads();
        if (part == from) {
#pragma unroll
          for (int i = 0; i < 16; ++i) red[i * PARLE_WAVE + lane] = dk[d][i], red[(16 + i) * PARLE_WAVE + lane] = dv[d][i];
        }
        __syncthreads();
        if (part == 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) dk[d][i] += red[i * PARLE_WAVE + lane], dv[d][i] += red[(16 + i) * PARLE_WAVE + lane];
        }
      }
    if (part) return;
  }
  if (far ? slot < 0 : key >= g.tokens) return;
  T *dkr = (T *)b.dk + rep * g.kv_stride + (long long)key * g.ld_kv + (long long)kvh * g.dim;
  T *dvr = (T *)b.dv + rep * g.kv_stride + (long long)key * g.ld_kv + (long long)kvh * g.dim;
  float *to = (far ? b.far : b.near) + (slot < 0 ? 0 : slot) * 2 * g.dim;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int at = 32 * d + 8 * n + 4 * h;
      if (at >= g.dim) continue;
      const f4 x = {dk[d][4 * n], dk[d][4 * n + 1], dk[d][4 * n + 2], dk[d][4 * n + 3]};
      const f4 y = {dv[d][4 * n], dv[d][4 * n + 1], dv[d][4 * n + 2], dv[d][4 * n + 3]};
      if (slot >= 0) {
        *(f4 *)(to + at) = x, *(f4 *)(to + g.dim + at) = y;
      } else {
        store4(dkr + at, x[0] * g.scale, x[1] * g.scale, x[2] * g.scale, x[3] * g.scale);
        store4(dvr + at, y[0], y[1], y[2], y[3]);
      }
    }
}

// The sinks of a sequence: what their own workgroup and the chunks behind its reach have summed, in order.  All latency: 7 us for up to 32 chunks.
// One workgroup of keys for all queries of a sink would take as long as the whole rest.  The workgroup of a chunk sees to the sinks
// whose first chunk it is; a thread takes four elements of dK or of dV.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sinks(BwdArgs b) {
  const Args &g = b.a;
  const int kvh = blockIdx.x % g.kv_heads, ch = blockIdx.x / g.kv_heads, rep = blockIdx.y;
  const int32_t *offsets = g.offsets ? g.offsets + (long long)rep * (g.sequences + 1) : nullptr;
  const Span s = span_of(offsets, g.sequences, g.tokens, ch * b.chunk);
  const long long first = (((long long)rep * g.kv_heads + kvh) * b.chunks + ch) * g.sinks, step = (long long)g.sinks * 2 * g.dim;
  const int per = g.dim / 2;  // pieces of four of a sink's dK and dV
  for (int it = threadIdx.x; it < g.sinks * per; it += 256) {
    const int sink = it / per, e = (it - sink * per) * 4, key = s.start + sink;
    if (key >= s.end || (reach(key, g.window, b.chunk, g.tokens) + b.chunk - 1) / b.chunk != ch) continue;
    const float *p = b.far + (first + sink) * 2 * g.dim + e;
    f4 x = *(const f4 *)(b.near + (first + sink) * 2 * g.dim + e);
    for (long long i = ch; i * b.chunk < s.end; ++i, p += step) x += *(const f4 *)p;
    const bool is_v = e >= g.dim;
    T *to = (T *)(is_v ? b.dv : b.dk) + rep * g.kv_stride + (long long)key * g.ld_kv + (long long)kvh * g.dim + (is_v ? e - g.dim : e);
    const float f = is_v ? 1.f : g.scale;
    store4(to, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
  }
}

// Chunks of 128 queries, longer where there were more than 64 of them: what a chunk sums is written and read again.
int chunk_of(const parle_attention_desc &d) { return kRows * tok::ceil_div(tok::ceil_div(d.tokens, kRows), 64); }
bool has_far(const parle_attention_desc &d) { return d.window > 0 && d.sinks > 0 && reach(0, d.window, chunk_of(d), d.tokens) < d.tokens; }
int64_t stats_bytes(const parle_attention_desc &d) { return tok::round_up((long long)d.n * d.heads * d.tokens * 8, 256); }
int64_t far_elems(const parle_attention_desc &d) {
  return has_far(d) ? (int64_t)d.n * d.kv_heads * tok::ceil_div(d.tokens, chunk_of(d)) * d.sinks * 2 * d.dim : 0;
}
// Wavefronts that share keys: two, or four where two make fewer workgroups than the chip has places (and LDS holds the tiles of four).  Eight heads of
// 8192 tokens, 64 elements each, take 331 us with two and 363 with four, 1000 tokens of eight heads that share one, 128 elements each, 81 and 67.
int parts_of(const parle_attention_desc &d) {
  const long long wgs = (long long)d.n * d.kv_heads * tok::ceil_div(d.tokens, kRows / 2), places = d.dtype && d.dim <= 64 ? 512 : 256;
  return wgs >= places || (!d.dtype && d.dim > 64) ? 2 : 4;
}

// Workgroups of k_attn_dkv, of a replica: of keys, and of the sinks' chunks.
int64_t dkv_workgroups(const parle_attention_desc &d) {
  const int keys = kRows / parts_of(d);
  return ((int64_t)tok::ceil_div(d.tokens, keys) + (has_far(d) ? (int64_t)tok::ceil_div(d.tokens, chunk_of(d)) * tok::ceil_div(d.sinks, keys) : 0)) * d.kv_heads;
}

}  // namespace

bool attention_bwd_fits(const parle_attention_desc &d) { return d.tokens == 0 || dkv_workgroups(d) * kThreads < 1LL << 32; }

int64_t attention_scratch_bytes(const parle_attention_desc &d) { return d.tokens == 0 ? 0 : stats_bytes(d) + 2 * far_elems(d) * 4; }

hipError_t launch_attention_bwd(hipStream_t st, const parle_attention_desc &d, const void *q, const void *k, const void *v,
                                const int32_t *offsets, const void *out, const float *lse, const void *dout, void *scratch, void *dq, void *dk,
                                void *dv) {
  const int tiles = tok::ceil_div(d.tokens, kRows), chunk = chunk_of(d), chunks = tok::ceil_div(d.tokens, chunk), parts = parts_of(d);
  const bool far = has_far(d);
  float *fp = far ? (float *)((char *)scratch + stats_bytes(d)) : nullptr;
  BwdArgs b{{q, k, v, offsets, (void *)out, (float *)lse, d.n, d.tokens, d.sequences, d.heads, d.kv_heads, d.dim, d.window, d.sinks, tiles, d.scale,
             d.ld_q, d.q_stride, d.ld_kv, d.kv_stride, d.ld_out, d.out_stride},
            dout, (float *)scratch, fp, far ? fp + far_elems(d) : nullptr, dq, dk, dv, chunk, chunks};
  const int size = d.dtype ? 2 : 4;
  const bool dma = direct(d.tokens, d.ld_kv, d.kv_stride, d.n, size) && direct(d.tokens, d.ld_q, d.q_stride, d.n, size) &&
                   direct(d.tokens, d.ld_out, d.out_stride, d.n, size);
  const bool few = shares_keys(d);  // as in the forward pass; 4096 tokens of 8 heads of 64 elements, bf16, the whole gradient: 139 us without, 115 with
  auto go = [&](auto *of_queries, auto *of_keys, auto *of_sinks) {
    b.a.tiles = tok::ceil_div(d.tokens, few ? kRows / most_parts(d) : kRows);
    of_queries<<<dim3(b.a.tiles * d.heads, d.n), kThreads, 0, st>>>(b);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    b.a.tiles = tok::ceil_div(d.tokens, kRows / parts);
    of_keys<<<dim3((uint32_t)dkv_workgroups(d), d.n), kThreads, 0, st>>>(b);
    e = hipGetLastError();
    if (e != hipSuccess || !far) return e;
    of_sinks<<<dim3(chunks * d.kv_heads, d.n), 256, 0, st>>>(b);
    return hipGetLastError();
  };
#define PARLE_QUERIES(T, DP, MOST, DMA) (few ? k_attn_dq<T, DP, MOST, DMA> : k_attn_dq<T, DP, 1, DMA>)
#define PARLE_KEYS(T, DP, MOST, DMA) (parts == 2 ? k_attn_dkv<T, DP, 2, DMA> : k_attn_dkv<T, DP, MOST, DMA>)
#define PARLE_GO(T, DP, MOST)                                                                  \
  (dma ? go(PARLE_QUERIES(T, DP, MOST, true), PARLE_KEYS(T, DP, MOST, true), k_attn_sinks<T>) \
       : go(PARLE_QUERIES(T, DP, MOST, false), PARLE_KEYS(T, DP, MOST, false), k_attn_sinks<T>))
  if (d.dtype) return d.dim <= 64 ? PARLE_GO(bf16_t, 64, 4) : d.dim <= 96 ? PARLE_GO(bf16_t, 96, 4) : PARLE_GO(bf16_t, 128, 4);
  return d.dim <= 64 ? PARLE_GO(float, 64, 4) : PARLE_GO(float, 128, 2);
#undef PARLE_KEYS
#undef PARLE_QUERIES
#undef PARLE_GO
}
