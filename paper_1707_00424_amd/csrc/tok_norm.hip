// Root-mean-square norm behind a residual addition, its result in the activation format or in 8 bits with a scale for
// 128 values of a row, and its gradient.
//
//   h = x + resid,  rstd = 1 / sqrt(mean h^2 + eps),  y = w h rstd
//   g = dy w,       dx = rstd (g - h rstd^2 mean(g h)) + dresid,   dw = sum over rows of dy h rstd
//
// Both directions read a row once into registers, reduce over it, and write: what they must move is what they move, and memory bounds
// them.  A row belongs to a group of LANES threads, each with CH vectors of eight elements, LANES * 8 elements apart; the fewest threads
// whose registers hold a row are taken, so that most lanes have work and most rows are in flight (12.6 M elements bf16 in rows of 256: 17 us
// with 32 threads a row, 24 with 64).
// 8192 rows of 4096 bf16 forward: 47 us, 5.0 TB/s, the rate of a plain copy; 8 rows 4.4 us, latency.  3 x 4099 rows of 2048
// backward: 47 us, 4.3 TB/s, 5 of them the join of dw; without the next row's loads ahead 57.
//
// Results may be written over what they come from (h or y over x or resid, dx over h, dout or dresid).  Threads at a row's end load
// elements that are their neighbours' too (Place), so those are not stored before the barrier in the row's sum, which a thread reaches once
// it has loaded its part of every input.  (All of h behind the barrier: 6000 rows of 8191 bf16 80 -> 85 us, as their stores start later.)
// The kernels of long rows read twice, and each thread only what it writes itself.
#include <algorithm>

#include "tok.h"

namespace {

using namespace tok;

template <typename W>
struct FwdArgs {
  const W *w;
  long long w_rs;
  uint8_t *q, *scales;
  float *rstd;
  int rows, D, pitch, s_pitch;
  float eps;
};

// Sum over a group of LANES threads, given to all of them.  Groups of more than a wavefront meet in LDS (`red`: one float per
// wavefront of the workgroup and call site).
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *red) {
  if (LANES == 8)
    v = row_sum8(v);
  else if (LANES == 16)
    v = row_sum16(v);
  else if (LANES == 32)
    v = row_sum16(v), v += __shfl_xor(v, 16, PARLE_WAVE);
  else
    v = wave_sum_all(v);
  if (LANES > PARLE_WAVE) {
    constexpr int kWaves = LANES / PARLE_WAVE;
    if ((threadIdx.x & (PARLE_WAVE - 1)) == 0) red[threadIdx.x / PARLE_WAVE] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += red[w];
  }
  return v;
}

// A thread's vector of a row that begins at `col`.  All threads load, without a branch, from `at`, where eight elements exist: its first
// `skip` are the neighbour's as well, eight or more where the row ends before it.  (A guard for the row's end splits the wavefront, and
// each load waits for the one before: 14 300 rows of 768 bf16 backward took 37 us.)  TINY: rows of less than eight elements, one thread's.
struct Place {
  int col, at, skip;
  __device__ __forceinline__ Place(int column, int D) : col(column), at(min(column, max(D - kVec, 0))), skip(col - at) {}
  __device__ __forceinline__ bool live() const { return skip < kVec; }
};
template <bool TINY, typename T>
__device__ __forceinline__ void load_at(const T *p, int D, float (&v)[kVec]) {
  load8(p, TINY ? D : kVec, 0.f, v);
}
template <bool TINY, typename T>
__device__ __forceinline__ void store_at(T *p, int D, const float (&v)[kVec]) {
  store8(p, TINY ? D : kVec, v);
}

// Columns col .. col + 7 of y as codes; 16 lanes hold the 128 values of a scale.  A row's scales are padded to four bytes.
template <int LANES, typename W>
__device__ __forceinline__ void put_codes(const FwdArgs<W> &a, long long row, int col, const float (&y)[kVec]) {
  const int left = a.D - col;
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kVec; ++i) most = max(most, i < left ? finite_bits(y[i]) : 0u);
  most = row_max16(most);
  const uint32_t sb = scale_byte(most);
  const float inv = scale_inverse(sb);
  if (col < a.pitch) {  // codes up to the row's pitch: zeros past D
    float c[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) c[i] = i < left ? scaled(y[i], inv) : 0.f;
    *(u2 *)(a.q + row * a.pitch + col) = u2{codes4(c[0], c[1], c[2], c[3]), codes4(c[4], c[5], c[6], c[7])};
  }
  if ((threadIdx.x & 15) != 0) return;
  uint8_t *scale = a.scales + row * a.s_pitch + (col >> 7);
  if (LANES == 16) {  // one scale, and three bytes of padding
    *(uint32_t *)scale = sb;
  } else if (LANES == 32) {  // two, and two of padding
    *scale = left > 0 ? sb : 0;
    if (col > 0) *(uint16_t *)(scale + 1) = 0;
  } else if ((col >> 7) < a.s_pitch) {
    *scale = left > 0 ? sb : 0;
  }
}

// y of one vector: stored, and as codes.
template <int LANES, bool TINY, typename T, typename W>
__device__ __forceinline__ void emit(const FwdArgs<W> &a, long long row, const Place &p, float (&y)[kVec], T *yo) {
  if (yo && p.live()) store_at<TINY>(yo + row * a.D + p.at, a.D, y);
  if (!a.q) return;
  if (p.skip > 0) {  // the vector's own elements to its front
#pragma unroll
    for (int s = 1; s < kVec; s *= 2)
      if (p.skip & s) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) y[i] = i + s < kVec ? y[i + s] : 0.f;
      }
  }
  put_codes<LANES, W>(a, row, p.col, y);
}

// A row in the registers of LANES threads, 256 / LANES rows to a workgroup where LANES is less than that.
template <typename T, typename W, int LANES, int CH, bool TINY>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rmsnorm_fwd(const T *x, const T *resid, T *h, T *yo, FwdArgs<W> a) {
  constexpr int kBlock = LANES < 256 ? 256 : LANES;
  __shared__ float red[kBlock / PARLE_WAVE];
  const int rep = blockIdx.y, lane = threadIdx.x & (LANES - 1);
  const int r = blockIdx.x * (kBlock / LANES) + threadIdx.x / LANES;
  const bool live = r < a.rows;  // groups past the end go along: the shuffles below want whole groups
  const long long row = (long long)rep * a.rows + min(r, a.rows - 1);
  const auto place = [&](int c) { return Place((c * LANES + lane) * kVec, a.D); };
  float v[CH][kVec];
#pragma unroll
  for (int c = 0; c < CH; ++c) load_at<TINY>(x + row * a.D + place(c).at, a.D, v[c]);
  if (resid) {
    float u[CH][kVec];
#pragma unroll
    for (int c = 0; c < CH; ++c) load_at<TINY>(resid + row * a.D + place(c).at, a.D, u[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[c][i] = stored<T>(v[c][i] + u[c][i]);
  }
  // Elements of two threads lie in the last sixteen columns; a wavefront by itself stores behind its own loads.
  const auto store_h = [&](bool shared) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const Place p = place(c);
      if (h && live && p.live() && (LANES > PARLE_WAVE && p.col + 2 * kVec > a.D) == shared) store_at<TINY>(h + row * a.D + p.at, a.D, v[c]);
    }
  };
  store_h(false);
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const Place p = place(c);
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum += i >= p.skip ? v[c][i] * v[c][i] : 0.f;
  }
  sum = row_sum<LANES>(sum, red);
  if (LANES > PARLE_WAVE) store_h(true);
  const float rs = 1.0f / sqrtf(sum / (float)a.D + a.eps);
  if (a.rstd && live && lane == 0) a.rstd[row] = rs;
  const W *w = a.w + rep * a.w_rs;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (!live) continue;
    const Place p = place(c);
    float g[kVec], y[kVec];
    load_at<TINY>(w + p.at, a.D, g);
#pragma unroll
    for (int i = 0; i < kVec; ++i) y[i] = v[c][i] * rs * g[i];
    emit<LANES, TINY, T, W>(a, row, p, y, yo);
  }
}

// Rows longer than the registers of 1024 threads: read twice, the second time from `h` where it is given.
template <typename T, typename W>
__global__ __launch_bounds__(1024) void k_rmsnorm_fwd_long(const T *x, const T *resid, T *h, T *yo, FwdArgs<W> a) {
  constexpr int kLanes = 1024;
  __shared__ float red[kLanes / PARLE_WAVE];
  const long long row = (long long)blockIdx.y * a.rows + blockIdx.x;
  const int padded = (int)round_up(a.D, 128 * 4);  // whole scales, and their padding
  float sum = 0.f;
  for (int col = threadIdx.x * kVec; col < a.D; col += kLanes * kVec) {
    float v[kVec], u[kVec];
    load8(x + row * a.D + col, a.D - col, 0.f, v);
    if (resid) {
      load8(resid + row * a.D + col, a.D - col, 0.f, u);
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = stored<T>(v[i] + u[i]);
    }
    if (h) store8(h + row * a.D + col, a.D - col, v);
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum += v[i] * v[i];
  }
  sum = row_sum<kLanes>(sum, red);
  const float rs = 1.0f / sqrtf(sum / (float)a.D + a.eps);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = rs;
  const W *w = a.w + blockIdx.y * a.w_rs;
  for (int col = threadIdx.x * kVec; col < padded; col += kLanes * kVec) {
    const int left = a.D - col;
    float v[kVec], u[kVec], g[kVec];
    load8((h ? h : x) + row * a.D + col, left, 0.f, v);
    if (resid && !h) {
      load8(resid + row * a.D + col, left, 0.f, u);
#pragma unroll
      for (int i = 0; i < kVec; ++i) v[i] = stored<T>(v[i] + u[i]);
    }
    load8(w + col, left, 0.f, g);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = v[i] * rs * g[i];
    if (yo) store8(yo + row * a.D + col, left, v);
    if (a.q) put_codes<kLanes, W>(a, row, col, v);
  }
}

// ---- gradient ----
template <typename W>
struct BwdArgs {
  const W *w;
  const float *rstd;
  float *partial;  // [n][strips][Dp]
  long long w_rs;
  int rows, D, Dp, strip;
};

// A workgroup takes a strip of rows, LANES threads a row, and keeps its columns' part of dw in registers; groups of a
// workgroup (LANES < 256) join theirs in LDS.
template <typename T, typename W, int LANES, int CH, bool TINY>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rmsnorm_bwd(const T *h, const T *dout, const T *dresid, T *dx, BwdArgs<W> a) {
  constexpr int kBlock = LANES < 256 ? 256 : LANES, kGroups = kBlock / LANES;
  __shared__ float red[2][kBlock / PARLE_WAVE];
  __shared__ float join[kGroups > 1 ? kGroups * LANES * CH * kVec : 1];
  const int rep = blockIdx.y, lane = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
  const int r0 = blockIdx.x * a.strip, r1 = min(r0 + a.strip, a.rows);
  const auto place = [&](int c) { return Place((c * LANES + lane) * kVec, a.D); };
  float w[CH][kVec], dw[CH][kVec] = {};
#pragma unroll
  for (int c = 0; c < CH; ++c) load_at<TINY>(a.w + rep * a.w_rs + place(c).at, a.D, w[c]);
  // a row of this group: the loads of the next one are on their way while one is reduced, but for the longest, whose threads have no
  // registers left for it
  constexpr bool kNext = LANES * CH < 2048;
  const auto row_of = [&](int r) { return (long long)rep * a.rows + min(r + group, r1 - 1); };
  Raw8<T> hv[CH], dv[CH], ev[CH];
  float next_rs;
  const auto load = [&](long long row) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int count = TINY ? a.D : kVec, at = place(c).at;
      hv[c].load(h + row * a.D + at, count);
      dv[c].load(dout + row * a.D + at, count);
      if (dresid) ev[c].load(dresid + row * a.D + at, count);
    }
    next_rs = a.rstd[row];
  };
  if (kNext) load(row_of(r0));
  int turn = 0;
  for (int r = r0; r < r1; r += kGroups) {  // the same number of turns for every thread: row_sum has a barrier
    const bool live = r + group < r1;
    const long long row = row_of(r);
    if (!kNext) load(row);
    const float rs = next_rs;
    float sum = 0.f, g[CH][kVec], x[CH][kVec], e[CH][kVec];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        x[c][i] = hv[c].at(i), e[c][i] = dresid ? ev[c].at(i) : 0.f;
        const float d = dv[c].at(i);
        if (live) dw[c][i] += d * (x[c][i] * rs);
        g[c][i] = d * w[c][i];
        sum += i >= place(c).skip ? g[c][i] * x[c][i] : 0.f;
      }
    if (kNext) load(row_of(r + kGroups));
    sum = row_sum<LANES>(sum, red[turn]);
    turn ^= 1;  // the next row's sums meet elsewhere: one barrier a row
    const float k = sum / (float)a.D * rs * rs;
    if (live) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const Place p = place(c);
        float o[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) o[i] = rs * (g[c][i] - x[c][i] * k) + e[c][i];
        if (p.live()) store_at<TINY>(dx + row * a.D + p.at, a.D, o);
      }
    }
  }
  float *out = a.partial + ((long long)rep * gridDim.x + blockIdx.x) * a.Dp;
  if (kGroups > 1) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!place(c).live()) continue;
#pragma unroll
      for (int i = 0; i < kVec; ++i) join[group * LANES * CH * kVec + place(c).at + i] = dw[c][i];
    }
    __syncthreads();
    for (int col = threadIdx.x; col < a.D; col += kBlock) {
      float s = 0.f;
      for (int g = 0; g < kGroups; ++g) s += join[g * LANES * CH * kVec + col];
      out[col] = s;
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (place(c).live()) store8(out + place(c).at, kVec, dw[c]);
    }
  }
}

// Rows longer than the registers: three reads (sum, dx, and dw by columns in the kernel below).
template <typename T, typename W>
__global__ __launch_bounds__(1024) void k_rmsnorm_bwd_long(const T *h, const T *dout, const T *dresid, T *dx, BwdArgs<W> a) {
  constexpr int kLanes = 1024;
  __shared__ float red[kLanes / PARLE_WAVE];
  const long long row = (long long)blockIdx.y * a.rows + blockIdx.x;
  const W *w = a.w + blockIdx.y * a.w_rs;
  float sum = 0.f;
  for (int col = threadIdx.x * kVec; col < a.D; col += kLanes * kVec) {
    float hv[kVec], dv[kVec], g[kVec];
    load8(h + row * a.D + col, a.D - col, 0.f, hv);
    load8(dout + row * a.D + col, a.D - col, 0.f, dv);
    load8(w + col, a.D - col, 0.f, g);
#pragma unroll
    for (int i = 0; i < kVec; ++i) sum += dv[i] * g[i] * hv[i];
  }
  sum = row_sum<kLanes>(sum, red);
  const float rs = a.rstd[row], k = sum / (float)a.D * rs * rs;
  for (int col = threadIdx.x * kVec; col < a.D; col += kLanes * kVec) {
    float hv[kVec], dv[kVec], g[kVec], o[kVec];
    load8(h + row * a.D + col, a.D - col, 0.f, hv);
    load8(dout + row * a.D + col, a.D - col, 0.f, dv);
    load8(w + col, a.D - col, 0.f, g);
#pragma unroll
    for (int i = 0; i < kVec; ++i) o[i] = rs * (dv[i] * g[i] - hv[i] * k);
    if (dresid) {
      load8(dresid + row * a.D + col, a.D - col, 0.f, g);
#pragma unroll
      for (int i = 0; i < kVec; ++i) o[i] += g[i];
    }
    store8(dx + row * a.D + col, a.D - col, o);
  }
}
template <typename T, typename W>
__global__ __launch_bounds__(256) void k_rmsnorm_dw_long(const T *h, const T *dout, BwdArgs<W> a) {
  const int rep = blockIdx.z, col = (blockIdx.x * 256 + threadIdx.x) * kVec;
  if (col >= a.D) return;
  const int r0 = blockIdx.y * a.strip, r1 = min(r0 + a.strip, a.rows);
  float dw[kVec] = {};
#pragma unroll 2
  for (int r = r0; r < r1; ++r) {
    const long long row = (long long)rep * a.rows + r;
    float hv[kVec], dv[kVec];
    load8(h + row * a.D + col, a.D - col, 0.f, hv);
    load8(dout + row * a.D + col, a.D - col, 0.f, dv);
    const float rs = a.rstd[row];
#pragma unroll
    for (int i = 0; i < kVec; ++i) dw[i] += dv[i] * (hv[i] * rs);
  }
  float *out = a.partial + ((long long)rep * gridDim.y + blockIdx.y) * a.Dp + col;
  *(f4 *)out = f4{dw[0], dw[1], dw[2], dw[3]};
  *(f4 *)(out + 4) = f4{dw[4], dw[5], dw[6], dw[7]};
}

// dw = sum of the strips' parts: 32 columns x kParts shares of the strips per workgroup.
constexpr int kParts = 32;
__global__ __launch_bounds__(32 * kParts) void k_rmsnorm_dw_join(const float *partial, int strips, int D, int Dp, float *dw, long long w_rs) {
  __shared__ float red[kParts][32];
  const int c = threadIdx.x & 31, part = threadIdx.x >> 5, rep = blockIdx.y, col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < D) {
#pragma unroll 8
    for (int i = part; i < strips; i += kParts) s += partial[((long long)rep * strips + i) * Dp + col];
  }
  red[part][c] = s;
  __syncthreads();
  if (part == 0 && col < D) {
    for (int p = 1; p < kParts; ++p) s += red[p][c];
    dw[rep * w_rs + col] = s;
  }
}

constexpr int kLongest = 1024 * kVec * 2;  // elements of a row that fit the registers of its threads

template <typename T, typename W>
hipError_t fwd(hipStream_t st, const parle_norm_desc &d, const void *x, const void *resid, const void *w, void *h, void *y,
               uint8_t *q, uint8_t *scales, float *rstd) {
  FwdArgs<W> a;
  a.w = (const W *)w, a.w_rs = d.w_stride, a.q = q, a.scales = scales, a.rstd = rstd;
  a.rows = d.rows, a.D = d.dim, a.pitch = (int)round_up(d.dim, 16), a.s_pitch = (int)round_up(ceil_div(d.dim, 128), 4), a.eps = d.eps;
  // whole scales and their padding: the threads of a row cover as much
  const int D = q && d.dim > 256 ? 128 * a.s_pitch : d.dim;
#define PARLE_NORM(LANES, CH, TINY)                                                                                             \
  k_rmsnorm_fwd<T, W, LANES, CH, TINY><<<dim3(ceil_div(d.rows, (LANES < 256 ? 256 : LANES) / LANES), d.n), LANES < 256 ? 256 : LANES, \
                                   0, st>>>((const T *)x, (const T *)resid, (T *)h, (T *)y, a)
  if (D < kVec)
    PARLE_NORM(16, 1, true);
  else if (D <= 8 * kVec && !q)  // with q, sixteen threads find a scale
    PARLE_NORM(8, 1, false);
  else if (D <= 16 * kVec)
    PARLE_NORM(16, 1, false);
  else if (D <= 32 * kVec)
    PARLE_NORM(32, 1, false);
  else if (D <= 64 * kVec)
    PARLE_NORM(64, 1, false);
  else if (D <= 64 * kVec * 2)
    PARLE_NORM(64, 2, false);
  else if (D <= 256 * kVec)
    PARLE_NORM(256, 1, false);
  else if (D <= 256 * kVec * 2)
    PARLE_NORM(256, 2, false);
  else if (D <= 1024 * kVec)
    PARLE_NORM(1024, 1, false);
  else if (D <= kLongest)
    PARLE_NORM(1024, 2, false);
  else
    k_rmsnorm_fwd_long<T, W><<<dim3(d.rows, d.n), 1024, 0, st>>>((const T *)x, (const T *)resid, (T *)h, (T *)y, a);
#undef PARLE_NORM
  return hipGetLastError();
}

// Rows that a workgroup of the gradient kernel takes at a time, by the threads that the dispatch below gives a row.
int rows_at_once(int dim) {
  const int lanes = dim < kVec ? 16 : dim <= 8 * kVec ? 8 : dim <= 16 * kVec ? 16 : dim <= 32 * kVec ? 32 : 64;
  return dim <= 64 * kVec * 2 ? 256 / lanes : 1;
}
// Strips of the gradient kernel: workgroups enough for the chip, and no more parts of dw than that needs.  bf16, 512 workgroups and 1024:
// 8192 x 2048 30.2 and 30.0 us, 3 x 4099 x 2048 53 and 49, 40000 x 200 16.4 and 17.3; but 2000 x 4096 17.7 and 21.3, 16384 x 4096 111 and 119,
// 2000 x 5000 22.4 and 27.3, 4096 x 8192 57 and 63, 2000 x 16384 65 and 75, as a part of a wide row is more to write
// and to read again.  2048 take longer than 1024 everywhere (8192 x 2048 35.2, 100000 x 64 15.1 for 13.5).  A strip is whole turns of a workgroup, or some of its threads never have a row
// (20000 x 33 bf16: 9.8 us with strips of 20 rows, 7.9 with 32).
int strip_rows(const parle_norm_desc &d) {
  const int want = std::max(1, (d.dim > 256 * kVec ? 512 : 1024) / d.n), at_once = rows_at_once(d.dim);
  return (int)round_up(std::max(ceil_div(d.rows, want), at_once > 1 ? 16 : 2), at_once);
}

template <typename T, typename W>
hipError_t bwd(hipStream_t st, const parle_norm_desc &d, const void *h, const void *w, const float *rstd, const void *dout,
               const void *dresid, float *partial, void *dx, float *dw) {
  BwdArgs<W> a;
  a.w = (const W *)w, a.rstd = rstd, a.partial = partial, a.w_rs = d.w_stride;
  a.rows = d.rows, a.D = d.dim, a.Dp = (int)round_up(d.dim, kVec), a.strip = strip_rows(d);
  const int strips = ceil_div(d.rows, a.strip);
#define PARLE_NORM(LANES, CH, TINY)                                                                                 \
  k_rmsnorm_bwd<T, W, LANES, CH, TINY><<<dim3(strips, d.n), LANES < 256 ? 256 : LANES, 0, st>>>(                    \
      (const T *)h, (const T *)dout, (const T *)dresid, (T *)dx, a)
  if (strips > 0) {
    if (d.dim < kVec)
      PARLE_NORM(16, 1, true);
    else if (d.dim <= 8 * kVec)
      PARLE_NORM(8, 1, false);
    else if (d.dim <= 16 * kVec)
      PARLE_NORM(16, 1, false);
    else if (d.dim <= 32 * kVec)
      PARLE_NORM(32, 1, false);
    else if (d.dim <= 64 * kVec)
      PARLE_NORM(64, 1, false);
    else if (d.dim <= 64 * kVec * 2)
      PARLE_NORM(64, 2, false);
    else if (d.dim <= 256 * kVec)
      PARLE_NORM(256, 1, false);
    else if (d.dim <= 256 * kVec * 2)
      PARLE_NORM(256, 2, false);
    else if (d.dim <= 1024 * kVec)
      PARLE_NORM(1024, 1, false);
    else if (d.dim <= kLongest)
      PARLE_NORM(1024, 2, false);
    else {
      // dw first: dx may be written over what it reads
      k_rmsnorm_dw_long<T, W><<<dim3(ceil_div(d.dim, 256 * kVec), strips, d.n), 256, 0, st>>>((const T *)h, (const T *)dout, a);
      k_rmsnorm_bwd_long<T, W><<<dim3(d.rows, d.n), 1024, 0, st>>>((const T *)h, (const T *)dout, (const T *)dresid, (T *)dx, a);
    }
  }
#undef PARLE_NORM
  k_rmsnorm_dw_join<<<dim3(ceil_div(d.dim, 32), d.n), 32 * kParts, 0, st>>>(partial, strips, d.dim, a.Dp, dw, d.w_stride);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm_fwd(hipStream_t st, const parle_norm_desc &d, const void *x, const void *resid, const void *w, void *h,
                              void *y, uint8_t *q, uint8_t *scales, float *rstd) {
  if (d.dtype)
    return d.w_dtype ? fwd<bf16_t, bf16_t>(st, d, x, resid, w, h, y, q, scales, rstd) : fwd<bf16_t, float>(st, d, x, resid, w, h, y, q, scales, rstd);
  return d.w_dtype ? fwd<float, bf16_t>(st, d, x, resid, w, h, y, q, scales, rstd) : fwd<float, float>(st, d, x, resid, w, h, y, q, scales, rstd);
}

int64_t rmsnorm_scratch_bytes(const parle_norm_desc &d) {
  return (int64_t)d.n * ceil_div(d.rows, strip_rows(d)) * round_up(d.dim, kVec) * 4;
}

hipError_t launch_rmsnorm_bwd(hipStream_t st, const parle_norm_desc &d, const void *h, const void *w, const float *rstd,
                              const void *dout, const void *dresid, float *partial, void *dx, float *dw) {
  if (d.dtype)
    return d.w_dtype ? bwd<bf16_t, bf16_t>(st, d, h, w, rstd, dout, dresid, partial, dx, dw) : bwd<bf16_t, float>(st, d, h, w, rstd, dout, dresid, partial, dx, dw);
  return d.w_dtype ? bwd<float, bf16_t>(st, d, h, w, rstd, dout, dresid, partial, dx, dw) : bwd<float, float>(st, d, h, w, rstd, dout, dresid, partial, dx, dw);
}
