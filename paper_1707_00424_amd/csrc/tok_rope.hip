// Rotary positions: pairs of a head's elements turned by position * frequency.  All memory: each element is read and written once.
//
// The sines and cosines of a token are the same for its heads, so a workgroup makes those of its tokens once, in LDS, and then streams the
// heads.  An angle is reduced to a turn in 64 bits: position * frequency as its rounded value and what that left out, times 1 / (2 pi) in two parts as well, so
// that what is lost does not grow with the position (a product rounded in between is off by 2^-21 of an angle near position 2^31 at a frequency of 1, by
// 2^-15 at 64).  Sine and cosine of the rest, half a turn at most either way, are fp32's, within 2^-22 of the true ones: 2^-25 * pi from the rest's
// rounding and two steps of the function; for frequencies up to 2^16.
//
// Three replicas of 4099 tokens, 20 heads of 80 elements of which 64 turn, fp32: 40 us, 3.9 TB/s for reads and writes; 8192 tokens of 40 heads of 128 elements in bf16
// 37 us, 4.5 TB/s; 16 tokens 6 us, a start, sines and a load.
#include "tok.h"

namespace {

using namespace tok;

constexpr int kThreads = 256;
constexpr int kPairs = 2048;  // sines and cosines of a workgroup, 16 KiB

struct Args {
  const void *x;
  const int32_t *positions;
  const float *freqs;
  void *out;
  int tokens, heads, dim, axes, pairs, at_once;
  int ends[PARLE_ROPE_MAX_AXES];  // pairs up to and with each axis
  int turned, per_head;           // pieces of eight pairs of a head; with the pieces of sixteen elements behind them
  float sign;
  long long ld, stride, ld_out, out_stride;
};

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void k_rope(Args g) {
  __shared__ __attribute__((aligned(16))) f2 turn[kPairs];
  const int tid = threadIdx.x, rep = blockIdx.y, t0 = blockIdx.x * g.at_once, count = min(g.at_once, g.tokens - t0);
  const T *x = (const T *)g.x + rep * g.stride + (long long)t0 * g.ld;
  T *out = (T *)g.out + rep * g.out_stride + (long long)t0 * g.ld_out;
  const int32_t *pos = g.positions + ((long long)rep * g.tokens + t0) * g.axes;

  // A piece: eight pairs as a and b, or sixteen elements that do not turn.  The first is on its way while sines are made.
  float a[kVec], b[kVec];
  auto place = [&](int it, int &piece, long long &from, long long &to) {
    const int row = it / g.per_head, t = row / g.heads, head = row - t * g.heads;
    piece = it - row * g.per_head;
    from = t * g.ld + (long long)head * g.dim, to = t * g.ld_out + (long long)head * g.dim;
    return t;
  };
  auto parts = [&](int piece, int &first, int &second, int &n, int &m) {
    if (piece >= g.turned) {
      first = 2 * g.pairs + (piece - g.turned) * 2 * kVec, second = first + kVec, n = g.dim - first, m = n - kVec;
    } else if (INTERLEAVED) {
      first = 2 * piece * kVec, second = first + kVec, n = 2 * g.pairs - first, m = n - kVec;
    } else {
      first = piece * kVec, second = first + g.pairs, n = m = g.pairs - first;
    }
  };
  auto load = [&](int it) {
    int piece, first, second, n, m;
    long long from, to;
    place(it, piece, from, to);
    parts(piece, first, second, n, m);
    load8(x + from + first, n, 0.f, a), load8(x + from + second, m, 0.f, b);
  };
  const int items = count * g.heads * g.per_head;
  int it = tid;
  if (it < items) load(it);

  for (int i = tid; i < count * g.pairs; i += kThreads) {
    const int t = i / g.pairs, p = i - t * g.pairs;
    int axis = 0;
    while (axis < g.axes - 1 && p >= g.ends[axis]) ++axis;
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -9.839338337591243e-18;  // 1 / (2 pi)
    const double at = pos[t * g.axes + axis], freq = g.freqs[p], angle = at * freq, rest = __builtin_fma(at, freq, -angle);
    const double turns = __builtin_fma(angle, kTurn, -rint(angle * kTurn));
    const float half = (float)(2.0 * __builtin_fma(rest, kTurn, __builtin_fma(angle, kTurnRest, turns)));
    float s, c;
    sincospif(half, &s, &c);
    turn[i] = f2{c, s * g.sign};
  }
  __syncthreads();

  while (it < items) {
    int piece, first, second, n, m;
    long long from, to;
    const int t = place(it, piece, from, to);
    parts(piece, first, second, n, m);
    if (piece < g.turned) {
      const f2 *cs = turn + t * g.pairs + piece * kVec;
      const int pairs = g.pairs - piece * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const f2 w = i < pairs ? cs[i] : f2{0.f, 0.f};
        float &u = !INTERLEAVED ? a[i] : i < 4 ? a[2 * (i & 3)] : b[2 * (i & 3)], &v = !INTERLEAVED ? b[i] : i < 4 ? a[2 * (i & 3) + 1] : b[2 * (i & 3) + 1];
        const float y = u * w.x - v * w.y, z = u * w.y + v * w.x;
        u = y, v = z;
      }
    }
    store8(out + to + first, n, a), store8(out + to + second, m, b);
    it += kThreads;
    if (it < items) load(it);
  }
}

}  // namespace

hipError_t launch_rope(hipStream_t st, const parle_rope_desc &d, const void *x, const int32_t *positions, const float *freqs, void *out) {
  Args g{x, positions, freqs, out, d.tokens, d.heads, d.dim, d.axes};
  for (int i = 0; i < d.axes; ++i) g.pairs += d.pairs[i], g.ends[i] = g.pairs;
  g.turned = ceil_div(g.pairs, kVec);
  // elements that do not turn stay where they are when written in place
  const bool in_place = x == out;
  g.per_head = g.turned + (in_place ? 0 : ceil_div(d.dim - 2 * g.pairs, 2 * kVec));
  if (g.per_head == 0) return hipSuccess;
  g.sign = d.inverse ? -1.f : 1.f;
  g.ld = d.ld, g.stride = d.stride, g.ld_out = d.ld_out, g.out_stride = d.out_stride;
  // Tokens of a workgroup: a piece for a thread.  Three times 4099 tokens of 20 heads take 40 us, 47 with four pieces a thread, where all workgroups make their
  // sines at once and then all wait for memory.
  const long long items = (long long)d.heads * g.per_head;
  long long n = kThreads / items;
  if (g.pairs > 0 && n > kPairs / g.pairs) n = kPairs / g.pairs;
  if (n < 1) n = 1;
  g.at_once = (int)n;
  const dim3 grid(ceil_div(d.tokens, n), d.n);
  auto go = [&](auto *kernel) {
    kernel<<<grid, kThreads, 0, st>>>(g);
    return hipGetLastError();
  };
  if (d.dtype) return d.interleaved ? go(k_rope<bf16_t, true>) : go(k_rope<bf16_t, false>);
  return d.interleaved ? go(k_rope<float, true>) : go(k_rope<float, false>);
}
