// Rows of a table by token, scaled, and the table's gradient.
//
// Forward: out[i] = scale * table[tokens[i]], a copy whose source rows are anywhere; memory bounds it.  Groups of lanes walk a row in
// steps of eight elements; four rows per group are on their way together where there are many (24576 rows of 1024 fp32: 37 us, 5.5
// TB/s, what a plain copy reaches), one where there are few (16 rows: 2.5 us, the latency of a token and of its row).
//
// Gradient: dtable[v] = scale * sum of dout[i] over the positions i with tokens[i] = v.  A row of the table belongs to a run of
// equal keys of the sorted tokens, so nothing is added atomically and the order of a sum depends on the tokens alone:
//   1. One workgroup per replica sorts (token, position) in LDS, a stable radix sort by 6 bits a pass; the other workgroups
//      meanwhile clear as much of the table as can be written in that time.  More tokens than a workgroup sorts are
//      sorted in tiles, and tiles are merged in pairs.
//   2. The sorted positions are cut into chunks of kChunk, whatever the tokens: a frequent token spreads over many
//      chunks.  A group of lanes sums the runs of its chunk; a run that ends inside goes to the table, one that crosses a border
//      to scratch.  More workgroups clear the rest of the table, except for the rows that the sorted keys name: sums wait for
//      keys and rows, and leave the memory to them.
//   3. Runs of several chunks are joined, chunk by chunk in order.
// 3 x 8192 tokens into 50001 x 512: 75 us, of them 26 for the sort with 127 MB of zeros, 42 for the sums with 180 MB of zeros (250 MB
// together, 5.9 TB/s) and 7 for the joins; 78 with all zeros beside the sort.  1000 tokens into 100000 x 1024: 94 and 82.  Chunks of 8 or 32 take
// the same or longer; rows to clear in 64 to 256 KiB a workgroup instead of 32: 77 to 80 and 83 to 85.
// Few tokens need none of this (in_one_launch): every workgroup owns a few rows of the table, looks through all tokens for them, sums
// those rows and clears the others (20 tokens into 12000 x 1024: 11 us, 4.5 TB/s, against 15 in three launches).
#include <algorithm>

#include "tok.h"

namespace {

using namespace tok;

constexpr int kThreads = 256;

// `lanes` = 2^lane_shift threads per row.  ROWS rows per group of lanes, their loads in flight together.
template <typename TI, typename TO, int ROWS>
__global__ __launch_bounds__(kThreads) void k_embed_fwd(const TI *table, long long table_rs, const int32_t *tokens, int T, int V,
                                                        int D, float scale, int lane_shift, TO *out) {
  const int lanes = 1 << lane_shift, per_block = kThreads >> lane_shift;
  const int rep = blockIdx.y;
  const long long first = ((long long)blockIdx.x * per_block + (threadIdx.x >> lane_shift)) * ROWS;
  if (first >= T) return;
  const TI *src[ROWS];
  bool live[ROWS], exists[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    exists[r] = first + r < T;
    const int t = exists[r] ? tokens[(long long)rep * T + first + r] : -1;
    live[r] = t >= 0 && t < V;
    src[r] = table + rep * table_rs + (long long)(live[r] ? t : 0) * D;
  }
  TO *dst = out + ((long long)rep * T + first) * D;
  const int count = min(D, kVec);
  for (int at = (threadIdx.x & (lanes - 1)) * kVec; at < D; at += lanes * kVec) {
    const int c = min(at, D - count);  // a row's last eight columns; a lane that shares some with its neighbour stores the same values
    float v[ROWS][kVec];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (live[r]) {
        load8(src[r] + c, count, 0.f, v[r]);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[r][i] = 0.f;
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (!exists[r]) continue;
      if (live[r]) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[r][i] *= scale;
      }
      store8(dst + (long long)r * D + c, count, v[r]);
    }
  }
}

// ---- gradient ----

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / PARLE_WAVE;
constexpr int kMostItems = 16, kTile = kSortThreads * kMostItems;  // tokens that one workgroup sorts
constexpr int kDigitBits = 6, kDigits = 1 << kDigitBits;
constexpr int kChunk = 16;  // sorted positions of one group of lanes: their rows are on the way together

// A stable sort of one tile by key, in LDS: thread t of wavefront w holds items w * 64 * ITEMS + 64 j + lane.
// The rank of an item among equal digits is its rank in the wavefront's vector (from ballots) plus what earlier vectors and
// wavefronts hold of the digit.
template <int ITEMS>
__device__ void sort_tile(const int32_t *tokens, int first, int count, int V, int bits, uint32_t *keys_out, uint32_t *pos_out,
                          uint32_t *lds) {
  constexpr int kItems = kSortThreads * ITEMS;
  uint32_t *skey = lds, *hist = lds + kItems;                       // hist [digit][wave]
  unsigned short *spos = (unsigned short *)(hist + kDigits * kSortWaves + kSortWaves);
  uint32_t *wave_tot = hist + kDigits * kSortWaves;
  const int lane = threadIdx.x & (PARLE_WAVE - 1), wave = threadIdx.x / PARLE_WAVE;
  const int base = wave * PARLE_WAVE * ITEMS + lane;
  uint32_t key[ITEMS];
  unsigned short pos[ITEMS];
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int i = base + PARLE_WAVE * j;
    const int t = i < count ? tokens[first + i] : -1;
    key[j] = t >= 0 && t < V ? (uint32_t)t : (uint32_t)V;  // what has no row goes to the end
    pos[j] = (unsigned short)i;
  }
  for (int shift = 0; shift < bits; shift += kDigitBits) {
    for (int i = threadIdx.x; i < kDigits * kSortWaves; i += kSortThreads) hist[i] = 0;
    __syncthreads();
    uint32_t rank[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const uint32_t digit = (key[j] >> shift) & (kDigits - 1);
      uint64_t same = ~0ull;
#pragma unroll
      for (int b = 0; b < kDigitBits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? set : ~set;
      }
      const uint32_t before = __popcll(same & ((1ull << lane) - 1));
      // All lanes of the digit read, then its first lane writes, then the next vector reads: LDS keeps a wavefront's order,
      // and volatile accesses keep the compiler's.
      volatile uint32_t *h = &hist[digit * kSortWaves + wave];
      const uint32_t held = *h;
      rank[j] = held + before;
      __builtin_amdgcn_wave_barrier();
      if (before == 0) *h = held + __popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // exclusive sum over [digit][wave]; 1024 counts, one per thread
    const uint32_t mine = hist[threadIdx.x];
    uint32_t sum = mine;
#pragma unroll
    for (int o = 1; o < PARLE_WAVE; o <<= 1) {
      const uint32_t up = __shfl_up(sum, o, PARLE_WAVE);
      if (lane >= o) sum += up;
    }
    if (lane == PARLE_WAVE - 1) wave_tot[wave] = sum;
    __syncthreads();
    uint32_t ahead = 0;
    for (int w = 0; w < wave; ++w) ahead += wave_tot[w];
    hist[threadIdx.x] = ahead + sum - mine;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      const uint32_t digit = (key[j] >> shift) & (kDigits - 1), to = hist[digit * kSortWaves + wave] + rank[j];
      skey[to] = key[j];
      spos[to] = pos[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      key[j] = skey[base + PARLE_WAVE * j];
      pos[j] = spos[base + PARLE_WAVE * j];
    }
  }
  // items past `count` have the largest key and came last: the sort leaves them at the end
#pragma unroll
  for (int j = 0; j < ITEMS; ++j) {
    const int i = base + PARLE_WAVE * j;
    if (i < count) {
      keys_out[first + i] = key[j];
      pos_out[first + i] = (uint32_t)(first + pos[j]);
    }
  }
}

constexpr size_t sort_lds(int items) {
  return (size_t)(kSortThreads * items + kDigits * kSortWaves + kSortWaves) * 4 + (size_t)kSortThreads * items * 2;
}

// Workgroups 0 .. sorters-1: one tile each of one replica; the others write zeros.
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort_zero(const int32_t *tokens, int T, int V, int bits, int tiles, int n,
                                                                  uint32_t *keys, uint32_t *pos, float *dtable, long long table_rs,
                                                                  long long table_elems) {
  extern __shared__ uint32_t lds[];
  const int sorters = tiles * n;
  if ((int)blockIdx.x < sorters) {
    const int rep = blockIdx.x / tiles, first = (blockIdx.x % tiles) * (kSortThreads * ITEMS);
    sort_tile<ITEMS>(tokens + (long long)rep * T, first, min(T - first, kSortThreads * ITEMS), V, bits, keys + (long long)rep * T,
                     pos + (long long)rep * T, lds);
    return;
  }
  const long long vecs = table_elems / 4, step = (long long)(gridDim.x - sorters) * kSortThreads;
  const long long me = (long long)(blockIdx.x - sorters) * kSortThreads + threadIdx.x;
  for (int rep = 0; rep < n; ++rep) {
    float *row = dtable + rep * table_rs;
    for (long long i = me; i < vecs; i += step) *(f4_any *)(row + 4 * i) = f4{0.f, 0.f, 0.f, 0.f};
    if (me < (table_elems & 3)) row[vecs * 4 + me] = 0.f;
  }
}

// Merges sorted runs of `len` in pairs: an item's place is its own index plus its rank in the partner run; equal keys
// of the left run come first.
__global__ __launch_bounds__(kThreads) void k_embed_merge(const uint32_t *keys, const uint32_t *pos, int T, long long len,
                                                          uint32_t *keys_out, uint32_t *pos_out) {
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (i >= T) return;
  const long long off = (long long)blockIdx.y * T, run = i / len, pair = run & ~1ll;
  const bool left = run == pair;
  const long long a0 = pair * len, b0 = min(a0 + len, (long long)T), b1 = min(a0 + 2 * len, (long long)T);
  const uint32_t k = keys[off + i];
  long long lo = left ? b0 : a0, hi = left ? b1 : b0;
  const long long from = lo;
  while (lo < hi) {
    const long long mid = (lo + hi) / 2;
    const uint32_t m = keys[off + mid];
    if (left ? m < k : m <= k)
      lo = mid + 1;
    else
      hi = mid;
  }
  const long long to = a0 + (i - (left ? a0 : b0)) + (lo - from);
  keys_out[off + to] = k;
  pos_out[off + to] = pos[off + i];
}

struct SumArgs {
  const uint32_t *keys, *pos;  // [n][T]
  float *dtable;
  float *part;                 // [n][chunks][2][Dp]: a run that began before the chunk; one that goes on after it
  long long table_rs;
  int T, V, D, Dp, chunks, lane_shift;
  float scale;
  int chunk_x, chunk_y, chunk_blocks;     // workgroups of the sums: per column slice, slices, all
  int zero_first, zero_rows, zero_blocks;  // the table's rows that are still to be cleared, rows of a workgroup, workgroups of a replica
};
constexpr int kZeroRows = 1024;

// First of the `count` ascending keys that is not below `v`; a whole wavefront, 64 keys a step.
__device__ __forceinline__ int first_not_below(const uint32_t *keys, int count, uint32_t v) {
  const int lane = threadIdx.x & (PARLE_WAVE - 1);
  int at = 0, left = count;
  while (left > 0) {
    const int step = (left + PARLE_WAVE - 1) / PARLE_WAVE, probe = (lane + 1) * step - 1;
    const int below = __popcll(__ballot(probe < left && keys[at + min(probe, left - 1)] < v));
    at += below * step;
    left = min(step - 1, left - below * step);
  }
  return at;
}

// Clears those of `rows` rows that are not `touched`, in vectors of 16 bytes of memory, wherever rows begin: misaligned stores of 16
// bytes take twice as long.  A vector of a row of four elements or more lies in two rows at most.
__device__ __forceinline__ void clear_others(float *table, int rows, int D, const uint8_t *touched) {
  const int all = rows * D, before = (int)((uintptr_t)table / 4 % 4);  // elements of the first 16 bytes that are not the table's
  constexpr int kStep = kThreads * 4;
  const int step_rows = kStep / D, step_cols = kStep % D;
  int e = (int)threadIdx.x * 4 - before, row = e < 0 ? -1 : e / D, col = e - row * D;
  for (; e < all; e += kStep) {
    const bool one = D >= 4 && e >= 0 && col + 4 <= D;  // in one row
    if (D >= 4 && e >= 0 && e + 4 <= all && !touched[row] && !touched[one ? row : row + 1]) {
      *(f4 *)(table + e) = f4{0.f, 0.f, 0.f, 0.f};
    } else if (!one) {
#pragma unroll 1
      for (int i = max(e, 0); i < min(e + 4, all); ++i)
        if (!touched[i / D]) table[i] = 0.f;
    }
    row += step_rows, col += step_cols;
    if (col >= D) col -= D, ++row;
  }
}

// Clears those of zero_rows rows that no token has: their keys are sorted by now.
__device__ __forceinline__ void clear_rows(const SumArgs &a, int block) {
  __shared__ uint8_t touched[kZeroRows];
  __shared__ int bound[2];
  const int rep = block / a.zero_blocks, v0 = a.zero_first + block % a.zero_blocks * a.zero_rows, rows = min(a.zero_rows, a.V - v0);
  const uint32_t *keys = a.keys + (long long)rep * a.T;
  const int wave = threadIdx.x / PARLE_WAVE;
  if (wave < 2) {
    const int at = first_not_below(keys, a.T, (uint32_t)(wave ? v0 + rows : v0));
    if (threadIdx.x % PARLE_WAVE == 0) bound[wave] = at;
  }
  for (int i = threadIdx.x; i < rows; i += kThreads) touched[i] = 0;
  __syncthreads();
  for (int i = bound[0] + threadIdx.x; i < bound[1]; i += kThreads) touched[keys[i] - v0] = 1;
  __syncthreads();
  clear_others(a.dtable + rep * a.table_rs + (long long)v0 * a.D, rows, a.D, touched);
}

// Columns of a row of dout, as they came: four, or the `count` < 4 of a shorter row (the others' places are not used).
template <bool FOUR>
__device__ __forceinline__ us4 load_raw(const bf16_t *p, int count) {
  if (FOUR) return *(const us4_any *)p;
  return us4{p[0], p[min(1, count - 1)], p[min(2, count - 1)], 0};
}
template <bool FOUR>
__device__ __forceinline__ f4 load_raw(const float *p, int count) {
  if (FOUR) return *(const f4_any *)p;
  return f4{p[0], p[min(1, count - 1)], p[min(2, count - 1)], 0.f};
}
__device__ __forceinline__ f4 widen(us4 v) { return f4{bf16_to_f32(v.x), bf16_to_f32(v.y), bf16_to_f32(v.z), bf16_to_f32(v.w)}; }
__device__ __forceinline__ f4 widen(f4 v) { return v; }

// A group of lanes sums one chunk for its columns, four to a lane: a wavefront stores a kilobyte of a row at once, and there are twice
// the wavefronts that eight columns to a lane give (3 x 8192 tokens of 512: 3 % of the whole call).  The workgroups behind these clear
// rows.  grid: chunk_x * chunk_y * n + zero_blocks * n
template <typename T, bool FOUR>
__global__ __launch_bounds__(kThreads) void k_embed_chunks(const T *dout, SumArgs a) {
  if ((int)blockIdx.x >= a.chunk_blocks) {
    clear_rows(a, blockIdx.x - a.chunk_blocks);
    return;
  }
  const int lanes = 1 << a.lane_shift, slice = blockIdx.x / a.chunk_x, rep = slice / a.chunk_y;
  const int chunk = blockIdx.x % a.chunk_x * (kThreads >> a.lane_shift) + (threadIdx.x >> a.lane_shift);
  int col = (slice % a.chunk_y * lanes + (threadIdx.x & (lanes - 1))) * 4;
  if (chunk >= a.chunks || col >= a.D) return;
  if (FOUR) col = min(col, a.D - 4);  // the last four columns; a lane that shares some with its neighbour stores the same sums
  const uint32_t *keys = a.keys + (long long)rep * a.T, *pos = a.pos + (long long)rep * a.T;
  const T *src = dout + (long long)rep * a.T * a.D + col;
  float *table = a.dtable + rep * a.table_rs + col;
  float *part = a.part + ((long long)rep * a.chunks + chunk) * 2 * a.Dp + col;
  const int first = chunk * kChunk, count = min(kChunk, a.T - first);
  // Sixteen keys and positions as vectors.  Past the last chunk's end they are what lies behind the lists in scratch, and are not used.
  uint32_t k[kChunk + 1];
  u4 at[kChunk / 4];
#pragma unroll
  for (int q = 0; q < kChunk / 4; ++q) {
    const u4 v = *(const u4_any *)(keys + first + 4 * q);
    at[q] = *(const u4_any *)(pos + first + 4 * q);
#pragma unroll
    for (int j = 0; j < 4; ++j) k[4 * q + j] = v[j];
  }
  k[kChunk] = first + kChunk < a.T ? keys[first + kChunk] : 0xffffffffu;
  bool from_before = first > 0 && keys[first - 1] == k[0];
#pragma unroll
  for (int j = 0; j < kChunk; ++j)
    if (j >= count) k[j] = 0xffffffffu;  // ends the run in front of it, and is none
  decltype(load_raw<FOUR>(src, a.D)) v[kChunk];
#pragma unroll
  for (int j = 0; j < kChunk; ++j) {
    const uint32_t row = k[j] < (uint32_t)a.V ? at[j / 4][j % 4] : 0;  // one that exists, and no branch
    v[j] = load_raw<FOUR>(src + (long long)row * a.D, a.D);
  }
  f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kChunk; ++j) {
    if (k[j] >= (uint32_t)a.V) break;  // no later key is less
    acc += widen(v[j]);
    const bool ends = k[j] != k[j + 1];
    if (ends || j + 1 == kChunk) {
      const bool whole = ends && !from_before;
      float *to = whole ? table + (long long)k[j] * a.D : part + (from_before ? 0 : a.Dp);
      acc *= whole ? a.scale : 1.f;
      if (FOUR) {
        *(f4_any *)to = acc;
      } else {
        for (int e = 0; e < a.D; ++e) to[e] = acc[e];
      }
      acc = f4{0.f, 0.f, 0.f, 0.f};
      from_before = false;
    }
  }
}

// Joins the run that begins in a chunk and goes on after it: its parts of this chunk and of all that follow, by four
// wavefronts that take a quarter of the chunks each.  grid: (chunks - 1, column slices, n)
__global__ __launch_bounds__(kThreads) void k_embed_join(SumArgs a) {
  constexpr int kWaves = kThreads / PARLE_WAVE;
  const int chunk = blockIdx.x, rep = blockIdx.z;
  const uint32_t *keys = a.keys + (long long)rep * a.T;
  const int first = chunk * kChunk, end = first + kChunk;  // there is a chunk behind this one, so end < T
  const uint32_t k = keys[end];
  if (k >= (uint32_t)a.V || keys[end - 1] != k) return;                             // no run crosses the border
  if (keys[first] == k && first > 0 && keys[first - 1] == k) return;               // it began before this chunk
  // the last chunk that holds the key: binary search over the chunks' first keys
  int lo = chunk + 1, hi = a.chunks;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (keys[mid * kChunk] == k)
      lo = mid + 1;
    else
      hi = mid;
  }
  const int parts = lo - chunk;  // chunk .. lo-1
  const int lane = threadIdx.x & (PARLE_WAVE - 1), wave = threadIdx.x / PARLE_WAVE;
  const int col = (blockIdx.y * PARLE_WAVE + lane) * 4;
  __shared__ f4 red[kWaves][PARLE_WAVE];
  const float *part = a.part + ((long long)rep * a.chunks + chunk) * 2 * a.Dp + col;
  const int each = (parts + kWaves - 1) / kWaves, p1 = min((wave + 1) * each, parts);
  f4 acc = {0.f, 0.f, 0.f, 0.f};
  if (col < a.D) {
#pragma unroll 8
    for (int p = wave * each; p < p1; ++p) acc += *(const f4 *)(part + (long long)p * 2 * a.Dp + (p == 0 ? a.Dp : 0));
  }
  red[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && col < a.D) {
    f4 s = red[0][lane];
    for (int w = 1; w < kWaves; ++w) s += red[w][lane];
    float *to = a.dtable + rep * a.table_rs + (long long)k * a.D + col;
    for (int e = 0; e < 4 && col + e < a.D; ++e) to[e] = s[e] * a.scale;
  }
}

// ---- gradient, few tokens ----
constexpr int kDirect = 512, kDirectRows = 64;

__device__ __forceinline__ float value(const float *p) { return *p; }
__device__ __forceinline__ float value(const bf16_t *p) { return bf16_to_f32(*p); }

// A workgroup owns `rows` rows of the table: it clears those that no token has, and its wavefronts sum the others, 256 columns at a
// time.  grid: (V / rows, n)
template <typename T>
__global__ __launch_bounds__(kThreads) void k_embed_direct(const int32_t *tokens, const T *dout, int count, int V, int D, float scale,
                                                           int rows, float *dtable, long long table_rs) {
  constexpr int kWaves = kThreads / PARLE_WAVE, kAhead = 16;
  __shared__ int hit[kDirect], sorted[kDirect];  // row of the workgroup's << 16 | position: by position, then by row and position
  __shared__ int start[kDirectRows + 1];         // of a row's hits
  __shared__ uint8_t touched[kDirectRows];
  __shared__ int found[kDirect / kThreads][kWaves];
  const int rep = blockIdx.y, v0 = blockIdx.x * rows, mine = min(rows, V - v0);
  const int lane = threadIdx.x & (PARLE_WAVE - 1), wave = threadIdx.x / PARLE_WAVE;
  int row_of[kDirect / kThreads];
  uint64_t in[kDirect / kThreads];
#pragma unroll
  for (int k = 0; k < kDirect / kThreads; ++k) {
    const int i = k * kThreads + threadIdx.x;
    row_of[k] = i < count ? tokens[(long long)rep * count + i] - v0 : -1;
    in[k] = __ballot(row_of[k] >= 0 && row_of[k] < mine);
    if (lane == 0) found[k][wave] = __popcll(in[k]);
  }
  __syncthreads();
  int hits = 0;
#pragma unroll
  for (int k = 0; k < kDirect / kThreads; ++k)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave && row_of[k] >= 0 && row_of[k] < mine)
        hit[hits + __popcll(in[k] & ((1ull << lane) - 1))] = row_of[k] << 16 | (k * kThreads + threadIdx.x);
      hits += found[k][w];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < hits; i += kThreads) {
    const int me = hit[i];
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < hits; ++j) before += hit[j] < me;
    sorted[before] = me;
  }
  if ((int)threadIdx.x <= mine) {
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < hits; ++j) before += hit[j] < (int)threadIdx.x << 16;
    start[threadIdx.x] = before;
  }
  __syncthreads();
  if ((int)threadIdx.x < mine) touched[threadIdx.x] = start[threadIdx.x] < start[threadIdx.x + 1];
  __syncthreads();
  const T *src = dout + (long long)rep * count * D;
  float *table = dtable + rep * table_rs + (long long)v0 * D;
  if (hits > 0 && D >= 4) {
    const int slices = (D + 4 * PARLE_WAVE - 1) / (4 * PARLE_WAVE);
    for (int it = wave; it < mine * slices; it += kWaves) {
      const int r = it / slices, first = start[r], last = start[r + 1], at = ((it - r * slices) * PARLE_WAVE + lane) * 4;
      if (first == last || at >= D) continue;
      const int col = min(at, D - 4);  // the last four columns; a lane that shares some with its neighbour stores the same sums
      f4 acc = {0.f, 0.f, 0.f, 0.f};
      for (int h = first; h < last; h += kAhead) {
        decltype(load_raw<true>(src, D)) x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u] = load_raw<true>(src + (long long)(sorted[min(h + u, last - 1)] & 0xffff) * D + col, D);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (h + u < last) acc += widen(x[u]);
      }
      *(f4_any *)(table + (long long)r * D + col) = acc * scale;
    }
  } else if (hits > 0) {
    for (int i = threadIdx.x; i < mine * D; i += kThreads) {
      const int r = i / D;
      float acc = 0.f;
      for (int h = start[r]; h < start[r + 1]; ++h) acc += value(src + (sorted[h] & 0xffff) * D + (i - r * D));
      if (touched[r]) table[i] = acc * scale;
    }
  }
  clear_others(table, mine, D, touched);
}

int lane_shift_of(int groups) {
  int s = 0;
  while (s < 6 && (1 << s) < groups) ++s;
  return s;
}

int digits_of(int V) {
  int bits = 1;
  while (bits < 31 && (V >> bits)) ++bits;  // keys are 0 .. V
  return bits;
}

template <typename TI, typename TO>
hipError_t fwd(hipStream_t st, const parle_embed_desc &d, const void *table, const int32_t *tokens, void *out) {
  int shift = 3;  // 8 .. 256 lanes per row
  while (shift < 8 && (kVec << shift) < d.dim) ++shift;
  const int per_block = kThreads >> shift;
  // Four rows per group keep enough loads in flight; few rows are spread over the chip instead.
  const bool many = (long long)d.n * ceil_div(d.tokens, per_block) >= 4096;
  const int rows = per_block * (many ? 4 : 1);
  const dim3 grid(ceil_div(d.tokens, rows), d.n);
  if (many)
    k_embed_fwd<TI, TO, 4><<<grid, kThreads, 0, st>>>((const TI *)table, d.table_stride, tokens, d.tokens, d.vocab, d.dim, d.scale, shift, (TO *)out);
  else
    k_embed_fwd<TI, TO, 1><<<grid, kThreads, 0, st>>>((const TI *)table, d.table_stride, tokens, d.tokens, d.vocab, d.dim, d.scale, shift, (TO *)out);
  return hipGetLastError();
}

template <typename T>
hipError_t direct(hipStream_t st, const parle_embed_desc &d, const int32_t *tokens, const void *dout, float *dtable) {
  // Rows of 32 KiB together: fewer look through the tokens more often, more leave the frequent tokens to too few workgroups.
  // Workgroups enough for the chip where the table is small.
  const long long all = (long long)d.vocab * d.n;
  const int rows = (int)std::max<long long>(1, std::min<long long>({8192 / d.dim, all / 2048, kDirectRows}));
  const dim3 grid(ceil_div(d.vocab, rows), d.n);
  k_embed_direct<T><<<grid, kThreads, 0, st>>>(
      tokens, (const T *)dout, d.tokens, d.vocab, d.dim, d.scale, rows, dtable, d.table_stride);
  return hipGetLastError();
}

// One launch, where its workgroups' chains of waits cost less than two more launches: they have no part in many tokens, nor in many
// rows.  us for one launch and for three, 4 MB of tables: 8 and 14 with 500 tokens; 15 MB: 14 and 16 with 256, 18 and 16 with 500; 49 MB: 14 and 16
// with 128, 21 and 17 with 500; 102 MB: 21 and 22 with 32, 23 and 22 with 64; 148 MB: 33 and 32 with 32, 53 and 35 with 500.
bool in_one_launch(const parle_embed_desc &d) {
  const double bytes = 4. * d.n * d.vocab * d.dim;
  return d.tokens <= kChunk || (d.tokens <= kDirect && d.tokens * bytes <= 6e9);
}

// Scratch: keys and positions (twice where tiles are merged), then the partial sums.
struct Scratch {
  long long list, lists, part, Dp;
  int chunks;
};
Scratch scratch_of(const parle_embed_desc &d) {
  Scratch s = {};
  if (in_one_launch(d)) return s;
  s.list = round_up((long long)d.n * d.tokens * 4, 256);
  s.lists = d.tokens > kTile ? 4 : 2;
  s.Dp = round_up(d.dim, 8);
  s.chunks = ceil_div(d.tokens, kChunk);
  s.part = (long long)d.n * s.chunks * 2 * s.Dp * 4;
  return s;
}

template <int ITEMS>
hipError_t sort_zero(hipStream_t st, const parle_embed_desc &d, int tiles, const int32_t *tokens, uint32_t *keys, uint32_t *pos,
                     float *dtable, int &cleared) {
  // A sort takes 2 us and, for each pass, 1.2 and 0.65 for each item of a thread; meanwhile the others clear 6 MB a microsecond.  What
  // they leave is cleared beside the sums.  Rows of less than a vector are all cleared here.
  const int passes = ceil_div(digits_of(d.vocab), kDigitBits);
  const double most = 6e6 * (2. + passes * (1.2 + 0.65 * ITEMS)) / (4. * d.n * d.dim);
  cleared = d.dim < 4 || most >= d.vocab ? d.vocab : (int)most;
  const long long elems = (long long)cleared * d.dim;
  const int zero = (int)std::min<long long>(1024, std::max<long long>(1, d.n * elems / (4 * kSortThreads * 4)));
  static const hipError_t lds_ok =
      hipFuncSetAttribute((const void *)k_embed_sort_zero<ITEMS>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sort_lds(ITEMS));
  if (lds_ok != hipSuccess) return lds_ok;
  k_embed_sort_zero<ITEMS><<<tiles * d.n + zero, kSortThreads, sort_lds(ITEMS), st>>>(
      tokens, d.tokens, d.vocab, digits_of(d.vocab), tiles, d.n, keys, pos, dtable, d.table_stride, elems);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed_fwd(hipStream_t st, const parle_embed_desc &d, const void *table, const int32_t *tokens, void *out) {
  if (d.table_dtype) return d.dtype ? fwd<bf16_t, bf16_t>(st, d, table, tokens, out) : fwd<bf16_t, float>(st, d, table, tokens, out);
  return d.dtype ? fwd<float, bf16_t>(st, d, table, tokens, out) : fwd<float, float>(st, d, table, tokens, out);
}

int64_t embed_scratch_bytes(const parle_embed_desc &d) {
  const Scratch s = scratch_of(d);
  return s.list * s.lists + s.part;
}

hipError_t launch_embed_bwd(hipStream_t st, const parle_embed_desc &d, const int32_t *tokens, const void *dout, void *scratch,
                            float *dtable) {
  if (in_one_launch(d)) return d.dtype ? direct<bf16_t>(st, d, tokens, dout, dtable) : direct<float>(st, d, tokens, dout, dtable);
  const Scratch s = scratch_of(d);
  char *at = (char *)scratch;
  uint32_t *keys = (uint32_t *)at, *pos = (uint32_t *)(at + s.list);
  const int tiles = ceil_div(d.tokens, kTile);
  const auto sort = d.tokens > 8 * kSortThreads   ? sort_zero<kMostItems>
                    : d.tokens > 4 * kSortThreads ? sort_zero<8>
                    : d.tokens > kSortThreads     ? sort_zero<4>
                                                  : sort_zero<1>;
  int cleared = 0;
  const hipError_t e = sort(st, d, tiles, tokens, keys, pos, dtable, cleared);
  if (e != hipSuccess) return e;
  if (tiles > 1) {
    uint32_t *keys2 = (uint32_t *)(at + 2 * s.list), *pos2 = (uint32_t *)(at + 3 * s.list);
    for (long long len = kTile; len < d.tokens; len *= 2) {
      k_embed_merge<<<dim3(ceil_div(d.tokens, kThreads), d.n), kThreads, 0, st>>>(keys, pos, d.tokens, len, keys2, pos2);
      std::swap(keys, keys2);
      std::swap(pos, pos2);
    }
  }
  SumArgs a;
  a.keys = keys, a.pos = pos, a.dtable = dtable, a.part = (float *)(at + s.list * s.lists);
  a.table_rs = d.table_stride, a.T = d.tokens, a.V = d.vocab, a.D = d.dim, a.Dp = (int)s.Dp, a.chunks = s.chunks, a.scale = d.scale;
  const int groups = ceil_div(d.dim, 4);
  a.lane_shift = lane_shift_of(groups);
  a.chunk_x = ceil_div(s.chunks, kThreads >> a.lane_shift), a.chunk_y = ceil_div(groups, 1 << a.lane_shift);
  a.chunk_blocks = a.chunk_x * a.chunk_y * d.n;
  a.zero_first = cleared, a.zero_rows = std::max(1, std::min(kZeroRows, 8192 / d.dim));  // 32 KiB together
  a.zero_blocks = ceil_div(d.vocab - cleared, a.zero_rows);
  const int grid = a.chunk_blocks + a.zero_blocks * d.n;
  if (d.dtype)
    (d.dim >= 4 ? k_embed_chunks<bf16_t, true> : k_embed_chunks<bf16_t, false>)<<<grid, kThreads, 0, st>>>((const bf16_t *)dout, a);
  else
    (d.dim >= 4 ? k_embed_chunks<float, true> : k_embed_chunks<float, false>)<<<grid, kThreads, 0, st>>>((const float *)dout, a);
  k_embed_join<<<dim3(s.chunks - 1, ceil_div(d.dim, 4 * PARLE_WAVE), d.n), kThreads, 0, st>>>(a);
  return hipGetLastError();
}
