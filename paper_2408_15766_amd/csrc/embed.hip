// Rows of an embedding table, and the gradient of the table (include/spec_step.h).
//
// The gradient sums rows of dy by token.  The positions are sorted by (token, position), so that a table row's sum is a walk over neighbours and its order is
// fixed: in tiles of kTile positions a position's place is the number of smaller ones (counted, kTile comparisons for each); over several
// tiles four sorted runs at a time become one, a position's place being that in its own run plus those that searches find in the other
// three.  Padding sorts behind the vocabulary and is never read.
// Tokens that occur often (padding apart, the most frequent word is a tenth of a text) would keep one workgroup busy long after the others: aligned runs of 32
// and of 1024 sorted positions that hold one token are summed first, by workgroups of their own, and the walk takes a run's sum where it meets one.
// Bound: memory (dy once in, the table once out).  Measured: 16384 rows into 128256 x 4096 in bf16: places 9 us, joined 5, runs 9 and 5,
// table 184 (6.4 TB/s).  2^20 rows into 2000 x 64: places 266, joined 4 times 30, of 475 in all.  The lookup of 16384 rows of that table
// 33.5 us in bf16 and 85 in fp32 (4.0 and 3.2 TB/s by the rows written alone).
#include "common.h"
#include "elements.h"
#include "kernels.h"

#include <type_traits>

namespace spec {

namespace {

constexpr int kTile = 4096, kRun = 32, kRuns = 1024;          // positions of a tile and of the two lengths of runs
constexpr int kLongLeast = 8192;                              // positions from which on the longer runs are summed (below, a walk meets 256 sums at most)
constexpr int kEmbedThreads = 256;

// Eight columns of a row, at any alignment of their type (the memory takes unaligned accesses of 16 bytes; a column at a time took 130 us
// where they take 58: the gradient of a 60000 x 2001 table in bf16), or the n that are left at its end.
typedef u32x4_t u32x4_any __attribute__((aligned(2)));
typedef f32x4_t f32x4_any __attribute__((aligned(4)));
struct Columns { float x[8]; };
// WHOLE: n >= 8 (asked at each load, every load waited for the one before)
template <bool WHOLE> __device__ __forceinline__ Columns load_columns(const void *p, int64_t i, int n, bool bf16) {
  Columns r;
  if constexpr (WHOLE) {
    Eight e;
    if (bf16) e.v[0] = *(const u32x4_any *)((const bf16_t *)p + i);
    else {
      e.v[0] = __builtin_bit_cast(u32x4_t, (f32x4_t)*(const f32x4_any *)((const float *)p + i));
      e.v[1] = __builtin_bit_cast(u32x4_t, (f32x4_t)*(const f32x4_any *)((const float *)p + i + 4));
    }
    widen8(e, bf16, r.x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++) r.x[j] = j < n ? load1(p, i + j, bf16) : 0.f;
  }
  return r;
}
__device__ __forceinline__ void store_columns(void *p, int64_t i, int n, bool bf16, const Columns &c) {
  if (n >= 8) {
    if (bf16) *(u32x4_any *)((bf16_t *)p + i) = u32x4_t{pack_bf16x2(c.x[0], c.x[1]), pack_bf16x2(c.x[2], c.x[3]), pack_bf16x2(c.x[4], c.x[5]), pack_bf16x2(c.x[6], c.x[7])};
    else {
      *(f32x4_any *)((float *)p + i) = f32x4_t{c.x[0], c.x[1], c.x[2], c.x[3]};
      *(f32x4_any *)((float *)p + i + 4) = f32x4_t{c.x[4], c.x[5], c.x[6], c.x[7]};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (j < n) store1(p, i + j, bf16, c.x[j]);
  }
}
// Zeros past the caches, which keep dy: the table's kernel 229 -> 183 us (16384 rows into 128256 x 4096)
__device__ __forceinline__ void clear_columns(void *p, int64_t i, int n, bool bf16) {
  if (n >= 8) {
    if (bf16) __builtin_nontemporal_store(u32x4_t{0u, 0u, 0u, 0u}, (u32x4_any *)((bf16_t *)p + i));
    else {
      __builtin_nontemporal_store(f32x4_t{0.f, 0.f, 0.f, 0.f}, (f32x4_any *)((float *)p + i));
      __builtin_nontemporal_store(f32x4_t{0.f, 0.f, 0.f, 0.f}, (f32x4_any *)((float *)p + i + 4));
    }
  } else {
    for (int j = 0; j < n; j++) store1(p, i + j, bf16, 0.f);
  }
}
__device__ __forceinline__ void add_columns(Columns &s, const Columns &v) {
#pragma unroll
  for (int j = 0; j < 8; j++) s.x[j] += v.x[j];
}

// A workgroup has a row, or as many short ones as its threads hold.
__global__ __launch_bounds__(kEmbedThreads) void embed_kernel(const void *table, int64_t ldt, int vocab, int d, const int *tok, int rows, float scale, int dtype, int out_dtype,
                                                              void *out, int64_t ldo) {
  const int cols = (d + 7) / 8, per = cols < kEmbedThreads ? kEmbedThreads / cols : 1;
  const int mine = cols < kEmbedThreads ? threadIdx.x / cols : 0, c0 = cols < kEmbedThreads ? threadIdx.x % cols : threadIdx.x;
  if (mine >= per) return;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * per + mine;
  if (row >= rows) return;
  const int t = tok[row];
  const bool real = t >= 0 && t < vocab;
  for (int c = c0; c < cols; c += kEmbedThreads) {
    const int n = d - 8 * c;
    Columns x = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
    if (real) {
      x = n >= 8 ? load_columns<true>(table, t * ldt + c * 8, n, dtype) : load_columns<false>(table, t * ldt + c * 8, n, dtype);
#pragma unroll
      for (int j = 0; j < 8; j++) x.x[j] *= scale;
    }
    store_columns(out, row * ldo + c * 8, n, out_dtype, x);
  }
}

// ---- sorting ------------------------------------------------------------------------------------

constexpr int kRankThreads = 1024, kRankMine = 64;            // a workgroup places 64 positions; each of its 16 wavefronts counts in a sixteenth of the tile
// The key of a position: its token, padding behind all tokens
__device__ __forceinline__ int key_of(int t, int vocab) { return t >= 0 && t < vocab ? t : vocab; }

__global__ __launch_bounds__(kRankThreads) void embed_rank_kernel(const int *tok, int rows, int vocab, int *keys, int *order) {
  __shared__ __attribute__((aligned(16))) int sh[kTile];
  __shared__ int count[kRankThreads];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * kRankMine, tile = first / kTile * kTile, n = min(rows - tile, kTile);
  for (int i = threadIdx.x; i < kTile; i += kRankThreads) sh[i] = i < n ? key_of(tok[tile + i], vocab) : 0x7FFFFFFF;
  __syncthreads();
  const int me = first - tile + lane, key = sh[me];
  constexpr int kEach = kTile / 16;
  const int j0 = wave * kEach;
  int smaller = 0;
  auto under = [&](int from, int to, int limit) {             // keys under the limit in part of the share (what lies behind n is larger than any key)
#pragma unroll 8
    for (int j = from; j < to; j += 4) {
      const int4 k = *(const int4 *)(sh + j);
      smaller += (k.x < limit) + (k.y < limit) + (k.z < limit) + (k.w < limit);
    }
  };
  if (j0 < n) {                                               // equal keys of earlier positions count
    const int begin = min(max(first - tile, j0), j0 + kEach), end = min(max(first - tile + kRankMine, j0), j0 + kEach);   // the workgroup's own positions
    under(j0, begin, key + 1);
    for (int j = begin; j < end; j += 4) {
      const int4 k = *(const int4 *)(sh + j);
      smaller += (k.x < key + (j < me)) + (k.y < key + (j + 1 < me)) + (k.z < key + (j + 2 < me)) + (k.w < key + (j + 3 < me));
    }
    under(end, j0 + kEach, key);
  }
  count[threadIdx.x] = smaller;
  __syncthreads();
  if (wave != 0 || me >= n) return;
  int place = 0;
#pragma unroll
  for (int w = 0; w < 16; w++) place += count[w * 64 + lane];
  keys[tile + place] = key;
  order[tile + place] = tile + me;
}

// Runs of `run` sorted positions, kWays at a time, to one each: the place of each among them.  A search looks at kProbes places at once,
// and the searches in all other runs go side by side: a step is one trip to memory.  (16384 positions 4.8 us, one tile after the other
// through the LDS 6, the other three in the LDS at once 6.4; 2^20 120 against 850.)
constexpr int kWays = 4, kProbes = 3, kMergeThreads = 256;
__global__ __launch_bounds__(kMergeThreads) void embed_merge_kernel(const int *from_keys, const int *from_order, int rows, int run, int *keys, int *order) {
  const int i = blockIdx.x * kMergeThreads + threadIdx.x;
  if (i >= rows) return;
  const int key = from_keys[i], at = from_order[i];
  const int base = blockIdx.x * kMergeThreads / run / kWays * kWays * run, mine = (blockIdx.x * kMergeThreads - base) / run;   // of the runs that meet
  int lo[kWays - 1], open[kWays - 1], below[kWays - 1], place = i - mine * run;
#pragma unroll
  for (int o = 0; o < kWays - 1; o++) {
    const int other = o < mine ? o : o + 1;
    lo[o] = min(rows, base + other * run);
    open[o] = min(rows, base + (other + 1) * run) - lo[o];
    below[o] = key + (other < mine ? 1 : 0);                  // equal keys of earlier runs come before
    place -= lo[o];
  }
  auto probe = [](int n, int q) { return (int)((unsigned)(n * q) / (kProbes + 1)); };   // of n open places, q = 1 .. kProbes
  for (int left = run; left > 0; left /= kProbes + 1) {       // keys[x] < below for x < lo, not for x >= lo + open; open <= left
    int k[kWays - 1][kProbes];
#pragma unroll
    for (int o = 0; o < kWays - 1; o++)
#pragma unroll
      for (int q = 0; q < kProbes; q++) k[o][q] = from_keys[min(lo[o] + probe(open[o], q + 1), rows - 1)];
#pragma unroll
    for (int o = 0; o < kWays - 1; o++) {
      const int n = open[o];
      int from = 0, to = n;
#pragma unroll
      for (int q = 0; q < kProbes; q++) from = k[o][q] < below[o] ? min(probe(n, q + 1) + 1, n) : from;
#pragma unroll
      for (int q = kProbes - 1; q >= 0; q--) to = k[o][q] < below[o] ? to : min(probe(n, q + 1), n);
      lo[o] += from;
      open[o] = to - from;
    }
  }
#pragma unroll
  for (int o = 0; o < kWays - 1; o++) place += lo[o];
  keys[place] = key;
  order[place] = at;
}

// ---- sums ---------------------------------------------------------------------------------------

// The number of keys below v, by one wavefront: 64 places are looked at at a time.  Every lane gets it.
__device__ __forceinline__ int keys_below(const int *keys, int rows, int v) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = rows;                                      // keys[i] < v for i < lo, not for i >= hi
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const uint64_t less = __ballot(at < hi && keys[min(at, rows - 1)] < v);   // (a run of the first lanes: the keys are sorted)
    const int n = __popcll(less);
    if (n == 0) return lo;
    hi = min(hi, lo + n * step);
    lo += (n - 1) * step + 1;
  }
  return lo;
}

// The first sorted position of every token (starts[vocab]: where padding begins; a workgroup has 256 tokens, whose share of the keys two
// of its wavefronts look up first), and the runs of 32.  BF16: dy's type (asked at each load, every load waited for the one before).
template <bool BF16>
__global__ __launch_bounds__(kEmbedThreads) void embed_runs_kernel(EmbedGradArgs a, const int *keys, const int *order, int *starts, int start_groups, float *runs) {
  __shared__ int range[2];
  if ((int)blockIdx.x < start_groups) {
    if (blockIdx.y != 0) return;
    const int v0 = blockIdx.x * kEmbedThreads, v = v0 + threadIdx.x, wave = threadIdx.x >> 6;
    if (wave < 2) {
      const int n = keys_below(keys, a.rows, v0 + wave * kEmbedThreads);
      if ((threadIdx.x & 63) == 0) range[wave] = n;
    }
    __syncthreads();
    if (v > a.vocab) return;
    int lo = range[0], hi = range[1];
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (keys[mid] < v) lo = mid + 1; else hi = mid;
    }
    starts[v] = lo;
    return;
  }
  const int run = blockIdx.x - start_groups;
  const int key = keys[run * kRun];
  if (key >= a.vocab || key != keys[run * kRun + kRun - 1]) return;
  for (int c = (blockIdx.y * kEmbedThreads + threadIdx.x) * 8; c < a.d; c += gridDim.y * kEmbedThreads * 8) {
    auto sum = [&](auto whole) __attribute__((always_inline)) {
      constexpr bool kWhole = decltype(whole)::value;
      Columns s = load_columns<kWhole>(a.dy, order[run * kRun] * a.ldy + c, a.d - c, BF16);
#pragma unroll 16
      for (int i = 1; i < kRun; i++) add_columns(s, load_columns<kWhole>(a.dy, order[run * kRun + i] * a.ldy + c, a.d - c, BF16));
      store_columns(runs, (int64_t)run * a.d + c, a.d - c, false, s);
    };
    if (a.d - c >= 8) sum(std::true_type{}); else sum(std::false_type{});
  }
}

// The runs of 1024, out of those of 32
__global__ __launch_bounds__(kEmbedThreads) void embed_long_runs_kernel(const int *keys, int vocab, int d, const float *runs, float *long_runs) {
  const int run = blockIdx.x, key = keys[run * kRuns];
  if (key >= vocab || key != keys[run * kRuns + kRuns - 1]) return;
  for (int c = blockIdx.y * kEmbedThreads + threadIdx.x; c < d; c += gridDim.y * kEmbedThreads) {
    const float *p = runs + (int64_t)run * (kRuns / kRun) * d + c;
    float s = p[0];
#pragma unroll 8
    for (int i = 1; i < kRuns / kRun; i++) s += p[(int64_t)i * d];
    long_runs[(int64_t)run * d + c] = s;
  }
}

// A few table rows to a workgroup (blockIdx.y: its share of the columns).  SPLIT: they are short, its threads take 2, 4 or 8 at once.
constexpr int kTableRows = 8;
template <bool BF16, bool SPLIT>
__global__ __launch_bounds__(kEmbedThreads) void embed_table_kernel(EmbedGradArgs a, const int *order, const int *starts, const float *runs, const float *long_runs) {
  const int v0 = blockIdx.x * kTableRows, vn = min(a.vocab - v0, kTableRows);
  int start[kTableRows + 1];                                  // (all asked for at once; most rows of a large vocabulary have no token, and their zeros go out first)
#pragma unroll
  for (int r = 0; r <= kTableRows; r++) start[r] = starts[min(v0 + r, a.vocab)];
  uint32_t full = 0;
#pragma unroll
  for (int r = 0; r < kTableRows; r++) {
    if (start[r] != start[r + 1]) full |= 1u << r;
    else if (!a.accumulate && r < vn)
      for (int c = (blockIdx.y * kEmbedThreads + threadIdx.x) * 8; c < a.d; c += gridDim.y * kEmbedThreads * 8)
        clear_columns(a.dtable, (v0 + r) * a.ldt + c, a.d - c, a.out_dtype);
  }
  auto walk = [&](int v, int c0) __attribute__((always_inline)) {
    const int s0 = starts[v], s1 = starts[v + 1];
    for (int c = c0; c < a.d; c += gridDim.y * kEmbedThreads * 8) {
      const int n = a.d - c;
      auto sum = [&](auto whole_columns) __attribute__((always_inline)) {
        constexpr bool kWhole = decltype(whole_columns)::value;
        Columns s = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
        int i = s0;
        auto single = [&](int to) __attribute__((always_inline)) {
#pragma unroll 4
          for (; i < to; i++) add_columns(s, load_columns<kWhole>(a.dy, order[i] * a.ldy + c, n, BF16));
        };
        auto whole = [&](const float *p, int length, int to) __attribute__((always_inline)) {   // runs, from a multiple of their length on
#pragma unroll 8
          for (; i + length <= to; i += length) add_columns(s, load_columns<kWhole>(p, (int64_t)(i / length) * a.d + c, n, false));
        };
        single(min(s1, (i + kRun - 1) / kRun * kRun));
        if (i + kRun <= s1) {
          if (a.rows >= kLongLeast) {
            whole(runs, kRun, min(s1, (i + kRuns - 1) / kRuns * kRuns));
            whole(long_runs, kRuns, s1);
          }
          whole(runs, kRun, s1);
        }
        single(s1);
        const int64_t at = v * a.ldt + c;
#pragma unroll
        for (int j = 0; j < 8; j++) s.x[j] *= a.scale;
        if (a.accumulate) add_columns(s, load_columns<kWhole>(a.dtable, at, n, a.out_dtype));
        store_columns(a.dtable, at, n, a.out_dtype, s);
      };
      if (n >= 8) sum(std::true_type{}); else sum(std::false_type{});
    }
  };
  if constexpr (!SPLIT) {
    for (; full != 0; full &= full - 1) walk(v0 + __builtin_ctz(full), (blockIdx.y * kEmbedThreads + threadIdx.x) * 8);
  } else {                                                    // rows r, r + at_once, ..
    const int cols = (a.d + 7) / 8, at_once = cols > kEmbedThreads / 4 ? 2 : cols > kEmbedThreads / 8 ? 4 : 8, mine = threadIdx.x / cols;
    if (mine >= at_once) return;
    for (full &= (at_once == 2 ? 0x55u : at_once == 4 ? 0x11u : 0x01u) << mine; full != 0; full &= full - 1) walk(v0 + __builtin_ctz(full), (threadIdx.x - mine * cols) * 8);
  }
}

// What the scratch holds, in order
struct EmbedScratch { uint64_t keys, order, tile_keys, tile_order, starts, runs, long_runs, bytes; };
EmbedScratch embed_scratch(int rows, int vocab, int d) {
  EmbedScratch s{};
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t here = at; at += (bytes + 255) / 256 * 256; return here; };
  s.keys = take(4ull * rows);
  s.order = take(4ull * rows);
  s.tile_keys = take(rows > kTile ? 4ull * rows : 0);
  s.tile_order = take(rows > kTile ? 4ull * rows : 0);
  s.starts = take(4ull * (vocab + 1));
  s.runs = take(4ull * (rows / kRun) * d);
  s.long_runs = take(rows >= kLongLeast ? 4ull * (rows / kRuns) * d : 0);
  s.bytes = at;
  return s;
}

template <bool BF16> hipError_t embed_sums(const EmbedGradArgs &a, const EmbedScratch &s, char *base, hipStream_t st) {
  int *keys = (int *)(base + s.keys), *order = (int *)(base + s.order), *starts = (int *)(base + s.starts);
  float *runs = (float *)(base + s.runs), *long_runs = (float *)(base + s.long_runs);
  const int slices = (a.d + kEmbedThreads * 8 - 1) / (kEmbedThreads * 8), start_groups = (a.vocab + kEmbedThreads) / kEmbedThreads;
  const int ys = slices > 64 ? 64 : slices;
  hipLaunchKernelGGL(embed_runs_kernel<BF16>, dim3(start_groups + a.rows / kRun, ys), dim3(kEmbedThreads), 0, st, a, keys, order, starts, start_groups, runs);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.rows >= kLongLeast) {
    const int wide = (a.d + kEmbedThreads - 1) / kEmbedThreads;
    hipLaunchKernelGGL(embed_long_runs_kernel, dim3(a.rows / kRuns, wide > 64 ? 64 : wide), dim3(kEmbedThreads), 0, st, keys, a.vocab, a.d, runs, long_runs);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  // Rows at once pay where most have tokens (16384 rows into 1000 x 256 44 -> 28 us, 65536 into 2000 x 256 88 -> 53); one after the
  // other they keep their places in scalar registers (8192 into 128256 x 512 46 us, at once 49).
  const bool split = a.d <= kEmbedThreads * 4 && a.rows >= a.vocab / 4;
  const auto table = split ? embed_table_kernel<BF16, true> : embed_table_kernel<BF16, false>;
  hipLaunchKernelGGL(table, dim3((a.vocab + kTableRows - 1) / kTableRows, ys), dim3(kEmbedThreads), 0, st, a, order, starts, runs, long_runs);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(int dtype, const void *table, int64_t ldt, int vocab, int d, const int *tok, int rows, float scale, int out_dtype, void *out, int64_t ldo,
                        hipStream_t st) {
  const int cols = (d + 7) / 8, per = cols < kEmbedThreads ? kEmbedThreads / cols : 1;
  const int64_t groups = ((int64_t)rows + per - 1) / per, deep = (groups + (1 << 23) - 1) >> 23;   // (a grid's dimension holds less than 2^32 threads)
  const dim3 grid((unsigned)((groups + deep - 1) / deep), (unsigned)deep);
  hipLaunchKernelGGL(embed_kernel, grid, dim3(kEmbedThreads), 0, st, table, ldt, vocab, d, tok, rows, scale, dtype, out_dtype, out, ldo);
  return hipGetLastError();
}

uint64_t embed_grad_scratch_bytes(int rows, int vocab, int d) { return embed_scratch(rows, vocab, d).bytes; }

hipError_t launch_embed_grad(EmbedGradArgs a, void *scratch, hipStream_t st) {
  const EmbedScratch s = embed_scratch(a.rows, a.vocab, a.d);
  char *base = (char *)scratch;
  int *keys[2] = {(int *)(base + s.keys), (int *)(base + s.tile_keys)}, *order[2] = {(int *)(base + s.order), (int *)(base + s.tile_order)};
  int at = 0;                                                 // where the runs are: the last ones, in [0]
  for (int64_t run = kTile; run < a.rows; run *= kWays) at ^= 1;
  hipLaunchKernelGGL(embed_rank_kernel, dim3((a.rows + kRankMine - 1) / kRankMine), dim3(kRankThreads), 0, st, a.tok, a.rows, a.vocab, keys[at], order[at]);
  hipError_t e = hipGetLastError();
  for (int64_t run = kTile; run < a.rows && e == hipSuccess; run *= kWays, at ^= 1) {
    hipLaunchKernelGGL(embed_merge_kernel, dim3((a.rows + kMergeThreads - 1) / kMergeThreads), dim3(kMergeThreads), 0, st, keys[at], order[at], a.rows, (int)run, keys[at ^ 1], order[at ^ 1]);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  return a.dtype ? embed_sums<true>(a, s, base, st) : embed_sums<false>(a, s, base, st);
}

}  // namespace spec
