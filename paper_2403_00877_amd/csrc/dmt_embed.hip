// dmt_embed_fwd, dmt_embed_bwd: a table's rows by id, scaled, and the table's gradient in dense form.
//
// Backward.  The lookups are sorted by id, stably, as (id, position) records: few of them in one launch, many by a
// radix sort of up to 11 bits a digit, three launches a digit.  Then equal tiles of the sorted records are walked, each
// gradient row read once, and rows whose run spans tiles are joined from partial sums in a last launch.  One
// writer per row, no atomics on values, every order fixed: the same bits every time.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256;

// ------------------------------------------------------------------ forward

// A group of 2^log2_lpr lanes per id; a lane takes 16 bytes of the table's row at a time.
template <int TD, int OD>
__global__ __launch_bounds__(kBlock) void embed_fwd_kernel(
    const char* __restrict__ table, int64_t rows, int cols, int64_t table_stride,
    const int32_t* __restrict__ ids, int64_t n, float scale, char* __restrict__ out, int64_t out_stride,
    unsigned long long* __restrict__ first_bad, int log2_lpr) {
  constexpr int E = dmt::ChunkElems<TD>::value, TB = dmt::EltBytes<TD>::value, OB = dmt::EltBytes<OD>::value;
  const int lane = threadIdx.x & ((1 << log2_lpr) - 1);
  const int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> log2_lpr;
  if (i >= n) return;
  const int32_t id = ids[i];
  const bool there = id >= 0 && id < rows;
  if (id >= rows && lane == 0 && first_bad) atomicMin(first_bad, (unsigned long long)i);
  const char* src = table + (there ? id : 0) * table_stride * TB;
  char* dst = out + i * out_stride * OB;
  for (int c = lane * E; c < cols; c += E << log2_lpr) {
    const int valid = min(E, cols - c);
    float x[E];
    if (there) {
      dmt::load_elems<TD, E>(src + (int64_t)c * TB, valid, x);
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] *= scale;
    } else {
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] = 0.f;
    }
    dmt::store_elems<OD, E>(dst + (int64_t)c * OB, valid, x);
  }
}

// ------------------------------------------------------------------ the lookups in order of their ids

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64, kMaxItems = 16;
constexpr int kMaxDigit = 11;
constexpr int64_t kSortFill = 256;           // blocks a pass is spread over, before a block takes more records

// An absent id gets the key `rows`, behind every row's.
__device__ __forceinline__ uint32_t id_key(int32_t id, uint32_t rows) {
  return id < 0 || (uint32_t)id >= rows ? rows : (uint32_t)id;
}

template <bool First>
__device__ __forceinline__ uint64_t record(const int32_t* ids, const uint64_t* in, int64_t j, uint32_t rows) {
  if constexpr (First) return (uint64_t)id_key(ids[j], rows) << 32 | (uint32_t)j;
  else return in[j];
}

// counts[block][digit] of the block's records.
template <bool First>
__global__ __launch_bounds__(kSortBlock) void embed_digits(
    const int32_t* __restrict__ ids, const uint64_t* __restrict__ in, int64_t n, uint32_t rows, int items,
    int shift, int bits, uint32_t* __restrict__ counts, uint32_t* __restrict__ touched, int64_t touched_words,
    unsigned long long* __restrict__ first_bad) {
  __shared__ uint32_t cnt[1 << kMaxDigit];
  const int nd = 1 << bits;
  if (First)                                 // (set by this digit's scatter)
    for (int64_t i = (int64_t)blockIdx.x * kSortBlock + threadIdx.x; i < touched_words; i += (int64_t)gridDim.x * kSortBlock)
      touched[i] = 0;
  for (int d = threadIdx.x; d < nd; d += kSortBlock) cnt[d] = 0;
  __syncthreads();
  const int64_t j0 = (int64_t)blockIdx.x * kSortBlock * items;
  for (int q = 0; q < items; ++q) {
    const int64_t j = j0 + q * kSortBlock + threadIdx.x;
    if (j >= n) break;
    if (First && first_bad && ids[j] >= 0 && (uint32_t)ids[j] >= rows) atomicMin(first_bad, (unsigned long long)j);
    const uint32_t key = (uint32_t)(record<First>(ids, in, j, rows) >> 32);
    atomicAdd(&cnt[key >> shift & (nd - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < nd; d += kSortBlock) counts[(int64_t)blockIdx.x * nd + d] = cnt[d];
}

// counts[block][digit] -> records of that digit in earlier blocks; totals[digit].
__global__ __launch_bounds__(64) void embed_digit_starts(uint32_t* __restrict__ counts, int64_t nblk,
                                                         int nd, uint32_t* __restrict__ totals) {
  const int d = blockIdx.x * 64 + threadIdx.x;
  if (d >= nd) return;
  uint32_t run = 0;
  for (int64_t b0 = 0; b0 < nblk; b0 += 16) {
    uint32_t v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = b0 + u < nblk ? counts[(b0 + u) * nd + d] : 0u;
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      if (b0 + u < nblk) counts[(b0 + u) * nd + d] = run;
      run += v[u];
    }
  }
  totals[d] = run;
}

// Stable scatter.  A wave ranks 64 * items consecutive records, 64 at a time, by ballots of the digit's bits.
template <bool First>
__global__ __launch_bounds__(kSortBlock) void embed_scatter(
    const int32_t* __restrict__ ids, const uint64_t* __restrict__ in, int64_t n, uint32_t rows, int items,
    int shift, int bits, const uint32_t* __restrict__ counts, const uint32_t* __restrict__ totals,
    uint64_t* __restrict__ out, uint8_t* __restrict__ touched) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  const int nd = 1 << bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t* base = lds;                                   // [nd]
  uint16_t* mine = (uint16_t*)(lds + nd);                 // [waves][nd] records of the digit in this wave so far
  __shared__ uint32_t sm[kSortWaves];
  for (int d = threadIdx.x; d < nd * kSortWaves / 2; d += kSortBlock) ((uint32_t*)mine)[d] = 0;
  // first record of each digit: a scan of the totals (two digits a thread at most), then the earlier blocks' share
  uint32_t before = 0;
  for (int d0 = 0; d0 < nd; d0 += kSortBlock) {
    const int d = d0 + (int)threadIdx.x;
    uint32_t all;
    const uint32_t e = dmt::block_exclusive_scan<kSortWaves>(d < nd ? totals[d] : 0u, sm, all);
    if (d < nd) base[d] = before + e + counts[(int64_t)blockIdx.x * nd + d];
    before += all;
  }
  __syncthreads();
  const int64_t j0 = ((int64_t)blockIdx.x * kSortWaves + wave) * 64 * items + lane;
  uint64_t rec[kMaxItems];
  uint16_t rank[kMaxItems];
#pragma unroll
  for (int q = 0; q < kMaxItems; ++q)
    if (q < items) {
      const int64_t j = j0 + q * 64;
      rec[q] = j < n ? record<First>(ids, in, j, rows) : ~0ull;
    }
#pragma unroll
  for (int q = 0; q < kMaxItems; ++q)
    if (q < items) {
      const bool here = j0 + q * 64 < n;
      const uint32_t d = (uint32_t)(rec[q] >> 32) >> shift & (nd - 1);
      uint64_t same = __ballot(here);
      for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot(d >> b & 1);
        same &= d >> b & 1 ? ones : ~ones;
      }
      const int below = __popcll(same & ((1ull << lane) - 1));
      if (here) {
        const uint16_t had = mine[wave * nd + d];
        rank[q] = had + below;
        // (the wave runs in step: all of its lanes have read before the first of them writes)
        __builtin_amdgcn_wave_barrier();
        if (below == 0) mine[wave * nd + d] = had + (uint16_t)__popcll(same);
      }
      __builtin_amdgcn_wave_barrier();
    }
  __syncthreads();
  // earlier waves' records of each digit
  for (int d = threadIdx.x; d < nd; d += kSortBlock) {
    uint32_t run = 0;
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = mine[w * nd + d];
      mine[w * nd + d] = (uint16_t)run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kMaxItems; ++q)
    if (q < items && j0 + q * 64 < n) {
      const uint32_t d = (uint32_t)(rec[q] >> 32) >> shift & (nd - 1);
      out[base[d] + mine[wave * nd + d] + rank[q]] = rec[q];
      if (First) touched[rec[q] >> 32] = 1;              // (absent ids have a byte of their own, behind the rows')
    }
}

// Few lookups: the whole sort in one launch.  A block owns a range of rows and looks at every id itself, twice:
// first it counts, per wave (a wave has a consecutive share of the ids) and row, and how many ids lie below its
// range; then every id of the range has its place.  Counts are 16 bits, so n stays below 65536.
constexpr int kFewRows = 4096;               // rows of a block, at most: counts of 16 waves take 128 KB
constexpr int64_t kFewBlocks = 256;          // ... and the least number of blocks
constexpr int64_t kFewNnz = 65535, kFewWork = 1 << 25;
constexpr int kFewUnroll = 8;
__global__ __launch_bounds__(kSortBlock) void embed_sort_few(
    const int32_t* __restrict__ ids, int n, uint32_t rows, int range, uint64_t* __restrict__ out,
    uint16_t* __restrict__ touched, unsigned long long* __restrict__ first_bad) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];        // [waves][range / 2], two rows a word
  __shared__ uint32_t sm[kSortWaves];
  __shared__ uint32_t s_below;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, words = range / 2;
  const uint32_t first = blockIdx.x * (uint32_t)range;
  for (int i = threadIdx.x; i < words * kSortWaves; i += kSortBlock) lds[i] = 0;
  if (threadIdx.x == 0) s_below = 0;
  __syncthreads();
  const int per = (n + kSortBlock - 1) / kSortBlock * 64;
  const int j0 = wave * per, j1 = min(n, j0 + per);
  uint32_t* mine = lds + wave * words;
  auto keys = [&](int j, uint32_t (&key)[kFewUnroll]) {
#pragma unroll
    for (int u = 0; u < kFewUnroll; ++u) {
      const int at = j + u * 64 + lane;
      key[u] = at < j1 ? (uint32_t)ids[at] : ~0u;
    }
  };
  uint32_t below = 0;
  for (int j = j0; j < j1; j += kFewUnroll * 64) {
    uint32_t key[kFewUnroll];
    keys(j, key);
#pragma unroll
    for (int u = 0; u < kFewUnroll; ++u) {
      const int at = j + u * 64 + lane;
      if (at >= j1) continue;
      if (blockIdx.x == 0 && first_bad && (int32_t)key[u] >= 0 && key[u] >= rows)
        atomicMin(first_bad, (unsigned long long)at);
      const uint32_t v = min(key[u], rows), d = v - first;              // (a negative id is a large unsigned one)
      below += v < first;
      if (d < (uint32_t)range) atomicAdd(&mine[d >> 1], 1u << (d & 1) * 16);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o);
  if (lane == 0) atomicAdd(&s_below, below);
  __syncthreads();
  // counts -> places inside the block's records
  uint32_t before = 0;
  for (int p0 = 0; p0 < words; p0 += kSortBlock) {
    const int p = p0 + (int)threadIdx.x;
    uint32_t c[kSortWaves], a = 0, b = 0;
    if (p < words) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t v = lds[w * words + p];
        c[w] = a | b << 16;
        a += v & 0xffffu;
        b += v >> 16;
      }
    }
    uint32_t all;
    const uint32_t at = before + dmt::block_exclusive_scan<kSortWaves>(a + b, sm, all);
    before += all;
    if (p < words) {
      const uint32_t add = (at & 0xffffu) | (at + a) << 16;             // (no place passes n)
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) lds[w * words + p] = c[w] + add;
      touched[first / 2 + p] = (uint16_t)((a > 0) | (b > 0) << 8);
    }
  }
  __syncthreads();
  uint64_t* dst = out + s_below;
  uint16_t* place = (uint16_t*)mine;
  for (int j = j0; j < j1; j += kFewUnroll * 64) {
    uint32_t key[kFewUnroll];
    keys(j, key);
#pragma unroll
    for (int u = 0; u < kFewUnroll; ++u) {
      const int at = j + u * 64 + lane;
      const uint32_t v = min(key[u], rows), d = v - first;
      const bool here = at < j1 && d < (uint32_t)range;
      uint64_t left = __ballot(here);
      while (left) {                                                    // one row of the 64 ids at a time
        const uint32_t row = __builtin_amdgcn_readlane(d, __builtin_ctzll(left));
        const uint64_t same = __ballot(here && d == row);
        const uint32_t from = place[row];
        __builtin_amdgcn_wave_barrier();
        if (here && d == row) {
          dst[from + __popcll(same & ((1ull << lane) - 1))] = (uint64_t)v << 32 | (uint32_t)at;
          place[row] = (uint16_t)(from + __popcll(same));               // (the same from every lane)
        }
        __builtin_amdgcn_wave_barrier();
        left &= ~same;
      }
    }
  }
}

// ------------------------------------------------------------------ the sums

// The sorted records are cut into tiles of equal length; a lane group walks one, with kUnroll gradient rows under way, and
// writes a row when its run ends.  Runs that cross a tile's end leave partial sums: part[tile][0] of the
// run that came from the tile before, part[tile][1] of one that starts here and goes on.  Blocks behind the
// tiles' clear the rows that no id names.
constexpr int kUnroll = 8;
constexpr int kFillBytes = 65536;            // of the table, cleared by a block

struct Sums {
  const uint64_t* recs;
  int64_t n, rows;
  const char* grad;
  int64_t grad_stride;
  float scale;
  float* out;
  int64_t out_stride;
  int cols, part_cols, accumulate, log2_lpr, tile;
  int64_t ntiles, tile_blocks;
  int slices;
  float* part;
  const uint8_t* touched;
  int log2_fill;                             // lanes that clear a row, and rows a block looks at
  int fill_rows;
};

__device__ __forceinline__ uint32_t key_at(const uint64_t* recs, int64_t j) { return (uint32_t)(recs[j] >> 32); }

template <int E>
__device__ __forceinline__ void write_row(const Sums& a, uint32_t row, int c, int valid, float (&acc)[E]) {
  char* dst = (char*)(a.out + row * a.out_stride + c);
  float x[E];
  if (a.accumulate) dmt::load_elems<DMT_F32, E>(dst, valid, x);
#pragma unroll
  for (int q = 0; q < E; ++q) acc[q] = a.accumulate ? fmaf(a.scale, acc[q], x[q]) : a.scale * acc[q];
  dmt::store_elems<DMT_F32, E>(dst, valid, acc);
}

__device__ __forceinline__ void clear_rows(const Sums& a) {
  const int lane = threadIdx.x & ((1 << a.log2_fill) - 1);
  const int64_t v0 = (blockIdx.x - a.tile_blocks) * a.fill_rows, v1 = min(a.rows, v0 + a.fill_rows);
  const float zero[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t v = v0 + (threadIdx.x >> a.log2_fill); v < v1; v += kBlock >> a.log2_fill) {
    if (a.touched[v]) continue;
    for (int c = lane * 4; c < a.cols; c += 4 << a.log2_fill)
      dmt::store_elems<DMT_F32, 4>((char*)(a.out + v * a.out_stride + c), min(4, a.cols - c), zero);
  }
}

template <int GD>
__global__ __launch_bounds__(kBlock) void embed_sums(const Sums a) {
  constexpr int E = dmt::ChunkElems<GD>::value, GB = dmt::EltBytes<GD>::value;
  if (blockIdx.x >= a.tile_blocks) {
    clear_rows(a);
    return;
  }
  const int lane = threadIdx.x & ((1 << a.log2_lpr) - 1);
  const int64_t tile = (int64_t)(blockIdx.x / (unsigned)a.slices) * (kBlock >> a.log2_lpr) + (threadIdx.x >> a.log2_lpr);
  const int c = (int)((blockIdx.x % (unsigned)a.slices << a.log2_lpr) + lane) * E;
  if (tile >= a.ntiles || c >= a.cols) return;
  const int valid = min(E, a.cols - c);
  const int64_t j0 = tile * a.tile, j1 = min(a.n, j0 + a.tile);
  const uint32_t rows = (uint32_t)a.rows;
  const uint32_t prev = j0 > 0 ? key_at(a.recs, j0 - 1) : ~0u, next = j1 < a.n ? key_at(a.recs, j1) : ~0u;
  uint32_t cur = rows;
  float acc[E];
  auto flush = [&]() {
    if (cur >= rows) return;
    if (cur == prev || cur == next)
      dmt::store_elems<DMT_F32, E>((char*)(a.part + (tile * 2 + (cur != prev)) * a.part_cols + c), E, acc);
    else
      write_row<E>(a, cur, c, valid, acc);
  };
  for (int64_t j = j0; j < j1; j += kUnroll) {
    uint64_t rec[kUnroll];
    dmt::Raw<GD, E> g[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) rec[u] = a.recs[min(j + u, j1 - 1)];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      g[u] = dmt::load_raw<GD, E>(a.grad + ((int64_t)(uint32_t)rec[u] * a.grad_stride + c) * GB, valid);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (j + u >= j1) break;
      const uint32_t key = (uint32_t)(rec[u] >> 32);
      if (key != cur) {
        flush();
        cur = key;
#pragma unroll
        for (int q = 0; q < E; ++q) acc[q] = 0.f;
      }
      float x[E];
      dmt::unpack<GD, E>(g[u], x);
#pragma unroll
      for (int q = 0; q < E; ++q) acc[q] += x[q];
    }
  }
  flush();
}

// Rows whose run spans tiles: their partial sums, in the tiles' order.  A block looks at kJoinTiles tiles; each
// lane group takes the runs that start in one of them in turn, and the whole block those of many tiles.
constexpr int kJoinTiles = 64, kJoinLong = 32;
__global__ __launch_bounds__(kBlock) void embed_join(const Sums a) {
  constexpr int E = 4;
  __shared__ int s_tile[kJoinTiles], s_len[kJoinTiles];
  __shared__ int s_count;
  __shared__ float s_sum[kBlock * E];
  if (threadIdx.x == 0) s_count = 0;
  __syncthreads();
  const int64_t t0 = (int64_t)blockIdx.x * kJoinTiles;
  if (threadIdx.x < kJoinTiles && t0 + (int)threadIdx.x + 1 < a.ntiles) {
    const int64_t t = t0 + threadIdx.x, b = t * a.tile, e = b + a.tile;
    const uint32_t v = key_at(a.recs, e - 1);
    if ((int64_t)v < a.rows && key_at(a.recs, e) == v &&
        (b == 0 || key_at(a.recs, b) != v || key_at(a.recs, b - 1) != v)) {
      // the last tile that starts with the run: doubling steps, then bisection
      int64_t good = t + 1, step = 1;
      while (good + step < a.ntiles && key_at(a.recs, (good + step) * a.tile) == v) good += step, step *= 2;
      int64_t bad = min(a.ntiles, good + step);
      while (bad - good > 1) {
        const int64_t mid = (good + bad) / 2;
        if (key_at(a.recs, mid * a.tile) == v) good = mid;
        else bad = mid;
      }
      const int at = atomicAdd(&s_count, 1);             // (which group takes which run changes no sum)
      s_tile[at] = (int)threadIdx.x;
      s_len[at] = (int)(good - t);
    }
  }
  __syncthreads();
  const int count = s_count, lane = threadIdx.x & ((1 << a.log2_fill) - 1);
  const int group = threadIdx.x >> a.log2_fill, groups = kBlock >> a.log2_fill;
  auto heads = [&](int64_t t, int from, int to, int c, float (&acc)[E]) {
    const float* p = a.part + t * 2 * a.part_cols + c;
    int i = from;
    for (; i + 8 <= to; i += 8) {
      float4 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = *(const float4*)(p + (int64_t)(i + u) * 2 * a.part_cols);
#pragma unroll
      for (int u = 0; u < 8; ++u) acc[0] += x[u].x, acc[1] += x[u].y, acc[2] += x[u].z, acc[3] += x[u].w;
    }
    for (; i < to; ++i) {
      const float4 x = *(const float4*)(p + (int64_t)i * 2 * a.part_cols);
      acc[0] += x.x, acc[1] += x.y, acc[2] += x.z, acc[3] += x.w;
    }
  };
  auto tail = [&](int64_t t, int c, float (&acc)[E]) {
    const float4 x = *(const float4*)(a.part + (t * 2 + 1) * a.part_cols + c);
    acc[0] = x.x, acc[1] = x.y, acc[2] = x.z, acc[3] = x.w;
  };
  for (int i = group; i < count; i += groups) {
    if (s_len[i] > kJoinLong) continue;
    const int64_t t = t0 + s_tile[i];
    const uint32_t v = key_at(a.recs, (t + 1) * a.tile);
    for (int c = lane * E; c < a.cols; c += E << a.log2_fill) {
      float acc[E];
      tail(t, c, acc);
      heads(t, 1, s_len[i] + 1, c, acc);
      write_row<E>(a, v, c, min(E, a.cols - c), acc);
    }
  }
  for (int i = 0; i < count; ++i) {
    if (s_len[i] <= kJoinLong) continue;
    const int64_t t = t0 + s_tile[i];
    const uint32_t v = key_at(a.recs, (t + 1) * a.tile);
    const int per = (s_len[i] + groups - 1) / groups, from = 1 + group * per, to = min(s_len[i] + 1, from + per);
    for (int c0 = 0; c0 < a.cols; c0 += E << a.log2_fill) {
      const int c = c0 + lane * E;
      float acc[E] = {0.f, 0.f, 0.f, 0.f};
      if (c < a.cols) heads(t, from, to, c, acc);
      __syncthreads();
#pragma unroll
      for (int q = 0; q < E; ++q) s_sum[threadIdx.x * E + q] = acc[q];
      __syncthreads();
      if (group == 0 && c < a.cols) {
        tail(t, c, acc);
        for (int g = 0; g < groups; ++g)
#pragma unroll
          for (int q = 0; q < E; ++q) acc[q] += s_sum[((g << a.log2_fill) + lane) * E + q];
        write_row<E>(a, v, c, min(E, a.cols - c), acc);
      }
    }
  }
}

int log2_lanes(int64_t cols, int E) {
  int l = 0;
  while (l < 6 && (int64_t)(E << l) < cols) ++l;
  return l;
}

// How a call is divided, and where everything lies in the workspace.
struct Ws {
  uint64_t *a, *b;
  uint32_t *counts, *totals;
  uint8_t* touched;
  float* part;
  int64_t nblk, touched_words, ntiles;
  bool few;                                  // one launch sorts
  int range;                                 // rows of a block of it
  int items, passes, bits;
  int tile, part_cols;
  size_t bytes;
};

// Records a lane group walks: as many as leave a wave's worth of groups for every place on the chip, at least 8.
constexpr int64_t kFillLanes = 256 * 2048;
constexpr int kLeastTile = 8;
int tile_of(int64_t n, int64_t cols) {
  int tile = 64;
  const int lanes = 1 << log2_lanes(cols, 8);
  while (tile > kLeastTile && (n + tile - 1) / tile * lanes < kFillLanes) tile /= 2;
  return tile;
}

Ws carve(int64_t n, int64_t rows, int64_t cols, void* at) {
  Ws w;
  w.items = (int)std::min<int64_t>(kMaxItems, std::max<int64_t>(1, (n + kSortBlock * kSortFill - 1) / (kSortBlock * kSortFill)));
  w.nblk = std::max<int64_t>(1, (n + kSortBlock * w.items - 1) / (kSortBlock * w.items));
  int64_t blocks = std::max<int64_t>(kFewBlocks, (rows + kFewRows) / kFewRows);
  w.range = (int)dmt_align_up((size_t)((rows + blocks) / blocks), 32);   // the key `rows` included
  w.few = n <= kFewNnz && n * blocks <= kFewWork;
  int bits = 1;
  while ((rows >> bits) != 0) ++bits;                    // the key `rows` included
  w.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  w.bits = (bits + w.passes - 1) / w.passes;
  w.tile = tile_of(n, cols);
  w.ntiles = (n + w.tile - 1) / w.tile;
  w.part_cols = (int)dmt_align_up((size_t)cols, 8);
  w.touched_words = (int64_t)dmt_align_up((size_t)rows + 1 + w.range, 4) / 4;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = dmt_align_up(off + bytes, 256);
    return (char*)((uintptr_t)at + o);
  };
  w.a = (uint64_t*)take(sizeof(uint64_t) * (size_t)n);
  w.b = (uint64_t*)take(sizeof(uint64_t) * (size_t)n);
  // (never less for fewer lookups in smaller blocks and tiles: a workspace sized for the most serves all calls)
  const int64_t most_blk = std::max(w.nblk, std::min(kSortFill, (n + kSortBlock - 1) / kSortBlock));
  const int64_t most_tiles =
      std::max((n + 63) / 64, std::min((n + kLeastTile - 1) / kLeastTile, 2 * kFillLanes >> log2_lanes(cols, 8)));
  w.counts = (uint32_t*)take(sizeof(uint32_t) * ((size_t)most_blk << w.bits));
  w.totals = (uint32_t*)take(sizeof(uint32_t) << w.bits);
  w.touched = (uint8_t*)take(sizeof(uint32_t) * (size_t)w.touched_words);
  w.part = (float*)take(sizeof(float) * 2 * (size_t)most_tiles * (size_t)w.part_cols);
  w.bytes = off;
  return w;
}

bool sizes_known(int64_t n, int64_t rows, int64_t cols) { return n >= 0 && rows >= 1 && cols >= 1; }
bool sizes_fit(int64_t n, int64_t rows, int64_t cols) {
  return n < (1ll << 31) && rows < (1ll << 31) && cols <= (1 << 24);
}

template <int TD>
void launch_fwd(int32_t od, const void* table, int64_t rows, int64_t cols, int64_t ts, const int32_t* ids,
                int64_t n, float scale, void* out, int64_t os, int64_t* bad, hipStream_t s) {
  const int l = log2_lanes(cols, dmt::ChunkElems<TD>::value);
  const dim3 grid((unsigned)(((n << l) + kBlock - 1) / kBlock));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, (const char*)table, rows, (int)cols, ts, ids, n, scale,
                       (char*)out, os, (unsigned long long*)bad, l);
  };
  if (od == DMT_F32) go(embed_fwd_kernel<TD, DMT_F32>);
  else if (od == DMT_F16) go(embed_fwd_kernel<TD, DMT_F16>);
  else go(embed_fwd_kernel<TD, DMT_BF16>);
}

template <bool First>
void launch_pass(const Ws& w, const int32_t* ids, const uint64_t* in, uint64_t* out, int64_t n, int64_t rows,
                 int shift, int64_t* bad, hipStream_t s) {
  const int nd = 1 << w.bits;
  hipLaunchKernelGGL(embed_digits<First>, dim3((unsigned)w.nblk), dim3(kSortBlock), 0, s, ids, in, n, (uint32_t)rows,
                     w.items, shift, w.bits, w.counts, (uint32_t*)w.touched, w.touched_words, (unsigned long long*)bad);
  hipLaunchKernelGGL(embed_digit_starts, dim3((nd + 63) / 64), dim3(64), 0, s, w.counts, w.nblk, nd, w.totals);
  static DmtPerDevice done;
  dmt_allow_lds(done, (const void*)embed_scatter<First>, (4 + 2 * kSortWaves) << kMaxDigit);
  hipLaunchKernelGGL(embed_scatter<First>, dim3((unsigned)w.nblk), dim3(kSortBlock), (4 + 2 * kSortWaves) << w.bits, s,
                     ids, in, n, (uint32_t)rows, w.items, shift, w.bits, w.counts, w.totals, out, w.touched);
}

void launch_few(const Ws& w, const int32_t* ids, int64_t n, int64_t rows, int64_t* bad, hipStream_t s) {
  static DmtPerDevice done;
  dmt_allow_lds(done, (const void*)embed_sort_few, kFewRows * kSortWaves * 2);
  hipLaunchKernelGGL(embed_sort_few, dim3((unsigned)((rows + w.range) / w.range)), dim3(kSortBlock),
                     w.range * kSortWaves * 2, s, ids, (int)n, (uint32_t)rows, w.range, w.a, (uint16_t*)w.touched,
                     (unsigned long long*)bad);
}

template <int GD>
void launch_sums(Sums a, hipStream_t s) {
  a.log2_lpr = log2_lanes(a.cols, dmt::ChunkElems<GD>::value);
  a.slices = (a.cols + (dmt::ChunkElems<GD>::value << a.log2_lpr) - 1) / (dmt::ChunkElems<GD>::value << a.log2_lpr);
  const int groups = kBlock >> a.log2_lpr;
  a.tile_blocks = (a.ntiles + groups - 1) / groups * a.slices;
  a.log2_fill = log2_lanes(a.cols, 4);
  a.fill_rows = (int)std::max<int64_t>(kBlock >> a.log2_fill, kFillBytes / (4 * a.cols));
  const int64_t fill_blocks = a.accumulate ? 0 : (a.rows + a.fill_rows - 1) / a.fill_rows;
  if (a.tile_blocks + fill_blocks > 0)
    hipLaunchKernelGGL(embed_sums<GD>, dim3((unsigned)(a.tile_blocks + fill_blocks)), dim3(kBlock), 0, s, a);
  if (a.ntiles > 1)
    hipLaunchKernelGGL(embed_join, dim3((unsigned)((a.ntiles + kJoinTiles - 1) / kJoinTiles)), dim3(kBlock), 0, s, a);
}

}  // namespace

extern "C" dmt_status dmt_embed_fwd(const void* table, int64_t rows, int64_t cols, int64_t table_stride,
                                    int32_t table_dtype, const int32_t* ids, int64_t n, float scale,
                                    void* out, int64_t out_stride, int32_t out_dtype, int64_t* first_bad,
                                    void* stream) {
  if (!sizes_known(n, rows, cols) || !dmt_is_dtype(table_dtype) || !dmt_is_dtype(out_dtype) ||
      table_stride < cols || out_stride < cols || !dmt_may_be_at(first_bad, 8))
    return DMT_EINVAL;
  if (!dmt_is_at(table, dmt_ebytes(table_dtype))) return DMT_EINVAL;
  if (n > 0 && (!dmt_is_at(ids, 4) || !dmt_is_at(out, dmt_ebytes(out_dtype)))) return DMT_EINVAL;
  if (!sizes_fit(n, rows, cols)) return DMT_ENOTSUP;
  if (n == 0) return DMT_OK;
  hipStream_t s = (hipStream_t)stream;
  if (table_dtype == DMT_F32)
    launch_fwd<DMT_F32>(out_dtype, table, rows, cols, table_stride, ids, n, scale, out, out_stride, first_bad, s);
  else if (table_dtype == DMT_F16)
    launch_fwd<DMT_F16>(out_dtype, table, rows, cols, table_stride, ids, n, scale, out, out_stride, first_bad, s);
  else
    launch_fwd<DMT_BF16>(out_dtype, table, rows, cols, table_stride, ids, n, scale, out, out_stride, first_bad, s);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" size_t dmt_embed_bwd_workspace_bytes(int64_t n, int64_t rows, int64_t cols) {
  if (!sizes_known(n, rows, cols) || !sizes_fit(n, rows, cols)) return 0;
  return carve(n, rows, cols, nullptr).bytes;
}

extern "C" dmt_status dmt_embed_bwd(const int32_t* ids, int64_t n, const void* grad, int64_t grad_stride,
                                    int32_t grad_dtype, float scale, float* grad_table, int64_t rows,
                                    int64_t cols, int64_t grad_table_stride, int32_t accumulate,
                                    int64_t* first_bad, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  if (!sizes_known(n, rows, cols) || !dmt_is_dtype(grad_dtype) || grad_stride < cols || grad_table_stride < cols ||
      !dmt_may_be_at(first_bad, 8) || !dmt_is_at(grad_table, 4))
    return DMT_EINVAL;
  if (n > 0 && (!dmt_is_at(ids, 4) || !dmt_is_at(grad, dmt_ebytes(grad_dtype)))) return DMT_EINVAL;
  if (!sizes_fit(n, rows, cols)) return DMT_ENOTSUP;
  if (!dmt_is_at(workspace, 256)) return DMT_EINVAL;
  const Ws w = carve(n, rows, cols, workspace);
  if (workspace_bytes < w.bytes) return DMT_ENOMEM;
  hipStream_t s = (hipStream_t)stream;
  uint64_t *in = w.b, *out = w.a;
  if (w.few) {
    launch_few(w, ids, n, rows, first_bad, s);
    std::swap(in, out);
  }
  for (int p = 0; p < w.passes && !w.few; ++p) {
    if (p == 0) launch_pass<true>(w, ids, nullptr, out, n, rows, 0, first_bad, s);
    else launch_pass<false>(w, ids, in, out, n, rows, p * w.bits, first_bad, s);
    std::swap(in, out);
  }
  Sums a = {};
  a.recs = in, a.n = n, a.rows = rows;
  a.grad = (const char*)grad, a.grad_stride = grad_stride, a.scale = scale;
  a.out = grad_table, a.out_stride = grad_table_stride, a.cols = (int)cols, a.accumulate = accumulate != 0;
  a.tile = w.tile, a.ntiles = w.ntiles, a.part = w.part, a.part_cols = w.part_cols, a.touched = w.touched;
  if (grad_dtype == DMT_F32) launch_sums<DMT_F32>(a, s);
  else if (grad_dtype == DMT_F16) launch_sums<DMT_F16>(a, s);
  else launch_sums<DMT_BF16>(a, s);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
