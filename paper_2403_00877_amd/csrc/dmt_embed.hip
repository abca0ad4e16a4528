// dmt_embed_fwd, dmt_embed_bwd: a table's rows by id, scaled, and the table's gradient in dense form.
//
// Forward: out[i] = s W[id_i], in float32, rounded once.  Backward: dW[v] = s sum over id_i = v of g[i], ascending i; zeros (or
// what was there) for rows that no id names.
//
// Backward.  The lookups are sorted by id, stably, as (id, position) records: few of them in one launch, many by a
// radix sort of up to 11 bits a digit, three launches a digit.  Then equal tiles of the sorted records are walked, each
// gradient row read once, and rows whose run spans tiles are joined from partial sums in a last launch.  Up to a few
// thousand ids one launch does it all: every block orders the ids of its own range of rows, sums them and clears the others.  One
// writer per row, no atomics on values, every order fixed: the same bits every time.
// 163840 ids, 1 M rows of 512 bytes (590 MB to move): 126 us, of which the order 35, the sums 53, the join 41, both with the
// clearing beside them.  1003 ids, 10007 x 100: 10 us, a chain of latencies.
#include <algorithm>
#include <type_traits>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256;

// Where the piece of E elements from column c on lies: the last one of a row that is no whole number of pieces ends with the row, and
// what it shares with the one before both write, alike.  (Element by element 100000 ids of 231 bfloat16 took 83.5 us backward, now
// 65, and 22.8 forward, now 19.)
template <int E> __device__ __forceinline__ int piece_at(int c, int cols) { return max(0, min(c, cols - E)); }

// ------------------------------------------------------------------ forward

// A group of 2^log2_lpr lanes per id; a lane takes 16 bytes of the table's row at a time.  Bound by the rows' bytes out and what of the
// table is not in a cache: 262144 ids, rows of 256 bytes, Zipf: 18 us (17 at the least), 67 MB written at 4 TB/s beside the reads; one id 1.6 us.
template <int TD, int OD>
__global__ __launch_bounds__(kBlock) void embed_fwd_kernel(
    unsigned first_block, const char* __restrict__ table, int64_t rows, int cols, int64_t table_stride,
    const int32_t* __restrict__ ids, int64_t n, float scale, char* __restrict__ out, int64_t out_stride,
    unsigned long long* __restrict__ first_bad, int log2_lpr) {
  constexpr int E = dmt::ChunkElems<TD>::value, TB = dmt::EltBytes<TD>::value, OB = dmt::EltBytes<OD>::value;
  const int lane = threadIdx.x & ((1 << log2_lpr) - 1);
  const int64_t i = ((int64_t)(first_block + blockIdx.x) * kBlock + threadIdx.x) >> log2_lpr;
  if (i >= n) return;
  const int32_t id = ids[i];
  const bool there = id >= 0 && id < rows;
  if (id >= rows && lane == 0 && first_bad) atomicMin(first_bad, (unsigned long long)i);
  const char* src = table + (there ? id : 0) * table_stride * TB;
  char* dst = out + i * out_stride * OB;
  for (int piece = lane * E; piece < cols; piece += E << log2_lpr) {
    const int c = piece_at<E>(piece, cols), valid = min(E, cols);
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

// ------------------------------------------------------------------ rows that no id names

// They are cleared by waves of blocks behind those of the sums and of the join, which are bound by latency where the
// clearing is bound by the rate of stores; they pass the caches by (sums and join 114 -> 93 us at 930 K rows of 512 bytes).
// (A row's last piece here not as piece_at(): whole pieces that overlap, past the caches, 80 us for 64 at 28399 ids of 246599 x 231.)
struct Fill {
  const uint8_t* touched;
  float* out;
  int64_t out_stride, rows;
  int cols, log2_lanes, rows_per_wave;       // lanes that clear a row, rows a wave looks at (at most 64)
  unsigned own_blocks;                       // the launch's blocks that do something else
  int64_t first;                             // wave units cleared by earlier launches
};
constexpr int64_t kFillBytes = 16384, kFillWaves = 8192;   // of the table, cleared by a wave, while there are so many of them

// Whether the block is one of those that clear rows; if so it is done.
template <int Waves> __device__ __forceinline__ bool fill_block(const Fill& f) {
  if (blockIdx.x < f.own_blocks) return false;
  const int lane = threadIdx.x & 63, sub = lane & ((1 << f.log2_lanes) - 1);
  const int64_t v0 = (f.first + (int64_t)(blockIdx.x - f.own_blocks) * Waves + (threadIdx.x >> 6)) * f.rows_per_wave;
  const uint64_t empty = __ballot(lane < f.rows_per_wave && v0 + lane < f.rows && !f.touched[v0 + lane]);
  for (int i = lane >> f.log2_lanes; i < f.rows_per_wave; i += 64 >> f.log2_lanes) {
    if (!(empty >> i & 1)) continue;
    for (int c = sub * 4; c < f.cols; c += 4 << f.log2_lanes)
      dmt::clear_elems<4>((char*)(f.out + (v0 + i) * f.out_stride + c), f.cols - c);
  }
  return true;
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

// counts[block][digit] -> records of that digit in earlier blocks; totals[digit].  A wave per 64 digits and sixteenth of the
// blocks (one thread per digit over all the blocks was a chain of dependent batches: 9.6 us at 160 blocks, now 5.1).
constexpr int kStartsSegs = 16, kStartsBatch = 16;
__global__ __launch_bounds__(64 * kStartsSegs) void embed_digit_starts(uint32_t* __restrict__ counts, int64_t nblk,
                                                                       int nd, uint32_t* __restrict__ totals) {
  __shared__ uint32_t sums[kStartsSegs][64];
  const int lane = threadIdx.x & 63, seg = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
  const int64_t per = (nblk + kStartsSegs - 1) / kStartsSegs, b0 = seg * per, b1 = min(nblk, b0 + per);
  uint32_t sum = 0, v[kStartsBatch];
  if (d < nd)
    for (int64_t b = b0; b < b1; b += kStartsBatch) {
#pragma unroll
      for (int u = 0; u < kStartsBatch; ++u) v[u] = b + u < b1 ? counts[(b + u) * nd + d] : 0u;
#pragma unroll
      for (int u = 0; u < kStartsBatch; ++u) sum += v[u];
    }
  sums[seg][lane] = sum;
  __syncthreads();
  uint32_t run = 0, all = 0;
  for (int g = 0; g < kStartsSegs; ++g) {
    run += g < seg ? sums[g][lane] : 0u;
    all += sums[g][lane];
  }
  if (d >= nd) return;
  if (seg == 0) totals[d] = all;
  for (int64_t b = b0; b < b1; b += kStartsBatch) {
    if (per > kStartsBatch)                  // (else they are still at hand)
#pragma unroll
      for (int u = 0; u < kStartsBatch; ++u) v[u] = b + u < b1 ? counts[(b + u) * nd + d] : 0u;
#pragma unroll
    for (int u = 0; u < kStartsBatch; ++u)
      if (b + u < b1) {
        counts[(b + u) * nd + d] = run;
        run += v[u];
      }
  }
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
  const int64_t j0 = ((int64_t)blockIdx.x * kSortWaves + wave) * 64 * items + lane;
  uint64_t rec[kMaxItems];
  uint16_t rank[kMaxItems];
#pragma unroll
  for (int q = 0; q < kMaxItems; ++q)
    if (q < items) {
      const int64_t j = j0 + q * 64;
      rec[q] = j < n ? record<First>(ids, in, j, rows) : ~0ull;
    }
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

// Few lookups: the whole order in one launch.  A block owns a range of rows and looks at every id itself: it counts them,
// per wave (a wave has a consecutive share of the ids) and row, and how many ids lie below its range; then every id of the range has
// its place.  A wave notes the few ids it finds, in their order, and places those; only a wave that finds more than kNotes, which
// the owner of a frequent row does, looks at its share again.  A lane reads four consecutive ids at a time.
// Counts are 16 bits, so n stays below 65536.  The last block's range holds the absent ids, as row `rows`.
//   lds [waves][range / 2], two rows a word: afterwards where each wave's share of a row ends, counted from the
//   block's first record;  counted(pair of rows, count of either) once per pair;
//   placed(ids below the range, place, row, position) once per id of the range
constexpr int kIdsLane = 4, kIdsWave = 64 * kIdsLane, kFewUnroll = 4, kNotes = 128;
template <typename Counted, typename Placed>
__device__ __forceinline__ void order_few(const int32_t* __restrict__ ids, int n, uint32_t rows, int range, uint32_t* lds,
                                          unsigned long long* __restrict__ first_bad, Counted counted,
                                          Placed placed) {
  __shared__ uint32_t sm[kSortWaves];
  __shared__ uint32_t s_below;
  __shared__ uint32_t s_notes[kSortWaves][kNotes];                      // row in the range << 16 | position
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, words = range / 2;
  const uint64_t lower = (1ull << lane) - 1;
  const uint32_t first = blockIdx.x * (uint32_t)range;
  const bool absent_too = first + (uint32_t)range > rows;                // (the last block)
  for (int i = threadIdx.x; i < words * kSortWaves; i += kSortBlock) lds[i] = 0;
  if (threadIdx.x == 0) s_below = 0;
  __syncthreads();
  const int per = (n + kSortWaves * kIdsWave - 1) / (kSortWaves * kIdsWave) * kIdsWave;
  const int j0 = min(n, wave * per), j1 = min(n, j0 + per);
  uint32_t* mine = lds + wave * words;
  // look(position of the first of a lane's four, their rows), 64 * 4 ids at a time
  auto each = [&](auto look) {
    for (int j = j0; j < j1; j += kFewUnroll * kIdsWave) {
      uint32_t key[kFewUnroll][kIdsLane];
      const bool whole = j + kFewUnroll * kIdsWave <= j1;
#pragma unroll
      for (int u = 0; u < kFewUnroll; ++u) {
        const int at = j + u * kIdsWave + lane * kIdsLane;
        if (whole) {
          const auto r = dmt::load_raw<DMT_F32, kIdsLane>((const char*)(ids + at), kIdsLane);
#pragma unroll
          for (int e = 0; e < kIdsLane; ++e) key[u][e] = r.w[e];
        } else {
#pragma unroll
          for (int e = 0; e < kIdsLane; ++e) key[u][e] = at + e < j1 ? (uint32_t)ids[at + e] : ~0u;
        }
      }
#pragma unroll
      for (int u = 0; u < kFewUnroll; ++u) {
        const int at = j + u * kIdsWave + lane * kIdsLane;
        if (absent_too) {                                               // (ids below 0 are large unsigned ones)
#pragma unroll
          for (int e = 0; e < kIdsLane; ++e) key[u][e] = at + e < j1 ? min(key[u][e], rows) : ~0u;
        }
        look(at, key[u]);
      }
    }
  };
  uint32_t below = 0;                                                   // (of the wave)
  int notes = 0;
  each([&](int at, const uint32_t (&key)[kIdsLane]) {
    uint64_t in[kIdsLane], any = 0;
    int before = notes;
#pragma unroll
    for (int e = 0; e < kIdsLane; ++e) {
      below += __popcll(__ballot(key[e] < first));
      in[e] = __ballot(key[e] - first < (uint32_t)range);
      any |= in[e];
    }
    if (!any) return;
#pragma unroll
    for (int e = 0; e < kIdsLane; ++e) {
      before += __popcll(in[e] & lower);
      notes += __popcll(in[e]);
    }
#pragma unroll
    for (int e = 0; e < kIdsLane; ++e) {
      if (!in[e]) continue;
      const uint32_t d = key[e] - first;
      const bool here = in[e] >> lane & 1;
      if (here && before < kNotes) s_notes[wave][before] = d << 16 | (uint32_t)(at + e);
      before += here;
      // of many at once, the first lane's row is counted for all lanes that have it: LDS adds to one address go one after another,
      // and a row may have a tenth of all ids
      uint32_t many = 1;
      bool counts = here;
      if (__popcll(in[e]) > 4) {
        const int lead = __builtin_ctzll(in[e]);
        const uint32_t row = __builtin_amdgcn_readlane(d, lead);
        const uint64_t same = __ballot(d == row) & in[e];
        if (lane == lead) many = (uint32_t)__popcll(same);
        else counts = here && d != row;
      }
      if (counts) atomicAdd(&mine[d >> 1], many << (d & 1) * 16);
    }
  });
  if (lane == 0) atomicAdd(&s_below, below);
  if (blockIdx.x == 0 && first_bad)
    for (int j = threadIdx.x; j < n; j += kSortBlock)
      if (ids[j] >= 0 && (uint32_t)ids[j] >= rows) atomicMin(first_bad, (unsigned long long)j);
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
      counted(first / 2 + p, a, b);
    }
  }
  __syncthreads();
  uint16_t* place = (uint16_t*)mine;
  if (notes <= kNotes) {
    for (int i0 = 0; i0 < notes; i0 += 64) {
      const int many = min(64, notes - i0);
      const uint32_t note = s_notes[wave][i0 + min(lane, many - 1)], d = note >> 16;
      for (uint64_t left = many < 64 ? (1ull << many) - 1 : ~0ull; left;) {       // one row at a time
        const uint32_t row = __builtin_amdgcn_readlane(d, __builtin_ctzll(left));
        const uint64_t same = __ballot(d == row) & left;
        const uint32_t to = place[row];
        __builtin_amdgcn_wave_barrier();
        if (same >> lane & 1) {
          placed(s_below, to + __popcll(same & lower), first + row, note & 0xffffu);
          place[row] = (uint16_t)(to + __popcll(same));                 // (the same from every lane)
        }
        __builtin_amdgcn_wave_barrier();
        left &= ~same;
      }
    }
    return;
  }
  each([&](int at, const uint32_t (&key)[kIdsLane]) {
    uint64_t left[kIdsLane], any = 0;
#pragma unroll
    for (int e = 0; e < kIdsLane; ++e) {
      left[e] = __ballot(key[e] - first < (uint32_t)range);
      any |= left[e];
    }
    while (any) {                                                       // one row of the 256 ids at a time
      const int lead = __builtin_ctzll(any);
      uint32_t row = 0;
#pragma unroll
      for (int e = kIdsLane - 1; e >= 0; --e)
        if (left[e] >> lead & 1) row = __builtin_amdgcn_readlane(key[e] - first, lead);
      uint64_t same[kIdsLane];
      const uint32_t from = place[row];
      uint32_t to = from, total = 0;                                    // positions rise by lane, then inside a lane
      any = 0;
#pragma unroll
      for (int e = 0; e < kIdsLane; ++e) {
        same[e] = __ballot(key[e] - first == row) & left[e];
        to += __popcll(same[e] & lower);
        total += __popcll(same[e]);
        left[e] &= ~same[e];
        any |= left[e];
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int e = 0; e < kIdsLane; ++e)
        if (same[e] >> lane & 1) placed(s_below, to++, key[e], (uint32_t)(at + e));
      if (lane == 0) place[row] = (uint16_t)(from + total);
      __builtin_amdgcn_wave_barrier();
    }
  });
}

constexpr int kFewRows = 4096;               // rows of a block, at most: counts of 16 waves take 128 KB
constexpr int64_t kFewBlocks = 256;          // ... and the least number of blocks
// The line to the radix sort, us, ids of Zipf's frequencies: 32768 21.6 for 30, 65535 43 for 33.  (Uniform 13 and 21.)
constexpr int64_t kFewNnz = 45056, kFewWork = 1 << 25;
__global__ __launch_bounds__(kSortBlock) void embed_sort_few(const int32_t* __restrict__ ids, int n, uint32_t rows, int range,
                                                             uint64_t* __restrict__ out, uint16_t* __restrict__ touched,
                                                             unsigned long long* __restrict__ first_bad) {
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  order_few(ids, n, rows, range, lds, first_bad,
            [&](uint32_t pair, uint32_t a, uint32_t b) { touched[pair] = (uint16_t)((a > 0) | (b > 0) << 8); },
            [&](uint32_t below, uint32_t place, uint32_t key, uint32_t at) {
              out[below + place] = (uint64_t)key << 32 | at;
            });
}

// ------------------------------------------------------------------ the sums

// The sorted records are cut into tiles of equal length; a lane group walks one, with kUnroll gradient rows under way,
// and writes a row when its run ends.  A run belongs to the tile it starts in, whose group follows it into the next.  Only
// long runs, those that hold the first records of two tiles, are shared: part[tile][0] is the sum of a long run
// that came from the tile before, part[tile][1] of one that starts here and goes on, and embed_join adds them up.
// kUnroll 16 took 91 us where 8 takes 61 (163840 lookups, with the clearing beside them): fewer waves fit.
constexpr int kUnroll = 8;

struct Sums {
  const uint64_t* recs;
  int64_t n, rows;
  const char* grad;
  int64_t grad_stride;
  float scale;
  float* out;
  int64_t out_stride;
  int cols, part_cols, accumulate, log2_lpr, tile;
  int64_t ntiles;
  int slices, log2_join;                     // log2 of the join's lanes per row (and of the one launch's that clear one)
  float* part;
  Fill fill;
};

__device__ __forceinline__ uint32_t key_at(const uint64_t* recs, int64_t j) { return (uint32_t)(recs[j] >> 32); }

template <int E, bool Add>
__device__ __forceinline__ void write_row(const Sums& a, uint32_t row, int c, int valid, float (&acc)[E]) {
  char* dst = (char*)(a.out + row * a.out_stride + c);
  float x[E];
  if (Add) dmt::load_elems<DMT_F32, E>(dst, valid, x);
#pragma unroll
  for (int q = 0; q < E; ++q) acc[q] = Add ? fmaf(a.scale, acc[q], x[q]) : a.scale * acc[q];
  dmt::store_elems<DMT_F32, E>(dst, valid, acc);
}

// Whole: every piece of a row is of E elements, the last one shares some with the one before (not with Add).  (A row may end at every one of the unrolled records, so what a row's end
// does is in the code kUnroll times; without the paths of ragged pieces and of Add 63.3 -> 61.3 us.)
template <int GD, bool Whole, bool Add>
__global__ __launch_bounds__(kBlock) void embed_sums(const Sums a) {
  constexpr int E = dmt::ChunkElems<GD>::value, GB = dmt::EltBytes<GD>::value;
  if (fill_block<kBlock / 64>(a.fill)) return;
  const int lane = threadIdx.x & ((1 << a.log2_lpr) - 1);
  const int64_t tile = (int64_t)(blockIdx.x / (unsigned)a.slices) * (kBlock >> a.log2_lpr) + (threadIdx.x >> a.log2_lpr);
  const int piece = (int)((blockIdx.x % (unsigned)a.slices << a.log2_lpr) + lane) * E;
  if (tile >= a.ntiles || piece >= a.cols) return;
  const int c = Whole ? piece_at<E>(piece, a.cols) : piece, valid = Whole ? E : min(E, a.cols - c);
  const int64_t j0 = tile * a.tile, j1 = min(a.n, j0 + a.tile);
  const uint32_t rows = (uint32_t)a.rows;
  // first records' keys of the tiles around this one, and the key before it
  const uint32_t prev = j0 > 0 ? key_at(a.recs, j0 - 1) : ~0u, before = tile > 0 ? key_at(a.recs, j0 - a.tile) : ~0u;
  const uint32_t first = key_at(a.recs, j0), last = key_at(a.recs, j1 - 1);
  const uint32_t next = j1 < a.n ? key_at(a.recs, j1) : ~0u;
  const uint32_t after = tile + 2 < a.ntiles ? key_at(a.recs, j1 + a.tile) : ~0u;
  const bool long_in = first == prev && (before == first || next == first);
  const bool long_out = last == next && (first == last || after == last);
  const uint32_t skip = long_in ? ~0u : prev;              // a short run that came from the tile before is done there
  uint32_t cur = rows;
  float acc[E];
  auto flush = [&]() {
    if (cur >= rows || cur == skip) return;
    const bool part = cur == prev || (cur == next && long_out);
    if (Add && !part) {
      write_row<E, true>(a, cur, c, valid, acc);
      return;
    }
    float* dst = part ? a.part + (tile * 2 + (cur != prev)) * a.part_cols + c : a.out + cur * a.out_stride + c;
    const float f = part ? 1.f : a.scale;
#pragma unroll
    for (int q = 0; q < E; ++q) acc[q] *= f;
    dmt::store_elems<DMT_F32, E>((char*)dst, part ? E : valid, acc);
  };
  // records j .. end - 1; past the tile's end only while they are the last run's
  auto walk = [&](int64_t j, int64_t end, bool beyond) {
    for (; j < end; j += kUnroll) {
      uint64_t rec[kUnroll];
      dmt::Raw<GD, E> g[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) rec[u] = a.recs[min(j + u, end - 1)];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const uint32_t key = (uint32_t)(rec[u] >> 32);
        if (beyond ? key == cur : key != skip && key < rows)
          g[u] = dmt::load_raw<GD, E>(a.grad + ((int64_t)(uint32_t)rec[u] * a.grad_stride + c) * GB, valid);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (j + u >= end) break;
        const uint32_t key = (uint32_t)(rec[u] >> 32);
        if (key != cur) {
          if (beyond) return;
          flush();
          cur = key;
#pragma unroll
          for (int q = 0; q < E; ++q) acc[q] = 0.f;
        }
        if (cur == skip || cur >= rows) continue;
        float x[E];
        dmt::unpack<GD, E>(g[u], x);
#pragma unroll
        for (int q = 0; q < E; ++q) acc[q] += x[q];
      }
    }
  };
  walk(j0, j1, false);
  if (cur == next && cur != skip && cur < rows && !long_out) walk(j1, min(a.n, j1 + a.tile), true);
  flush();
}

// Sums over the block's groups of 2^log2 lanes, into group 0: within the waves, then the waves' in order.  lds [B][E].  (Group by group,
// the 512 groups of two lanes that columns of 16 leave took 20 us a row.)
template <int B, int E> __device__ __forceinline__ void join_groups(float (&acc)[E], int log2, float* lds) {
  for (int o = 1 << log2; o < 64; o <<= 1)
#pragma unroll
    for (int q = 0; q < E; ++q) acc[q] += __shfl_xor(acc[q], o);
  const int lane = threadIdx.x & 63;
  const bool first = lane < 1 << log2;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < E; ++q)
    if (first) lds[(((threadIdx.x >> 6) << log2) + lane) * E + q] = acc[q];
  __syncthreads();
  if ((int)threadIdx.x < 1 << log2)
    for (int w = 1; w < B / 64; ++w)
#pragma unroll
      for (int q = 0; q < E; ++q) acc[q] += lds[((w << log2) + lane) * E + q];
}

// Rows of long runs: their partial sums, in the tiles' order.  A block looks at kJoinTiles tiles; each
// lane group takes the runs that start in one of them in turn, and the whole block those of many tiles.
constexpr int kJoinTiles = 64, kJoinLong = 16, kJoinBlock = 1024;

// How many tiles from t + 1 on start with row v, tile t + 1 among them.  By a whole wave: 64 tiles, then every 64th ... of
// them at a time, so a run of thousands of tiles takes a few reads after one another (bisection took twenty).
__device__ __forceinline__ int64_t tiles_of_run(const Sums& a, int64_t t, uint32_t v) {
  const int lane = threadIdx.x & 63;
  int64_t good = t + 1, stride = 1;          // tile `good` starts with v
  for (;;) {                                 // wider steps while all 64 do
    const int64_t at = good + (lane + 1) * stride;
    const bool is = at < a.ntiles && key_at(a.recs, at * a.tile) == v;
    const int many = __builtin_popcountll(__ballot(is));     // (a prefix of the lanes: the records are sorted)
    good += many * stride;
    if (many == 64) {
      stride *= 64;
      continue;
    }
    if (stride == 1) return good - t;
    stride /= 64;
  }
}

template <bool Add>
__global__ __launch_bounds__(kJoinBlock) void embed_join(const Sums a) {
  constexpr int E = 4;
  __shared__ int s_tile[kJoinTiles], s_len[kJoinTiles];
  __shared__ uint32_t s_row[kJoinTiles];
  __shared__ float s_sum[kJoinBlock * E];
  if (fill_block<kJoinBlock / 64>(a.fill)) return;
  const int64_t t0 = (int64_t)blockIdx.x * kJoinTiles;
  bool owns = false;
  uint32_t row = 0;
  if (t0 + (threadIdx.x & 63) + 1 < a.ntiles) {             // (every wave looks at all of the tiles)
    const int64_t t = t0 + (threadIdx.x & 63), b = t * a.tile, e = b + a.tile;
    const uint32_t v = key_at(a.recs, e - 1), next = key_at(a.recs, e), first = key_at(a.recs, b);
    const uint32_t prev = b > 0 ? key_at(a.recs, b - 1) : ~0u, after = t + 2 < a.ntiles ? key_at(a.recs, e + a.tile) : ~0u;
    owns = (int64_t)v < a.rows && next == v && (first != v || prev != v) && (first == v || after == v);
    row = v;
  }
  const uint64_t starts = __ballot(owns);
  const int count = __builtin_popcountll(starts);
  if (count == 0) return;
  uint64_t left = starts;
  for (int i = 0; i < count; ++i, left &= left - 1) {
    if (i % (kJoinBlock / 64) != threadIdx.x >> 6) continue;
    const int at = __builtin_ctzll(left);
    const uint32_t v = __builtin_amdgcn_readlane(row, at);
    const int64_t many = tiles_of_run(a, t0 + at, v);
    s_tile[i] = at;
    s_row[i] = v;
    s_len[i] = (int)many;
  }
  __syncthreads();
  const int lane = threadIdx.x & ((1 << a.log2_join) - 1);
  const int group = threadIdx.x >> a.log2_join, groups = kJoinBlock >> a.log2_join;
  auto heads = [&](int64_t t, int from, int to, int c, float (&acc)[E]) {
    const float* p = a.part + t * 2 * a.part_cols + c;
    for (int i = from; i < to; i += 8) {                    // (past the end: the last one again, not added)
      float4 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = *(const float4*)(p + (int64_t)min(i + u, to - 1) * 2 * a.part_cols);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i + u < to) acc[0] += x[u].x, acc[1] += x[u].y, acc[2] += x[u].z, acc[3] += x[u].w;
    }
  };
  auto tail = [&](int64_t t, int c, float (&acc)[E]) {
    const float4 x = *(const float4*)(a.part + (t * 2 + 1) * a.part_cols + c);
    acc[0] = x.x, acc[1] = x.y, acc[2] = x.z, acc[3] = x.w;
  };
  for (int i = group; i < count; i += groups) {
    if (s_len[i] > kJoinLong) continue;
    const int64_t t = t0 + s_tile[i];
    const uint32_t v = s_row[i];
    for (int c = lane * E; c < a.cols; c += E << a.log2_join) {
      float acc[E];
      tail(t, c, acc);
      heads(t, 1, s_len[i] + 1, c, acc);
      write_row<E, Add>(a, v, c, min(E, a.cols - c), acc);
    }
  }
  for (int i = 0; i < count; ++i) {
    if (s_len[i] <= kJoinLong) continue;
    const int64_t t = t0 + s_tile[i];
    const uint32_t v = s_row[i];
    const int per = (s_len[i] + groups - 1) / groups, from = 1 + group * per, to = min(s_len[i] + 1, from + per);
    for (int c0 = 0; c0 < a.cols; c0 += E << a.log2_join) {
      const int c = c0 + lane * E;
      float acc[E] = {0.f, 0.f, 0.f, 0.f};
      if (group == 0 && c < a.cols) tail(t, c, acc);
      if (c < a.cols) heads(t, from, to, c, acc);
      join_groups<kJoinBlock>(acc, a.log2_join, s_sum);
      if (group == 0 && c < a.cols) write_row<E, Add>(a, v, c, min(E, a.cols - c), acc);
    }
  }
}

// ------------------------------------------------------------------ very few lookups: the whole backward in one launch

// The sort of embed_sort_few with the block's positions left in LDS, then the block sums (or clears) its rows at once.  Lane groups
// take a row each; rows of more than kFusedLong lookups are shared out over all the groups and joined in LDS.
constexpr int kFusedRows = 2048, kFusedLong = 32, kFusedUnroll = 8;
constexpr int64_t kFusedNnz = 4096, kFusedWork = 1 << 23;
template <int E> constexpr int fused_lds(int range) {
  return range * kSortWaves * 2 + (int)kFusedNnz * 2 + (int)kFusedNnz / kFusedLong * 2 + kSortBlock * E * 4;
}
template <int GD, bool Whole, bool Add>
__global__ __launch_bounds__(kSortBlock) void embed_bwd_few(const int32_t* __restrict__ ids, int n, int range,
                                                            unsigned long long* __restrict__ first_bad, const Sums a) {
  constexpr int E = dmt::ChunkElems<GD>::value, GB = dmt::EltBytes<GD>::value;
  extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
  __shared__ uint32_t s_many;
  uint16_t* list = (uint16_t*)(lds + range / 2 * kSortWaves);           // [kFusedNnz] positions in order of their rows
  uint16_t* many = list + kFusedNnz;                                    // rows of many lookups
  float* sums = (float*)(many + kFusedNnz / kFusedLong);
  if (threadIdx.x == 0) s_many = 0;
  const uint32_t rows = (uint32_t)a.rows, first = blockIdx.x * (uint32_t)range;
  order_few(ids, n, rows, range, lds, first_bad, [&](uint32_t, uint32_t, uint32_t) {},
            [&](uint32_t, uint32_t place, uint32_t, uint32_t at) { list[place] = (uint16_t)at; });
  __syncthreads();
  const uint16_t* ends = (const uint16_t*)lds + (kSortWaves - 1) * range;
  const int lane = threadIdx.x & ((1 << a.log2_lpr) - 1), group = threadIdx.x >> a.log2_lpr;
  const int groups = kSortBlock >> a.log2_lpr;
  auto sum = [&](int from, int to, int c, int valid, float (&acc)[E]) {
    for (int i = from; i < to; i += kFusedUnroll) {
      dmt::Raw<GD, E> g[kFusedUnroll];
#pragma unroll
      for (int u = 0; u < kFusedUnroll; ++u)
        if (i + u < to) g[u] = dmt::load_raw<GD, E>(a.grad + ((int64_t)list[i + u] * a.grad_stride + c) * GB, valid);
#pragma unroll
      for (int u = 0; u < kFusedUnroll; ++u) {
        if (i + u >= to) break;
        float x[E];
        dmt::unpack<GD, E>(g[u], x);
#pragma unroll
        for (int q = 0; q < E; ++q) acc[q] += x[q];
      }
    }
  };
  // (plain stores, where fill_block's go past the caches: 18.2 us for 22.4 with one id and 87 MB to
  // clear, 30 for 32 with 50 ids and 107 MB, 72 for 74 with 193 and 306 MB; 43.5 for 41.2 with
  // 4096 and 131 MB, whose gradients the caches then hold less of)
  if (!Add)
    for (int r = threadIdx.x >> a.log2_join; r < range && first + r < rows; r += kSortBlock >> a.log2_join) {
      if (ends[r] != (r > 0 ? ends[r - 1] : 0)) continue;
      for (int c = (threadIdx.x & ((1 << a.log2_join) - 1)) * 4; c < a.cols; c += 4 << a.log2_join) {
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        dmt::store_elems<DMT_F32, 4>((char*)(a.out + (first + r) * a.out_stride + piece_at<4>(c, a.cols)), a.cols, zero);
      }
    }
  for (int r = group; r < range && first + r < rows; r += groups) {
    const int from = r > 0 ? ends[r - 1] : 0, to = ends[r];
    if (to - from > kFusedLong) {
      if (lane == 0) many[atomicAdd(&s_many, 1u)] = (uint16_t)r;        // (their order changes no sum)
      continue;
    }
    if (to == from) continue;
    for (int piece = lane * E; piece < a.cols; piece += E << a.log2_lpr) {
      float acc[E];
#pragma unroll
      for (int q = 0; q < E; ++q) acc[q] = 0.f;
      const int c = Whole ? piece_at<E>(piece, a.cols) : piece, valid = Whole ? E : min(E, a.cols - c);
      sum(from, to, c, valid, acc);
      write_row<E, Add>(a, first + r, c, valid, acc);
    }
  }
  __syncthreads();
  const int count = (int)s_many;
  for (int i = 0; i < count; ++i) {
    const int r = many[i], from = r > 0 ? ends[r - 1] : 0, to = ends[r];
    const int per = (to - from + groups - 1) / groups, mine = min(to, from + group * per), end = min(to, mine + per);
    for (int c0 = 0; c0 < a.cols; c0 += E << a.log2_lpr) {
      const int piece = c0 + lane * E, c = Whole ? piece_at<E>(piece, a.cols) : piece, valid = Whole ? E : min(E, a.cols - c);
      float acc[E];
#pragma unroll
      for (int q = 0; q < E; ++q) acc[q] = 0.f;
      if (piece < a.cols) sum(mine, end, c, valid, acc);
      join_groups<kSortBlock>(acc, a.log2_lpr, sums);
      if (group == 0 && piece < a.cols) write_row<E, Add>(a, first + r, c, valid, acc);
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
  bool fused, few;                           // one launch does everything, sorts
  int range;                                 // rows of a block of it
  int items, passes, bits;
  int tile, part_cols;
  size_t bytes;
};

// Records a lane group walks: as many as leave a wave's worth of groups for every place on the chip, at least kLeastTile (of 8: as fast,
// and the join 45 us for 31).
constexpr int64_t kFillLanes = 256 * 512;
constexpr int kLeastTile = 16, kMostTile = 32;
int tile_of(int64_t n, int64_t cols) {
  int tile = kMostTile;
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
  const int64_t narrow = std::max<int64_t>(kFewBlocks, (rows + kFusedRows - 1) / kFusedRows);
  w.fused = n <= kFusedNnz && n * narrow <= kFusedWork;
  if (w.fused) w.range = (int)dmt_align_up((size_t)((rows + narrow - 1) / narrow), 32);
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
      std::max((n + kMostTile - 1) / kMostTile, std::min((n + kLeastTile - 1) / kLeastTile, 2 * kFillLanes >> log2_lanes(cols, 8)));
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
  auto go = [&](auto kernel) {
    dmt_launches(((n << l) + kBlock - 1) / kBlock, kBlock, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, first, (const char*)table, rows, (int)cols, ts, ids, n, scale,
                         (char*)out, os, (unsigned long long*)bad, l);
    });
  };
  if (od == DMT_F32) go(embed_fwd_kernel<TD, DMT_F32>);
  else if (od == DMT_F16) go(embed_fwd_kernel<TD, DMT_F16>);
  else go(embed_fwd_kernel<TD, DMT_BF16>);
}

// The sums' share of the clearing, percent; the join has the rest.  (With a tenth in each of the sort's last launches too
// the whole call took as long: what they hide they cost.)
constexpr int kSumsShare = 55;

// The table's rows in wave units, handed out to the two launches.
struct Clearing {
  Fill fill = {};
  int64_t units = 0, done = 0;
  Clearing(const Ws& w, const Sums& a) {
    fill.touched = w.touched, fill.out = a.out, fill.out_stride = a.out_stride, fill.rows = a.rows, fill.cols = a.cols;
    fill.log2_lanes = log2_lanes(a.cols, 4);
    const int64_t per = std::min<int64_t>(64, std::min(kFillBytes / (4 * (int64_t)a.cols), a.rows / kFillWaves));
    fill.rows_per_wave = (int)std::max<int64_t>(64 >> fill.log2_lanes, per);
    if (!a.accumulate) units = (a.rows + fill.rows_per_wave - 1) / fill.rows_per_wave;
  }
  // A launch of `own` blocks of `waves` waves takes `percent` of all the units: its grid, with `f` for its kernel.
  dim3 share(unsigned own, int waves, int percent, Fill& f) {
    f = fill;
    f.own_blocks = own;
    f.first = done;
    const int64_t want = percent >= 100 ? units - done : std::min(units - done, units * percent / 100);
    const int64_t blocks = (want + waves - 1) / waves;
    done = std::min(units, done + blocks * waves);
    return dim3((unsigned)(own + blocks));
  }
};

template <bool First>
void launch_pass(const Ws& w, const int32_t* ids, const uint64_t* in, uint64_t* out, int64_t n, int64_t rows,
                 int shift, int64_t* bad, hipStream_t s) {
  const int nd = 1 << w.bits;
  hipLaunchKernelGGL(embed_digits<First>, dim3((unsigned)w.nblk), dim3(kSortBlock), 0, s, ids, in, n, (uint32_t)rows,
                     w.items, shift, w.bits, w.counts, (uint32_t*)w.touched, w.touched_words, (unsigned long long*)bad);
  hipLaunchKernelGGL(embed_digit_starts, dim3((nd + 63) / 64), dim3(64 * kStartsSegs), 0, s, w.counts, w.nblk, nd, w.totals);
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

// run(whole pieces, add to what is there), each a std::true_type or std::false_type.
template <typename Run> void variants(bool whole, bool add, Run run) {
  if (whole) add ? run(std::true_type(), std::true_type()) : run(std::true_type(), std::false_type());
  else add ? run(std::false_type(), std::true_type()) : run(std::false_type(), std::false_type());
}

template <int GD>
void launch_fused(const Ws& w, Sums a, const int32_t* ids, int64_t* bad, hipStream_t s) {
  constexpr int E = dmt::ChunkElems<GD>::value;
  a.log2_lpr = log2_lanes(a.cols, E);
  a.log2_join = log2_lanes(a.cols, 4);
  variants(a.cols % E == 0 || (a.cols > E && !a.accumulate), a.accumulate, [&](auto whole, auto add) {
    auto kernel = embed_bwd_few<GD, decltype(whole)::value, decltype(add)::value>;
    static DmtPerDevice done;
    dmt_allow_lds(done, (const void*)kernel, fused_lds<E>(kFusedRows));
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.rows + w.range - 1) / w.range)), dim3(kSortBlock), fused_lds<E>(w.range), s,
                       ids, (int)a.n, w.range, (unsigned long long*)bad, a);
  });
}

template <int GD>
void launch_sums(Sums a, Clearing& clear, hipStream_t s) {
  constexpr int E = dmt::ChunkElems<GD>::value;
  a.log2_lpr = log2_lanes(a.cols, E);
  a.log2_join = log2_lanes(a.cols, 4);
  a.slices = (a.cols + (E << a.log2_lpr) - 1) / (E << a.log2_lpr);
  const int groups = kBlock >> a.log2_lpr;
  const bool join = a.ntiles > 1;                           // (else no run is long)
  const dim3 sums = clear.share((unsigned)((a.ntiles + groups - 1) / groups * a.slices), kBlock / 64, join ? kSumsShare : 100, a.fill);
  if (sums.x > 0)
    variants(a.cols % E == 0 || (a.cols > E && !a.accumulate), a.accumulate, [&](auto whole, auto add) {
      hipLaunchKernelGGL((embed_sums<GD, decltype(whole)::value, decltype(add)::value>), sums, dim3(kBlock), 0, s, a);
    });
  if (!join) return;
  const dim3 grid = clear.share((unsigned)((a.ntiles + kJoinTiles - 1) / kJoinTiles), kJoinBlock / 64, 100, a.fill);
  if (a.accumulate) hipLaunchKernelGGL(embed_join<true>, grid, dim3(kJoinBlock), 0, s, a);
  else hipLaunchKernelGGL(embed_join<false>, grid, dim3(kJoinBlock), 0, s, a);
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
  Sums a = {};
  a.n = n, a.rows = rows, a.grad = (const char*)grad, a.grad_stride = grad_stride, a.scale = scale;
  a.out = grad_table, a.out_stride = grad_table_stride, a.cols = (int)cols, a.accumulate = accumulate != 0;
  a.tile = w.tile, a.ntiles = w.ntiles, a.part = w.part, a.part_cols = w.part_cols;
  if (w.fused) {
    if (grad_dtype == DMT_F32) launch_fused<DMT_F32>(w, a, ids, first_bad, s);
    else if (grad_dtype == DMT_F16) launch_fused<DMT_F16>(w, a, ids, first_bad, s);
    else launch_fused<DMT_BF16>(w, a, ids, first_bad, s);
    return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
  }
  Clearing clear(w, a);
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
  a.recs = in;
  if (grad_dtype == DMT_F32) launch_sums<DMT_F32>(a, clear, s);
  else if (grad_dtype == DMT_F16) launch_sums<DMT_F16>(a, clear, s);
  else launch_sums<DMT_BF16>(a, clear, s);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
