// dmt_expert_sort, dmt_expert_gather, dmt_expert_combine, dmt_expert_combine_bwd: rows sent to experts and back.
//
// The order is a counting sort with the expert as the only digit: counts of a tile of assignments, then places.  A tile is a
// block's; there are at most 64 tiles, so that a block finds the counts before it by adding up to 64 rows of counts itself and no
// launch of its own scans them.  Inside a tile every wave has a stretch of its own and ranks 64 assignments at a time: the
// lanes that name the same expert are found with one ballot a bit of the expert's number.  Places depend on the assignments'
// order alone.  One tile needs one launch.  65536 x 2 assignments to 64 experts 4.5 + 8.9 us, 131072 x 8 to 256 7.7 + 25.6, 64 x 2 4.2: chains of
// latencies, of the counts before a tile (16 rows of them requested together: 17 us for 9) and of four times 64 ranks.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64, kTiles = 64, kBlock = 256;

struct Sort {
  const int32_t* experts;
  int64_t m, rows;              // assignments, rows of the order
  int64_t stretch;              // assignments a wave has, a multiple of 64
  int E, bits, tiles;
  int64_t capacity;
  int32_t *slot, *source, *offsets, *counts, *part;      // part [tiles][E]
  unsigned long long* first_bad;
};

// The wave's stretch of the tile's assignments.
__device__ __forceinline__ void stretch_of(const Sort& a, int64_t& from, int64_t& to) {
  from = min(a.m, ((int64_t)blockIdx.x * kSortWaves + (threadIdx.x >> 6)) * a.stretch);
  to = min(a.m, from + a.stretch);
}

// Four times 64 assignments from i0 on, a lane's requested together (-1 behind the stretch).
constexpr int kBatch = 4;
__device__ __forceinline__ void load_batch(const Sort& a, int64_t i0, int64_t to, int (&e)[kBatch]) {
#pragma unroll
  for (int b = 0; b < kBatch; ++b) {
    const int64_t i = i0 + b * 64 + (threadIdx.x & 63);
    e[b] = i < to ? a.experts[i] : -1;
  }
}

// Counts of the wave's assignments by expert, added to count[E] (LDS, zero).
__device__ __forceinline__ void count_stretch(const Sort& a, int* count) {
  int64_t from, to;
  stretch_of(a, from, to);
  for (int64_t i0 = from; i0 < to; i0 += kBatch * 64) {
    int e[kBatch];
    load_batch(a, i0, to, e);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if ((uint32_t)e[b] < (uint32_t)a.E) atomicAdd(&count[e[b]], 1);
      else if (e[b] >= 0 && a.first_bad) atomicMin(a.first_bad, (unsigned long long)(i0 + b * 64 + (threadIdx.x & 63)));
    }
  }
}

__global__ __launch_bounds__(kSortBlock) void expert_count(const Sort a) {
  extern __shared__ int lds[];
  for (int e = threadIdx.x; e < a.E; e += kSortBlock) lds[e] = 0;
  __syncthreads();
  count_stretch(a, lds);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kSortBlock) a.part[(int64_t)blockIdx.x * a.E + e] = lds[e];
}

// LDS: place [waves][E], total [E], begin [E], and a word a wave.
__global__ __launch_bounds__(kSortBlock) void expert_place(const Sort a) {
  extern __shared__ int lds[];
  const int E = a.E, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int *place = lds, *total = place + kSortWaves * E, *begin = total + E, *sums = begin + E;
  for (int i = threadIdx.x; i < kSortWaves * E; i += kSortBlock) place[i] = 0;
  __syncthreads();
  count_stretch(a, place + wave * E);
  __syncthreads();
  // an expert a thread (E <= kSortBlock): its assignments in all, those of the tiles before, those of the waves before
  const int e = threadIdx.x;
  int all = 0, before = 0;
  if (e < E) {
    if (a.tiles > 1)
      for (int t0 = 0; t0 < a.tiles; t0 += 16) {           // 16 rows of counts requested together
        int c[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) c[t] = a.part[(int64_t)min(t0 + t, a.tiles - 1) * E + e];
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          all += t0 + t < a.tiles ? c[t] : 0;
          before += t0 + t < (int)blockIdx.x ? c[t] : 0;
        }
      }
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = place[w * E + e];
      place[w * E + e] = before;
      before += c;
      if (a.tiles == 1) all += c;
    }
  }
  uint32_t sum;
  const int at = (int)dmt::block_exclusive_scan<kSortWaves>((uint32_t)all, (uint32_t*)sums, sum);
  if (e < E) {
    total[e] = all;
    begin[e] = a.capacity ? (int)(e * a.capacity) : at;
    if (blockIdx.x == 0) {
      if (a.offsets) a.offsets[e] = begin[e];
      if (a.counts) a.counts[e] = all;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.offsets) a.offsets[E] = a.capacity ? (int)(E * a.capacity) : (int)sum;
  __syncthreads();
  int64_t from, to;
  stretch_of(a, from, to);
  for (int64_t b0 = from; b0 < to; b0 += kBatch * 64) {
    int e4[kBatch];
    load_batch(a, b0, to, e4);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int64_t i = b0 + b * 64 + lane;
      const int x = e4[b];
      const bool named = (uint32_t)x < (uint32_t)E;
      uint64_t same = __ballot(named);
      for (int p = 0; p < a.bits; ++p) {
        const uint64_t set = __ballot((x >> p) & 1);
        same &= (x >> p) & 1 ? set : ~set;
      }
      const int rank = __popcll(same & ((1ull << lane) - 1));
      int base = 0;
      if (named && rank == 0) base = atomicAdd(&place[wave * E + x], (int)__popcll(same));
      base = __shfl(base, named ? __ffsll((unsigned long long)same) - 1 : lane);
      if (i < to) {
        int64_t row = -1;
        if (named) {
          const int64_t r = (int64_t)base + rank;
          if (!a.capacity || r < a.capacity) row = begin[x] + r;
        }
        a.slot[i] = (int)row;
        if (row >= 0) a.source[row] = (int)i;
      }
    }
  }
  // rows without an assignment: behind the last one (of an expert)
  for (int64_t r = (int64_t)blockIdx.x * kSortBlock + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * kSortBlock) {
    if (a.capacity) {
      const uint32_t x = (uint32_t)r / (uint32_t)a.capacity;
      if ((int)((uint32_t)r - x * (uint32_t)a.capacity) >= total[x]) a.source[r] = -1;
    } else if (r >= (int64_t)sum) {
      a.source[r] = -1;
    }
  }
}

// ------------------------------------------------------------------ rows there and back
//
// A group of G lanes has a token, 16 bytes a lane at a time of what is moved (8 elements of what is computed), and takes its assignments
// four at a time, so that as many rows are under way.  All of it is bound by memory: rows are read once, and written once.  65536 tokens of 512
// bfloat16 to two of 64 experts 46 us, 5.1 TB/s (by rows of the order, a token's row read twice: 67); back from four, 32768 x 1024, 65 us, 5.1 TB/s;
// gradients of 32768 x 512 in float32 61 + 37 us.

constexpr int kAtOnce = 4;

struct Move {
  const char *x, *z;
  char* out;
  int64_t x_stride, z_stride, out_stride, n, rows;
  const int32_t *slot, *source;
  const float* weights;
  float* dweights;
  unsigned token_blocks;        // blocks that have tokens; those behind them clear rows
  int cols, k;
};

// A lane's piece of a row, E elements from c on: the last piece of a row of no whole number of them starts earlier, so that it ends with
// the row (its first `skip` elements are the piece before's too).  Rows shorter than a piece have `valid` elements.
template <int E> struct Place {
  int c, skip, valid;
  __device__ __forceinline__ Place(int at, int cols) {
    c = max(0, min(at, cols - E));
    skip = at - c;
    valid = min(E, cols);
  }
};

// The E elements (16 bytes) of type-less words at p.
template <int EB> __device__ __forceinline__ void store_raw(char* p, int valid, const dmt::Raw<EB == 4 ? DMT_F32 : DMT_F16, 16 / EB>& v) {
  constexpr int E = 16 / EB;
  if (valid >= E) {
    const dmt::dmt_u32x4 w = {v.w[0], v.w[1], v.w[2], v.w[3]};
    *(DMT_GLOBAL typename dmt::Piece<EB>::v4*)p = w;
  } else {
#pragma unroll
    for (int i = 0; i < E - 1; ++i)
      if (i < valid) {
        if constexpr (EB == 4) *(DMT_GLOBAL uint32_t*)(p + i * 4) = v.w[i];
        else *(DMT_GLOBAL uint16_t*)(p + i * 2) = (uint16_t)(v.w[i / 2] >> i % 2 * 16);
      }
  }
}

// Zeros into those of the wave's 64 rows that have no assignment.
template <int EB> __device__ __forceinline__ void clear_rows(const Move& a, int64_t block) {
  constexpr int E = 16 / EB;
  const int lane = threadIdx.x & 63;
  const int64_t r0 = (block * (kBlock / 64) + (threadIdx.x >> 6)) * 64, r = r0 + lane;
  uint64_t empty = __ballot(r < a.rows && a.source[min(r, a.rows - 1)] < 0);
  const dmt::Raw<EB == 4 ? DMT_F32 : DMT_F16, E> zero = {};
  for (; empty; empty &= empty - 1) {
    char* to = a.out + (r0 + __builtin_ctzll(empty)) * a.out_stride * EB;
    for (int c = lane * E; c < a.cols; c += 64 * E) {
      const Place<E> at(c, a.cols);
      store_raw<EB>(to + (int64_t)at.c * EB, at.valid, zero);
    }
  }
}

// Token's slots j0 .. j0 + kAtOnce - 1 (-1: none).
__device__ __forceinline__ void slots_of(const Move& a, int64_t i, int j0, int (&s)[kAtOnce]) {
#pragma unroll
  for (int q = 0; q < kAtOnce; ++q) {
    const int v = j0 + q < a.k ? a.slot[i * a.k + j0 + q] : -1;
    s[q] = (int64_t)v < a.rows ? v : -1;
  }
}
__device__ __forceinline__ void weights_of(const Move& a, int64_t i, int j0, float (&w)[kAtOnce]) {
#pragma unroll
  for (int q = 0; q < kAtOnce; ++q) w[q] = a.weights && j0 + q < a.k ? a.weights[i * a.k + j0 + q] : 1.f;
}

template <int EB, int G> __global__ __launch_bounds__(kBlock) void expert_gather(const Move a, unsigned first) {
  constexpr int DT = EB == 4 ? DMT_F32 : DMT_F16, E = 16 / EB;
  const unsigned block = first + blockIdx.x;
  if (block >= a.token_blocks) return clear_rows<EB>(a, block - a.token_blocks);
  const int64_t i = (int64_t)block * (kBlock / G) + threadIdx.x / G;
  if (i >= a.n) return;
  for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
    int s[kAtOnce];
    slots_of(a, i, j0, s);
    for (int c = (threadIdx.x % G) * E; c < a.cols; c += G * E) {
      const Place<E> at(c, a.cols);
      const auto v = dmt::load_raw<DT, E>(a.x + (i * a.x_stride + at.c) * EB, at.valid);
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q)
        if (s[q] >= 0) store_raw<EB>(a.out + (s[q] * a.out_stride + at.c) * EB, at.valid, v);
    }
  }
}

template <int DT, int OD, int G> __global__ __launch_bounds__(kBlock) void expert_combine(const Move a, unsigned first) {
  constexpr int EB = dmt::EltBytes<DT>::value, OB = dmt::EltBytes<OD>::value, E = 8;
  const int64_t i = (int64_t)(first + blockIdx.x) * (kBlock / G) + threadIdx.x / G;
  if (i >= a.n) return;
  int s[kAtOnce];
  float w[kAtOnce];
  slots_of(a, i, 0, s);
  weights_of(a, i, 0, w);
  for (int c = (threadIdx.x % G) * E; c < a.cols; c += G * E) {
    const Place<E> at(c, a.cols);
    float sum[E] = {};
    for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
      if (a.k > kAtOnce) {
        slots_of(a, i, j0, s);
        weights_of(a, i, j0, w);
      }
      dmt::Raw<DT, E> z[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        z[q] = {};
        if (s[q] >= 0) z[q] = dmt::load_raw<DT, E>(a.z + (s[q] * a.z_stride + at.c) * EB, at.valid);
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        float v[E];
        dmt::unpack<DT, E>(z[q], v);
        const float by = s[q] >= 0 ? w[q] : 0.f;
#pragma unroll
        for (int p = 0; p < E; ++p) sum[p] = fmaf(by, v[p], sum[p]);
      }
    }
    dmt::store_elems<OD, E>(a.out + (i * a.out_stride + at.c) * OB, at.valid, sum);
  }
}

// x is dy here, out dz.
template <int DT, int GD, int G> __global__ __launch_bounds__(kBlock) void expert_combine_bwd(const Move a, unsigned first) {
  constexpr int EB = dmt::EltBytes<DT>::value, GB = dmt::EltBytes<GD>::value, E = 8;
  const unsigned block = first + blockIdx.x;
  if (block >= a.token_blocks) return clear_rows<GB>(a, block - a.token_blocks);
  const int64_t i = (int64_t)block * (kBlock / G) + threadIdx.x / G;
  if (i >= a.n) return;
  for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
    int s[kAtOnce];
    float w[kAtOnce], dot[kAtOnce] = {};
    slots_of(a, i, j0, s);
    weights_of(a, i, j0, w);
    for (int c = (threadIdx.x % G) * E; c < a.cols; c += G * E) {
      const Place<E> at(c, a.cols);
      float g[E];
      dmt::load_elems<GD, E>(a.x + (i * a.x_stride + at.c) * GB, at.valid, g);
      dmt::Raw<DT, E> z[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        z[q] = {};
        if (a.dweights && s[q] >= 0) z[q] = dmt::load_raw<DT, E>(a.z + (s[q] * a.z_stride + at.c) * EB, at.valid);
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        if (s[q] < 0) continue;
        float v[E], d[E];
        dmt::unpack<DT, E>(z[q], v);
#pragma unroll
        for (int p = 0; p < E; ++p) {
          dot[q] = p >= at.skip ? fmaf(g[p], v[p], dot[q]) : dot[q];
          d[p] = w[q] * g[p];
        }
        if (a.out) dmt::store_elems<GD, E>(a.out + (s[q] * a.out_stride + at.c) * GB, at.valid, d);
      }
    }
    if (a.dweights) {
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        dot[q] = dmt::group_sum<G>(dot[q]);
        if (threadIdx.x % G == 0 && j0 + q < a.k) a.dweights[i * a.k + j0 + q] = dot[q];
      }
    }
  }
}

template <int V> struct Int { static constexpr int value = V; };
template <typename Go> void by_type(int32_t t, Go go) {
  if (t == DMT_F32) go(Int<DMT_F32>());
  else if (t == DMT_F16) go(Int<DMT_F16>());
  else go(Int<DMT_BF16>());
}

constexpr int64_t kMost = (1ll << 31) - 1;
bool few(int64_t n, int64_t k) { return k <= kMost && n <= kMost / std::max<int64_t>(k, 1); }
int64_t stretch(int64_t m) {                       // of a wave: at most kTiles tiles of kSortWaves stretches
  const int64_t per = (m + kTiles * kSortWaves - 1) / (kTiles * kSortWaves);
  return std::max<int64_t>(256, (per + 63) / 64 * 64);
}
int64_t tiles(int64_t m) { return std::max<int64_t>(1, (m + kSortWaves * stretch(m) - 1) / (kSortWaves * stretch(m))); }

}  // namespace

extern "C" size_t dmt_expert_sort_workspace_bytes(int64_t n, int64_t k, int64_t num_experts) {
  if (n < 0 || k < 1 || num_experts < 1 || num_experts > DMT_EXPERT_MAX || !few(n, k)) return 0;
  return sizeof(int32_t) * (size_t)(tiles(n * k) > 1 ? tiles(n * k) * num_experts : 0);
}

extern "C" dmt_status dmt_expert_sort(const int32_t* experts, int64_t n, int64_t k, int64_t num_experts,
                                      int64_t capacity, int32_t* slot, int32_t* source, int32_t* offsets,
                                      int32_t* counts, int64_t* first_bad, void* workspace, size_t workspace_bytes,
                                      void* stream) {
  if (n < 0 || k < 1 || num_experts < 1 || capacity < 0) return DMT_EINVAL;
  if (n > 0 && (!dmt_is_at(experts, 4) || !dmt_is_at(slot, 4))) return DMT_EINVAL;
  if (!dmt_may_be_at(offsets, 4) || !dmt_may_be_at(counts, 4) || !dmt_may_be_at(first_bad, 8)) return DMT_EINVAL;
  if (num_experts > DMT_EXPERT_MAX || !few(n, k) || capacity > kMost / num_experts) return DMT_ENOTSUP;
  Sort a = {};
  a.m = n * k, a.rows = capacity ? num_experts * capacity : a.m;
  if (a.rows > 0 && !dmt_is_at(source, 4)) return DMT_EINVAL;
  a.tiles = (int)tiles(a.m), a.stretch = stretch(a.m);
  const size_t need = dmt_expert_sort_workspace_bytes(n, k, num_experts);
  if (need > 0 && !dmt_is_at(workspace, 256)) return DMT_EINVAL;
  if (workspace_bytes < need) return DMT_ENOMEM;
  a.experts = experts, a.E = (int)num_experts, a.capacity = capacity;
  while ((1 << a.bits) < a.E) ++a.bits;
  a.slot = slot, a.source = source, a.offsets = offsets, a.counts = counts, a.part = (int32_t*)workspace;
  a.first_bad = (unsigned long long*)first_bad;
  hipStream_t s = (hipStream_t)stream;
  const int lds = (int)sizeof(int) * ((kSortWaves + 2) * a.E + kSortWaves + 1);
  static DmtPerDevice allowed;
  dmt_allow_lds(allowed, (const void*)expert_place, (int)sizeof(int) * ((kSortWaves + 2) * DMT_EXPERT_MAX + kSortWaves + 1));
  if (a.tiles > 1) hipLaunchKernelGGL(expert_count, dim3(a.tiles), dim3(kSortBlock), (unsigned)(sizeof(int) * a.E), s, a);
  hipLaunchKernelGGL(expert_place, dim3(a.tiles), dim3(kSortBlock), lds, s, a);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

// Groups of lanes that a row of `cols` elements, E a lane, is given: of 4, 16, 32 or 64.
template <typename Go> static void by_group(int64_t cols, int64_t E, Go go) {
  const int64_t lanes = (cols + E - 1) / E;
  if (lanes <= 4) go(Int<4>());
  else if (lanes <= 16) go(Int<16>());
  else if (lanes <= 32) go(Int<32>());
  else go(Int<64>());
}

// Blocks for the tokens, a group of G lanes each, and then, where rows are cleared, for 64 rows a wave.
template <typename Kernel> static void by_tokens(Kernel kernel, Move& a, int G, int64_t clear, hipStream_t s) {
  const int64_t tokens = (a.n + kBlock / G - 1) / (kBlock / G), all = tokens + (clear + kBlock - 1) / kBlock;
  a.token_blocks = (unsigned)tokens;
  dmt_launches(all, kBlock, [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, a, first); });
}

extern "C" dmt_status dmt_expert_gather(const void* x, int64_t n, int64_t cols, int64_t x_stride, int32_t dtype,
                                        const int32_t* slot, int64_t k, const int32_t* source, int64_t rows, void* out,
                                        int64_t out_stride, void* stream) {
  if (n < 0 || rows < 0 || cols < 1 || k < 1 || x_stride < cols || out_stride < cols || !dmt_is_dtype(dtype)) return DMT_EINVAL;
  const int64_t e = dmt_ebytes(dtype);
  if (n > 0 && (!dmt_is_at(x, e) || !dmt_is_at(slot, 4))) return DMT_EINVAL;
  if (rows > 0 && (!dmt_is_at(out, e) || !dmt_is_at(source, 4))) return DMT_EINVAL;
  if (!few(n, k) || rows > kMost || cols > 1 << 24) return DMT_ENOTSUP;
  if (rows == 0) return DMT_OK;
  Move a = {};
  a.x = (const char*)x, a.out = (char*)out, a.x_stride = x_stride, a.out_stride = out_stride, a.n = n, a.rows = rows;
  a.slot = slot, a.source = source, a.cols = (int)cols, a.k = (int)k;
  by_group(cols, 16 / e, [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (dtype == DMT_F32) by_tokens(expert_gather<4, G>, a, G, rows, (hipStream_t)stream);
    else by_tokens(expert_gather<2, G>, a, G, rows, (hipStream_t)stream);
  });
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" dmt_status dmt_expert_combine(const void* z, int64_t rows, int64_t cols, int64_t z_stride, int32_t dtype,
                                         const int32_t* slot, int64_t n, int64_t k, const float* weights, void* y,
                                         int64_t y_stride, int32_t y_dtype, void* stream) {
  if (n < 0 || rows < 0 || cols < 1 || k < 1 || z_stride < cols || y_stride < cols || !dmt_is_dtype(dtype) || !dmt_is_dtype(y_dtype))
    return DMT_EINVAL;
  if (rows > 0 && !dmt_is_at(z, dmt_ebytes(dtype))) return DMT_EINVAL;
  if (n > 0 && (!dmt_is_at(y, dmt_ebytes(y_dtype)) || !dmt_is_at(slot, 4))) return DMT_EINVAL;
  if (!dmt_may_be_at(weights, 4)) return DMT_EINVAL;
  if (!few(n, k) || rows > kMost || cols > 1 << 24) return DMT_ENOTSUP;
  if (n == 0) return DMT_OK;
  Move a = {};
  a.z = (const char*)z, a.out = (char*)y, a.z_stride = z_stride, a.out_stride = y_stride, a.n = n, a.rows = rows;
  a.slot = slot, a.weights = weights, a.cols = (int)cols, a.k = (int)k;
  by_type(dtype, [&](auto d) {
    by_type(y_dtype, [&](auto o) {
      by_group(cols, 8, [&](auto g) {
        constexpr int G = decltype(g)::value;
        by_tokens(expert_combine<decltype(d)::value, decltype(o)::value, G>, a, G, 0, (hipStream_t)stream);
      });
    });
  });
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" dmt_status dmt_expert_combine_bwd(const void* dy, int64_t n, int64_t cols, int64_t dy_stride,
                                             int32_t grad_dtype, const void* z, int64_t rows, int64_t z_stride,
                                             int32_t dtype, const int32_t* slot, int64_t k, const int32_t* source,
                                             const float* weights, void* dz, int64_t dz_stride, float* dweights,
                                             void* stream) {
  if (n < 0 || rows < 0 || cols < 1 || k < 1 || dy_stride < cols || !dmt_is_dtype(dtype)) return DMT_EINVAL;
  if (grad_dtype != dtype && grad_dtype != DMT_F32) return DMT_EINVAL;
  const int64_t ge = dmt_ebytes(grad_dtype);
  if (n > 0 && (!dmt_is_at(dy, ge) || !dmt_is_at(slot, 4))) return DMT_EINVAL;
  if (dz && (dz_stride < cols || !dmt_is_at(dz, ge) || (rows > 0 && !dmt_is_at(source, 4)))) return DMT_EINVAL;
  if (dweights && (z_stride < cols || !dmt_is_at(dweights, 4) || (rows > 0 && !dmt_is_at(z, dmt_ebytes(dtype))))) return DMT_EINVAL;
  if (!dmt_may_be_at(weights, 4)) return DMT_EINVAL;
  if (!few(n, k) || rows > kMost || cols > 1 << 24) return DMT_ENOTSUP;
  if (n == 0 && (!dz || rows == 0)) return DMT_OK;
  Move a = {};
  a.x = (const char*)dy, a.z = (const char*)z, a.out = (char*)dz, a.x_stride = dy_stride, a.z_stride = z_stride;
  a.out_stride = dz_stride, a.n = n, a.rows = rows, a.slot = slot, a.source = source, a.weights = weights;
  a.dweights = dweights, a.cols = (int)cols, a.k = (int)k;
  if (!dz && !dweights) return DMT_OK;
  by_type(dtype, [&](auto d) {
    by_group(cols, 8, [&](auto g) {
      constexpr int D = decltype(d)::value, G = decltype(g)::value;
      const int64_t clear = dz ? rows : 0;
      if (grad_dtype == D) by_tokens(expert_combine_bwd<D, D, G>, a, G, clear, (hipStream_t)stream);
      else by_tokens(expert_combine_bwd<D, DMT_F32, G>, a, G, clear, (hipStream_t)stream);
    });
  });
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
