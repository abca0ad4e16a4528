// dmt_embed_fwd, dmt_embed_bwd: a table's rows by id, scaled, and the table's gradient in dense form.
//
// Backward.  Lookups are sorted by id (stable radix sort of (id, position) records: digits of up to 11
// bits, three launches a digit), then a lane group per table row finds the row's records by bisection and
// adds their gradient rows in ascending position.  One writer per row, no atomics on values: the same bits every time.
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
    int shift, int bits, uint32_t* __restrict__ counts, unsigned long long* __restrict__ first_bad) {
  __shared__ uint32_t cnt[1 << kMaxDigit];
  const int nd = 1 << bits;
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
    uint64_t* __restrict__ out) {
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
    }
}

// ------------------------------------------------------------------ the sums

template <int GD>
__global__ __launch_bounds__(kBlock) void embed_reduce(
    const uint64_t* __restrict__ recs, int64_t n, const char* __restrict__ grad, int64_t grad_stride,
    float scale, float* __restrict__ out, int64_t rows, int cols, int64_t out_stride, int accumulate,
    int log2_lpr) {
  constexpr int E = dmt::ChunkElems<GD>::value, GB = dmt::EltBytes<GD>::value;
  const int lane = threadIdx.x & ((1 << log2_lpr) - 1);
  const int64_t v = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> log2_lpr;
  if (v >= rows) return;
  int64_t lo = 0, hi = n;                                // the first record whose key is not below v
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if ((int64_t)(recs[mid] >> 32) < v) lo = mid + 1;
    else hi = mid;
  }
  const bool any = lo < n && (int64_t)(recs[lo] >> 32) == v;
  if (!any && accumulate) return;
  for (int c = lane * E; c < cols; c += E << log2_lpr) {
    const int valid = min(E, cols - c);
    float acc[E], x[E];
#pragma unroll
    for (int q = 0; q < E; ++q) acc[q] = 0.f;
    for (int64_t j = lo; j < n && (int64_t)(recs[j] >> 32) == v; ++j) {
      dmt::load_elems<GD, E>(grad + ((int64_t)(uint32_t)recs[j] * grad_stride + c) * GB, valid, x);
#pragma unroll
      for (int q = 0; q < E; ++q) acc[q] += x[q];
    }
    char* dst = (char*)(out + v * out_stride + c);
    if (accumulate) dmt::load_elems<DMT_F32, E>(dst, valid, x);
#pragma unroll
    for (int q = 0; q < E; ++q) acc[q] = accumulate ? x[q] + scale * acc[q] : scale * acc[q];
    dmt::store_elems<DMT_F32, E>(dst, valid, acc);
  }
}

int log2_lanes(int64_t cols, int E) {
  int l = 0;
  while (l < 6 && (int64_t)(E << l) < cols) ++l;
  return l;
}

struct Ws {
  uint64_t *a, *b;
  uint32_t *counts, *totals;
  int64_t nblk;
  int items, passes, bits;
  size_t bytes;
};

Ws carve(int64_t n, int64_t rows, void* at) {
  Ws w;
  w.items = (int)std::min<int64_t>(kMaxItems, std::max<int64_t>(1, (n + kSortBlock * kSortFill - 1) / (kSortBlock * kSortFill)));
  w.nblk = std::max<int64_t>(1, (n + kSortBlock * w.items - 1) / (kSortBlock * w.items));
  int bits = 1;
  while ((rows >> bits) != 0) ++bits;                    // the key `rows` included
  w.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  w.bits = (bits + w.passes - 1) / w.passes;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = dmt_align_up(off + bytes, 256);
    return (char*)((uintptr_t)at + o);
  };
  w.a = (uint64_t*)take(sizeof(uint64_t) * (size_t)n);
  w.b = (uint64_t*)take(sizeof(uint64_t) * (size_t)n);
  w.counts = (uint32_t*)take(sizeof(uint32_t) * ((size_t)w.nblk << w.bits));
  w.totals = (uint32_t*)take(sizeof(uint32_t) << w.bits);
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
                     w.items, shift, w.bits, w.counts, (unsigned long long*)bad);
  hipLaunchKernelGGL(embed_digit_starts, dim3((nd + 63) / 64), dim3(64), 0, s, w.counts, w.nblk, nd, w.totals);
  static DmtPerDevice done;
  dmt_allow_lds(done, (const void*)embed_scatter<First>, (4 + 2 * kSortWaves) << kMaxDigit);
  hipLaunchKernelGGL(embed_scatter<First>, dim3((unsigned)w.nblk), dim3(kSortBlock), (4 + 2 * kSortWaves) << w.bits, s,
                     ids, in, n, (uint32_t)rows, w.items, shift, w.bits, w.counts, w.totals, out);
}

template <int GD>
void launch_reduce(const uint64_t* recs, int64_t n, const void* grad, int64_t gs, float scale, float* out,
                   int64_t rows, int64_t cols, int64_t os, int acc, hipStream_t s) {
  const int l = log2_lanes(cols, dmt::ChunkElems<GD>::value);
  hipLaunchKernelGGL(embed_reduce<GD>, dim3((unsigned)(((rows << l) + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, recs,
                     n, (const char*)grad, gs, scale, out, rows, (int)cols, os, acc, l);
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
  return carve(n, rows, nullptr).bytes;
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
  const Ws w = carve(n, rows, workspace);
  if (workspace_bytes < w.bytes) return DMT_ENOMEM;
  hipStream_t s = (hipStream_t)stream;
  uint64_t *in = w.b, *out = w.a;
  for (int p = 0; p < w.passes && n > 0; ++p) {
    if (p == 0) launch_pass<true>(w, ids, nullptr, out, n, rows, 0, first_bad, s);
    else launch_pass<false>(w, ids, in, out, n, rows, p * w.bits, first_bad, s);
    std::swap(in, out);
  }
  if (grad_dtype == DMT_F32)
    launch_reduce<DMT_F32>(in, n, grad, grad_stride, scale, grad_table, rows, cols, grad_table_stride, accumulate, s);
  else if (grad_dtype == DMT_F16)
    launch_reduce<DMT_F16>(in, n, grad, grad_stride, scale, grad_table, rows, cols, grad_table_stride, accumulate, s);
  else
    launch_reduce<DMT_BF16>(in, n, grad, grad_stride, scale, grad_table, rows, cols, grad_table_stride, accumulate, s);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
