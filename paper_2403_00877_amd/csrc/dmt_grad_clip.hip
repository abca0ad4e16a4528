// dmt_grad_norm, dmt_grad_clip: the 2-norm over many gradients, and the gradients scaled by what it says.
//
// The tensors are cut into units and the blocks stride over them.  A block sums squares in float64; the scaling's blocks each
// add the blocks' sums up again, in the same order, rather than wait for a launch that does.  Bound by memory: the
// gradients are read, then read and written: 872 MB in 180 tensors 574 us, 4.6 TB/s; 3.5 MB in 16 tensors 10 us, two launches.  (The
// scaling backwards, from what was read last: no faster.)
// The tensors' addresses travel as kernel arguments: nothing is copied to the device and a call may be captured.
#include <algorithm>
#include <type_traits>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;
constexpr int64_t kLeastUnit = 2048;
constexpr int64_t kMostUnit = 16384;
// Gradients of more bytes than the Infinity Cache holds need not pass through it before the scaling: 872 MB, squares 197 ->
// 169 us, the scaling 358 -> 369.
constexpr int64_t kCacheBytes = 256 << 20;
constexpr int64_t kBlocks = 2048;                 // of a launch, at most, and sums
constexpr int kVecs = 4;                          // 16-byte pieces of a thread under way

// The tensors of a launch, as many as kernel arguments of 4 KB hold.  Without Outs nothing is written, or in place.
// (130 tensors, 13 MB of bfloat16: 21 us in one launch each, 31 in two.)
template <bool Outs> struct Tensors {
  static constexpr int kMost = Outs ? 134 : 188;
  const char* in[kMost];
  char* outs[Outs ? kMost : 1];
  int64_t numel_dt[kMost];                        // elements << 2 | type
  uint32_t first[kMost + 1];                      // first unit, of the launch's
  int32_t count;
  int32_t unit;                                   // elements
  __device__ __forceinline__ char* out(int i) const { return Outs ? outs[i] : (char*)in[i]; }
};
static_assert(sizeof(Tensors<true>) <= 3800 && sizeof(Tensors<false>) <= 3800, "kernel arguments: 4 KB with the others and the launch's sizes");

// Calls go(tensor, from, to) for the block's units, every gridDim.x-th of all.
template <bool Outs, typename Go> __device__ __forceinline__ void each_unit(const Tensors<Outs>& t, Go go) {
  const uint32_t all = t.first[t.count];
  for (uint32_t u = blockIdx.x; u < all; u += gridDim.x) {
    int lo = 0, hi = t.count;                     // first[lo] <= u < first[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (t.first[mid] <= u) lo = mid;
      else hi = mid;
    }
    const int64_t from = (int64_t)(u - t.first[lo]) * t.unit;
    go(lo, from, min(from + t.unit, t.numel_dt[lo] >> 2));
  }
}

template <int DT, bool Once> __device__ __forceinline__ void squares(const char* in, int64_t from, int64_t to, double& s) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value;
  for (int64_t c0 = from; c0 < to; c0 += kBlock * E * kVecs) {
    dmt::Raw<DT, E> r[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int64_t c = c0 + (v * kBlock + (int)threadIdx.x) * E;
      if (c < to) r[v] = dmt::load_raw<DT, E, Once>(in + c * EB, (int)min((int64_t)E, to - c));
    }
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      if (c0 + (v * kBlock + (int)threadIdx.x) * E >= to) break;
      float x[E];
      dmt::unpack<DT, E>(r[v], x);
#pragma unroll
      for (int q = 0; q < E; ++q) s = fma((double)x[q], (double)x[q], s);
    }
  }
}

// Sum over the block, the same in every thread; of NW waves.
template <int NW> __device__ __forceinline__ double block_sum_f64(double v, double* smem) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) s += smem[w];
  return s;
}

// part[block] = or += (launches behind the first) the squares of its run.
// Once: the gradients pass the caches by.
template <bool Once>
__global__ __launch_bounds__(kBlock) void grad_squares(const Tensors<false> t, int later, double* __restrict__ part) {
  __shared__ double sm[kWaves];
  double s = 0;
  each_unit(t, [&](int i, int64_t from, int64_t to) {
    const int dt = (int)(t.numel_dt[i] & 3);
    if (dt == DMT_F32) squares<DMT_F32, Once>(t.in[i], from, to, s);
    else if (dt == DMT_F16) squares<DMT_F16, Once>(t.in[i], from, to, s);
    else squares<DMT_BF16, Once>(t.in[i], from, to, s);
  });
  s = block_sum_f64<kWaves>(s, sm);
  if (threadIdx.x == 0) part[blockIdx.x] = later ? part[blockIdx.x] + s : s;
}

// The norm from `n` sums, the same in every thread of the block.
__device__ __forceinline__ float norm_of(const double* __restrict__ part, int n, double* smem) {
  double s = 0;
  for (int i = threadIdx.x; i < n; i += kBlock) s += part[i];
  return (float)sqrt(block_sum_f64<kWaves>(s, smem));
}

__global__ __launch_bounds__(kBlock) void grad_norm(const double* __restrict__ part, int n, float* __restrict__ norm) {
  __shared__ double sm[kWaves];
  const float v = norm_of(part, n, sm);
  if (threadIdx.x == 0) *norm = v;
}

template <int DT> __device__ __forceinline__ void scale(const char* in, char* out, int64_t from, int64_t to, float f) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value;
  constexpr int64_t step = (int64_t)kBlock * E * kVecs;
  for (int64_t c0 = from; c0 < to; c0 += step) {
    dmt::Raw<DT, E> r[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int64_t c = c0 + (v * kBlock + (int)threadIdx.x) * E;
      if (c < to) r[v] = dmt::load_raw<DT, E>(in + c * EB, (int)min((int64_t)E, to - c));
    }
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int64_t c = c0 + (v * kBlock + (int)threadIdx.x) * E;
      if (c >= to) break;
      float x[E];
      dmt::unpack<DT, E>(r[v], x);
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] *= f;
      dmt::store_elems<DT, E>(out + c * EB, (int)min((int64_t)E, to - c), x);
    }
  }
}

template <bool Outs>
__global__ __launch_bounds__(kBlock) void grad_scale(const Tensors<Outs> t, const double* __restrict__ part, int n,
                                                     float max_norm, float* __restrict__ norm) {
  __shared__ double sm[kWaves];
  const float v = norm_of(part, n, sm), q = max_norm / (v + 1e-6f), f = q >= 1.f ? 1.f : q;     // (NaN stays)
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
  each_unit(t, [&](int i, int64_t from, int64_t to) {
    char* out = t.out(i);
    if (f == 1.f && t.in[i] == out) return;
    const int dt = (int)(t.numel_dt[i] & 3);
    if (dt == DMT_F32) scale<DMT_F32>(t.in[i], out, from, to, f);
    else if (dt == DMT_F16) scale<DMT_F16>(t.in[i], out, from, to, f);
    else scale<DMT_BF16>(t.in[i], out, from, to, f);
  });
}

// Elements of a unit: at least eight units for every block, as far as they are not too short or too long.
struct Division {
  int64_t unit, blocks, bytes;
  bool in_place;                                  // all that is written
};

dmt_status check(const dmt_grad_tensor* t, int64_t count, bool outs, Division* d) {
  if (count < 0 || (count > 0 && !t)) return DMT_EINVAL;
  if (count > (1 << 20)) return DMT_ENOTSUP;
  int64_t total = 0, there = 0;
  d->bytes = 0;
  d->in_place = true;
  for (int64_t i = 0; i < count; ++i) {
    if (t[i].numel < 0 || !dmt_is_dtype(t[i].dtype)) return DMT_EINVAL;
    if (t[i].numel > (1ll << 40)) return DMT_ENOTSUP;
    if (t[i].numel == 0) continue;
    const int64_t e = dmt_ebytes(t[i].dtype);
    if (!dmt_is_at(t[i].data, e) || (outs && !dmt_is_at(t[i].out, e))) return DMT_EINVAL;
    total += t[i].numel;
    d->bytes += t[i].numel * e;
    d->in_place = d->in_place && t[i].out == t[i].data;
    ++there;
    if (total > (1ll << 44)) return DMT_ENOTSUP;            // (units are numbered in 32 bits)
  }
  d->unit = kLeastUnit;
  while (d->unit < kMostUnit && total / (2 * d->unit) >= 8 * kBlocks) d->unit *= 2;
  d->blocks = std::min(kBlocks, total / d->unit + there);   // (never fewer than there are units, below kBlocks)
  return DMT_OK;
}

// Calls go(tensors, number of the launch) for every launch.
template <bool Outs, typename Go> void launches(const dmt_grad_tensor* t, int64_t count, int64_t unit, Go go) {
  Tensors<Outs> a;
  int launch = 0;
  a.count = 0;
  a.first[0] = 0;
  a.unit = (int32_t)unit;
  auto flush = [&]() {
    if (a.count > 0) go(a, launch++);
    a.count = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    if (t[i].numel == 0) continue;
    const int at = a.count++;
    a.in[at] = (const char*)t[i].data;
    if (Outs) a.outs[at] = (char*)t[i].out;
    a.numel_dt[at] = t[i].numel << 2 | t[i].dtype;
    a.first[a.count] = a.first[at] + (uint32_t)((t[i].numel + unit - 1) / unit);
    if (a.count == Tensors<Outs>::kMost) flush();
  }
  flush();
}

dmt_status norm_run(const dmt_grad_tensor* t, int64_t count, float max_norm, float* norm, bool clip, void* workspace,
                    size_t workspace_bytes, hipStream_t s) {
  Division d;
  const dmt_status ok = check(t, count, clip, &d);
  if (ok != DMT_OK) return ok;
  if (!dmt_is_at(workspace, 256)) return DMT_EINVAL;
  if (workspace_bytes < sizeof(double) * (size_t)std::max<int64_t>(d.blocks, 1)) return DMT_ENOMEM;
  double* part = (double*)workspace;
  // blocks of a launch; the first one writes all the blocks' sums
  auto grid = [&](const auto& a, bool all) { return dim3((unsigned)(all ? d.blocks : std::min<int64_t>(d.blocks, a.first[a.count]))); };
  launches<false>(t, count, d.unit, [&](const Tensors<false>& a, int launch) {
    const dim3 g = grid(a, launch == 0);
    if (d.bytes > kCacheBytes) hipLaunchKernelGGL(grad_squares<true>, g, dim3(kBlock), 0, s, a, launch > 0, part);
    else hipLaunchKernelGGL(grad_squares<false>, g, dim3(kBlock), 0, s, a, launch > 0, part);
  });
  auto scaling = [&](auto outs) {
    constexpr bool Outs = decltype(outs)::value;
    launches<Outs>(t, count, d.unit, [&](const Tensors<Outs>& a, int launch) {
      hipLaunchKernelGGL(grad_scale<Outs>, grid(a, false), dim3(kBlock), 0, s, a, part, (int)d.blocks, max_norm,
                         launch == 0 ? norm : nullptr);
    });
  };
  if (clip && d.blocks > 0) d.in_place ? scaling(std::false_type()) : scaling(std::true_type());
  else if (norm)
    hipLaunchKernelGGL(grad_norm, dim3(1), dim3(kBlock), 0, s, part, (int)d.blocks, norm);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

}  // namespace

extern "C" size_t dmt_grad_norm_workspace_bytes(const dmt_grad_tensor* tensors, int64_t count) {
  Division d;
  if (check(tensors, count, false, &d) != DMT_OK) return 0;
  return sizeof(double) * (size_t)std::max<int64_t>(1, d.blocks);
}

extern "C" dmt_status dmt_grad_norm(const dmt_grad_tensor* tensors, int64_t count, float* norm,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!dmt_is_at(norm, 4)) return DMT_EINVAL;
  return norm_run(tensors, count, 0.f, norm, false, workspace, workspace_bytes, (hipStream_t)stream);
}

extern "C" dmt_status dmt_grad_clip(const dmt_grad_tensor* tensors, int64_t count, float max_norm, float* norm,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!dmt_may_be_at(norm, 4) || !(max_norm >= 0.f)) return DMT_EINVAL;
  return norm_run(tensors, count, max_norm, norm, true, workspace, workspace_bytes, (hipStream_t)stream);
}
