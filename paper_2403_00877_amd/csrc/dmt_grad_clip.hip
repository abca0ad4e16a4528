// dmt_grad_norm, dmt_grad_clip: the 2-norm over many gradients, and the gradients scaled by what it says.
// The tensors are cut into chunks; a block per chunk sums squares in float64, one block adds the chunks up in a
// fixed order.  The tensors' addresses travel as kernel arguments: nothing is copied to the device and a
// call may be captured.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;
constexpr int64_t kChunk = 32768;                 // elements
constexpr int kTensors = 120;                     // of one launch: kernel arguments end at 4 KB

struct Tensors {
  const char* in[kTensors];
  char* out[kTensors];
  int64_t numel_dt[kTensors];                     // elements << 2 | type
  uint32_t first[kTensors + 1];                   // first chunk, of the launch's
  int32_t count;
};
static_assert(sizeof(Tensors) <= 4000, "kernel arguments");

// The tensor of a launch's chunk.
__device__ __forceinline__ int tensor_of(const Tensors& t, uint32_t chunk) {
  int lo = 0, hi = t.count;                       // first[lo] <= chunk < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.first[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int DT>
__device__ __forceinline__ double chunk_squares(const char* in, int64_t n) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value;
  double s = 0;
  for (int64_t c = threadIdx.x * E; c < n; c += kBlock * E) {
    float x[E];
    dmt::load_elems<DT, E>(in + c * EB, (int)min((int64_t)E, n - c), x);
#pragma unroll
    for (int q = 0; q < E; ++q) s = fma((double)x[q], (double)x[q], s);
  }
  return s;
}

__device__ __forceinline__ double block_sum_f64(double v, double* smem) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += smem[w];
  return s;
}

__global__ __launch_bounds__(kBlock) void grad_squares(const Tensors t, double* __restrict__ part) {
  __shared__ double sm[kWaves];
  const int i = tensor_of(t, blockIdx.x);
  const int dt = (int)(t.numel_dt[i] & 3);
  const int64_t at = (int64_t)(blockIdx.x - t.first[i]) * kChunk, n = min(kChunk, (t.numel_dt[i] >> 2) - at);
  double s;
  if (dt == DMT_F32) s = chunk_squares<DMT_F32>(t.in[i] + at * 4, n);
  else if (dt == DMT_F16) s = chunk_squares<DMT_F16>(t.in[i] + at * 2, n);
  else s = chunk_squares<DMT_BF16>(t.in[i] + at * 2, n);
  s = block_sum_f64(s, sm);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void grad_norm_sum(const double* __restrict__ part, int64_t n, float* __restrict__ norm,
                                                      float max_norm, float* __restrict__ coef) {
  __shared__ double sm[16];
  double s = 0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = block_sum_f64(s, sm);
  if (threadIdx.x == 0) {
    const float v = (float)sqrt(s), c = max_norm / (v + 1e-6f);
    if (norm) *norm = v;
    if (coef) *coef = c >= 1.f ? 1.f : c;         // (NaN stays)
  }
}

template <int DT>
__device__ __forceinline__ void chunk_scale(const char* in, char* out, int64_t n, float c) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value;
  for (int64_t e = threadIdx.x * E; e < n; e += kBlock * E) {
    const int valid = (int)min((int64_t)E, n - e);
    float x[E];
    dmt::load_elems<DT, E>(in + e * EB, valid, x);
#pragma unroll
    for (int q = 0; q < E; ++q) x[q] *= c;
    dmt::store_elems<DT, E>(out + e * EB, valid, x);
  }
}

__global__ __launch_bounds__(kBlock) void grad_scale(const Tensors t, const float* __restrict__ coef) {
  const float c = *coef;
  const int i = tensor_of(t, blockIdx.x);
  if (c == 1.f && t.in[i] == t.out[i]) return;
  const int dt = (int)(t.numel_dt[i] & 3);
  const int64_t at = (int64_t)(blockIdx.x - t.first[i]) * kChunk, n = min(kChunk, (t.numel_dt[i] >> 2) - at);
  if (dt == DMT_F32) chunk_scale<DMT_F32>(t.in[i] + at * 4, t.out[i] + at * 4, n, c);
  else if (dt == DMT_F16) chunk_scale<DMT_F16>(t.in[i] + at * 2, t.out[i] + at * 2, n, c);
  else chunk_scale<DMT_BF16>(t.in[i] + at * 2, t.out[i] + at * 2, n, c);
}

int64_t chunks_of(int64_t numel) { return (numel + kChunk - 1) / kChunk; }

dmt_status check(const dmt_grad_tensor* t, int64_t count, bool outs, int64_t* chunks) {
  if (count < 0 || (count > 0 && !t)) return DMT_EINVAL;
  if (count > (1 << 20)) return DMT_ENOTSUP;
  *chunks = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (t[i].numel < 0 || !dmt_is_dtype(t[i].dtype)) return DMT_EINVAL;
    if (t[i].numel > (1ll << 40)) return DMT_ENOTSUP;
    if (t[i].numel == 0) continue;
    const int64_t e = dmt_ebytes(t[i].dtype);
    if (!dmt_is_at(t[i].data, e) || (outs && !dmt_is_at(t[i].out, e))) return DMT_EINVAL;
    *chunks += chunks_of(t[i].numel);
  }
  return *chunks < (1ll << 31) ? DMT_OK : DMT_ENOTSUP;
}

// Calls go(tensors, chunks of the launch, chunks before it) for every launch.
template <typename Go>
void launches(const dmt_grad_tensor* t, int64_t count, Go go) {
  Tensors a;
  int64_t before = 0;
  a.count = 0;
  a.first[0] = 0;
  auto flush = [&]() {
    if (a.count > 0) go(a, a.first[a.count], before);
    before += a.first[a.count];
    a.count = 0;
  };
  for (int64_t i = 0; i < count; ++i) {
    if (t[i].numel == 0) continue;
    const int at = a.count++;
    a.in[at] = (const char*)t[i].data;
    a.out[at] = (char*)t[i].out;
    a.numel_dt[at] = t[i].numel << 2 | t[i].dtype;
    a.first[a.count] = a.first[at] + (uint32_t)chunks_of(t[i].numel);
    if (a.count == kTensors) flush();
  }
  flush();
}

dmt_status norm_run(const dmt_grad_tensor* t, int64_t count, float max_norm, float* norm, bool clip, void* workspace,
                    size_t workspace_bytes, hipStream_t s) {
  int64_t chunks = 0;
  const dmt_status ok = check(t, count, clip, &chunks);
  if (ok != DMT_OK) return ok;
  if (!dmt_is_at(workspace, 256)) return DMT_EINVAL;
  if (workspace_bytes < sizeof(double) * (size_t)(chunks + 1)) return DMT_ENOMEM;
  float* coef = (float*)workspace;
  double* part = (double*)workspace + 1;
  launches(t, count, [&](const Tensors& a, uint32_t n, int64_t before) {
    hipLaunchKernelGGL(grad_squares, dim3(n), dim3(kBlock), 0, s, a, part + before);
  });
  hipLaunchKernelGGL(grad_norm_sum, dim3(1), dim3(1024), 0, s, part, chunks, norm, max_norm, clip ? coef : nullptr);
  if (clip)
    launches(t, count, [&](const Tensors& a, uint32_t n, int64_t) {
      hipLaunchKernelGGL(grad_scale, dim3(n), dim3(kBlock), 0, s, a, coef);
    });
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

}  // namespace

extern "C" size_t dmt_grad_norm_workspace_bytes(const dmt_grad_tensor* tensors, int64_t count) {
  int64_t chunks = 0;
  if (check(tensors, count, false, &chunks) != DMT_OK) return 0;
  return sizeof(double) * (size_t)(chunks + 1);
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
