// dmt_token_logprob_fwd, dmt_token_logprob_bwd: rows of scores as distributions.
//   M = max x, S = sum exp(x - M), T = sum exp(x - M) (x - M):  log p_j = x_j - M - log S,  H = log S - T / S.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;
constexpr float kInf = __builtin_inff();

template <int DT>
__global__ __launch_bounds__(kBlock) void logprob_fwd(const char* __restrict__ x, int vocab, int64_t stride,
                                                      const int32_t* __restrict__ targets,
                                                      float* __restrict__ logprob, float* __restrict__ entropy,
                                                      float* __restrict__ stats, int k,
                                                      int32_t* __restrict__ top_ids,
                                                      float* __restrict__ top_logprobs,
                                                      unsigned long long* __restrict__ first_bad) {
  constexpr int EB = dmt::EltBytes<DT>::value;
  __shared__ float sm[kWaves];
  __shared__ int si[kWaves];
  const int64_t r = blockIdx.x;
  const char* xr = x + r * stride * EB;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float m = -kInf;
  for (int j = threadIdx.x; j < vocab; j += kBlock) m = fmaxf(m, dmt::load1<DT>(xr + (int64_t)j * EB));
  m = dmt::group_max<64>(m);
  if (lane == 0) sm[wave] = m;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sm[w]);
  __syncthreads();
  float s = 0.f, t = 0.f;
  for (int j = threadIdx.x; j < vocab; j += kBlock) {
    const float v = dmt::load1<DT>(xr + (int64_t)j * EB);
    if (v == -kInf) continue;
    const float z = v - m, e = __expf(z);
    s += e;
    t += e * z;
  }
  s = dmt::block_sum<kWaves>(s, sm);
  t = dmt::block_sum<kWaves>(t, sm);
  const bool empty = s == 0.f;
  const float ls = logf(s);
  if (threadIdx.x == 0) {
    const int32_t at = targets ? targets[r] : -1;
    if (at >= vocab && first_bad) atomicMin(first_bad, (unsigned long long)r);
    if (logprob)
      logprob[r] = at < 0 || at >= vocab ? 0.f : empty ? -kInf : dmt::load1<DT>(xr + (int64_t)at * EB) - m - ls;
    if (entropy) entropy[r] = empty ? 0.f : ls - t / s;
    if (stats) stats[2 * r] = m, stats[2 * r + 1] = s;
  }
  // the largest score behind the last one taken, k times over
  float last = kInf;
  int last_at = -1;
  for (int i = 0; i < k; ++i) {
    float best = -kInf;
    int at = -1;
    if (last != -kInf)
      for (int j = threadIdx.x; j < vocab; j += kBlock) {
        const float v = dmt::load1<DT>(xr + (int64_t)j * EB);
        if ((v < last || (v == last && j > last_at)) && v > best) best = v, at = j;
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float b = __shfl_xor(best, o);
      const int a = __shfl_xor(at, o);
      if (b > best || (b == best && a >= 0 && a < at)) best = b, at = a;
    }
    if (lane == 0) sm[wave] = best, si[wave] = at;
    __syncthreads();
    best = -kInf, at = -1;
    for (int w = 0; w < kWaves; ++w)
      if (sm[w] > best || (sm[w] == best && si[w] >= 0 && si[w] < at)) best = sm[w], at = si[w];
    __syncthreads();
    if (threadIdx.x == 0) {
      top_ids[r * k + i] = at;
      if (top_logprobs) top_logprobs[r * k + i] = at < 0 ? -kInf : best - m - ls;
    }
    last = best, last_at = at;
  }
}

template <int DT>
__global__ __launch_bounds__(kBlock) void logprob_bwd(const char* x, int vocab, int64_t stride,
                                                      const int32_t* __restrict__ targets,
                                                      const float* __restrict__ stats,
                                                      const float* __restrict__ entropy,
                                                      const float* __restrict__ grad_logprob,
                                                      const float* __restrict__ grad_entropy, char* dx,
                                                      int64_t dx_stride) {
  constexpr int EB = dmt::EltBytes<DT>::value;
  const int64_t r = blockIdx.x;
  const char* xr = x + r * stride * EB;
  char* dr = dx + r * dx_stride * EB;
  const float m = stats[2 * r], s = stats[2 * r + 1];
  const int32_t at = targets ? targets[r] : -1;
  const bool aimed = at >= 0 && at < vocab;
  const float gl = grad_logprob && aimed ? grad_logprob[r] : 0.f;
  const float gh = grad_entropy ? grad_entropy[r] : 0.f, h = grad_entropy ? entropy[r] : 0.f;
  const float inv = 1.f / s, ls = logf(s);
  for (int j = threadIdx.x; j < vocab; j += kBlock) {
    const float v = dmt::load1<DT>(xr + (int64_t)j * EB);
    float d = 0.f;
    if (v != -kInf) {
      const float z = v - m, p = __expf(z) * inv;
      d = -gl * p - gh * (p * (z - ls + h));
      if (j == at) d += gl;
    }
    dmt::store1<DT>(dr + (int64_t)j * EB, d);
  }
}

bool fits(int64_t rows, int64_t vocab) { return rows < (1ll << 31) && vocab <= (1ll << 30); }

}  // namespace

extern "C" size_t dmt_token_logprob_workspace_bytes(int64_t rows, int64_t vocab, int32_t k) {
  if (rows < 0 || vocab < 1 || k < 0 || k > DMT_TOP_MAX || !fits(rows, vocab)) return 0;
  return 0;
}

extern "C" dmt_status dmt_token_logprob_fwd(const void* x, int64_t rows, int64_t vocab, int64_t x_stride,
                                            int32_t dtype, const int32_t* targets, float* logprob,
                                            float* entropy, float* stats, int32_t k, int32_t* top_ids,
                                            float* top_logprobs, int64_t* first_bad, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  if (rows < 0 || vocab < 1 || x_stride < vocab || !dmt_is_dtype(dtype) || k < 0 || k > DMT_TOP_MAX) return DMT_EINVAL;
  if (!dmt_may_be_at(targets, 4) || !dmt_may_be_at(logprob, 4) || !dmt_may_be_at(entropy, 4) || !dmt_may_be_at(stats, 4) ||
      !dmt_may_be_at(top_ids, 4) || !dmt_may_be_at(top_logprobs, 4) || !dmt_may_be_at(first_bad, 8))
    return DMT_EINVAL;
  if (rows > 0 && (!dmt_is_at(x, dmt_ebytes(dtype)) || (logprob && !targets) || (k > 0 && !top_ids))) return DMT_EINVAL;
  if (!fits(rows, vocab)) return DMT_ENOTSUP;
  const size_t need = dmt_token_logprob_workspace_bytes(rows, vocab, k);
  if (need > 0 && !dmt_is_at(workspace, 256)) return DMT_EINVAL;
  if (workspace_bytes < need) return DMT_ENOMEM;
  if (rows == 0) return DMT_OK;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kBlock), 0, (hipStream_t)stream, (const char*)x, (int)vocab,
                       x_stride, targets, logprob, entropy, stats, (int)k, top_ids, top_logprobs,
                       (unsigned long long*)first_bad);
  };
  if (dtype == DMT_F32) go(logprob_fwd<DMT_F32>);
  else if (dtype == DMT_F16) go(logprob_fwd<DMT_F16>);
  else go(logprob_fwd<DMT_BF16>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" dmt_status dmt_token_logprob_bwd(const void* x, int64_t rows, int64_t vocab, int64_t x_stride,
                                            int32_t dtype, const int32_t* targets, const float* stats,
                                            const float* entropy, const float* grad_logprob,
                                            const float* grad_entropy, void* dx, int64_t dx_stride,
                                            void* stream) {
  if (rows < 0 || vocab < 1 || x_stride < vocab || dx_stride < vocab || !dmt_is_dtype(dtype)) return DMT_EINVAL;
  if (!dmt_may_be_at(targets, 4) || !dmt_may_be_at(stats, 4) || !dmt_may_be_at(entropy, 4) ||
      !dmt_may_be_at(grad_logprob, 4) || !dmt_may_be_at(grad_entropy, 4))
    return DMT_EINVAL;
  const int64_t e = dmt_ebytes(dtype);
  if (rows > 0 && (!dmt_is_at(x, e) || !dmt_is_at(dx, e) || !stats || (grad_logprob && !targets) ||
                   (grad_entropy && !entropy)))
    return DMT_EINVAL;
  if (x == dx && x_stride != dx_stride && rows > 1) return DMT_EINVAL;
  if (!fits(rows, vocab)) return DMT_ENOTSUP;
  if (rows == 0) return DMT_OK;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kBlock), 0, (hipStream_t)stream, (const char*)x, (int)vocab,
                       x_stride, targets, stats, entropy, grad_logprob, grad_entropy, (char*)dx, dx_stride);
  };
  if (dtype == DMT_F32) go(logprob_bwd<DMT_F32>);
  else if (dtype == DMT_F16) go(logprob_bwd<DMT_F16>);
  else go(logprob_bwd<DMT_BF16>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
