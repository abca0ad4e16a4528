// dmt_layer_norm_fwd, dmt_layer_norm_bwd.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;

template <int XD>
__global__ __launch_bounds__(kBlock) void norm_fwd(const char* x, int cols, int64_t x_stride,
                                                   const void* __restrict__ gamma,
                                                   const void* __restrict__ beta, int wdt, float eps, char* y,
                                                   int64_t y_stride, float* __restrict__ mean,
                                                   float* __restrict__ rstd) {
  constexpr int E = dmt::ChunkElems<XD>::value, XB = dmt::EltBytes<XD>::value;
  __shared__ float sm[kWaves];
  const int64_t r = blockIdx.x;
  const char* xr = x + r * x_stride * XB;
  float s = 0.f, v[E];
  for (int c = threadIdx.x * E; c < cols; c += kBlock * E) {
    dmt::load_elems<XD, E>(xr + (int64_t)c * XB, min(E, cols - c), v);
#pragma unroll
    for (int q = 0; q < E; ++q) s += v[q];
  }
  const float m = dmt::block_sum<kWaves>(s, sm) / (float)cols;
  s = 0.f;
  for (int c = threadIdx.x * E; c < cols; c += kBlock * E) {
    const int valid = min(E, cols - c);
    dmt::load_elems<XD, E>(xr + (int64_t)c * XB, valid, v);
#pragma unroll
    for (int q = 0; q < E; ++q) s += q < valid ? (v[q] - m) * (v[q] - m) : 0.f;
  }
  const float rs = 1.f / sqrtf(dmt::block_sum<kWaves>(s, sm) / (float)cols + eps);
  for (int c = threadIdx.x * E; c < cols; c += kBlock * E) {
    const int valid = min(E, cols - c);
    dmt::load_elems<XD, E>(xr + (int64_t)c * XB, valid, v);
#pragma unroll
    for (int q = 0; q < E; ++q) {
      v[q] = (v[q] - m) * rs;
      if (gamma && q < valid) v[q] *= dmt::load1_dyn(gamma, c + q, wdt);
      if (beta && q < valid) v[q] += dmt::load1_dyn(beta, c + q, wdt);
    }
    dmt::store_elems<XD, E>(y + (r * y_stride + c) * XB, valid, v);
  }
  if (threadIdx.x == 0) {
    if (mean) mean[r] = m;
    if (rstd) rstd[r] = rs;
  }
}

template <int XD, int GD>
__global__ __launch_bounds__(kBlock) void norm_bwd_rows(const char* __restrict__ x, int cols, int64_t x_stride,
                                                        const void* __restrict__ gamma, int wdt,
                                                        const float* __restrict__ mean,
                                                        const float* __restrict__ rstd, const char* dy,
                                                        int64_t dy_stride, char* dx, int64_t dx_stride) {
  constexpr int XB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  __shared__ float sm[kWaves];
  const int64_t r = blockIdx.x;
  const float m = mean[r], rs = rstd[r];
  float a = 0.f, b = 0.f;
  for (int c = threadIdx.x; c < cols; c += kBlock) {
    const float h = (dmt::load1<XD>(x + (r * x_stride + c) * XB) - m) * rs;
    const float g = dmt::load1<GD>(dy + (r * dy_stride + c) * GB) * (gamma ? dmt::load1_dyn(gamma, c, wdt) : 1.f);
    a += g;
    b += g * h;
  }
  a = dmt::block_sum<kWaves>(a, sm) / (float)cols;
  b = dmt::block_sum<kWaves>(b, sm) / (float)cols;
  for (int c = threadIdx.x; c < cols; c += kBlock) {
    const float h = (dmt::load1<XD>(x + (r * x_stride + c) * XB) - m) * rs;
    const float g = dmt::load1<GD>(dy + (r * dy_stride + c) * GB) * (gamma ? dmt::load1_dyn(gamma, c, wdt) : 1.f);
    dmt::store1<GD>(dx + (r * dx_stride + c) * GB, rs * (g - a - h * b));
  }
}

// Sums over the rows, one slice of them a block.
constexpr int64_t kSlices = 128;
template <int XD, int GD>
__global__ __launch_bounds__(kBlock) void norm_bwd_slices(const char* __restrict__ x, int64_t rows, int cols,
                                                          int64_t x_stride, const float* __restrict__ mean,
                                                          const float* __restrict__ rstd,
                                                          const char* __restrict__ dy, int64_t dy_stride,
                                                          int64_t per, float* __restrict__ part) {
  constexpr int XB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  const int c = blockIdx.x * kBlock + threadIdx.x;
  if (c >= cols) return;
  const int64_t r0 = blockIdx.y * per, r1 = min(rows, r0 + per);
  float a = 0.f, b = 0.f;
  for (int64_t r = r0; r < r1; ++r) {
    const float d = dmt::load1<GD>(dy + (r * dy_stride + c) * GB);
    a += d * ((dmt::load1<XD>(x + (r * x_stride + c) * XB) - mean[r]) * rstd[r]);
    b += d;
  }
  part[(int64_t)blockIdx.y * 2 * cols + c] = a;
  part[((int64_t)blockIdx.y * 2 + 1) * cols + c] = b;
}

__global__ __launch_bounds__(kBlock) void norm_bwd_sum(const float* __restrict__ part, int64_t slices, int cols,
                                                       float* __restrict__ dgamma, float* __restrict__ dbeta) {
  const int c = blockIdx.x * kBlock + threadIdx.x;
  if (c >= cols) return;
  float a = 0.f, b = 0.f;
  for (int64_t s = 0; s < slices; ++s) {
    a += part[s * 2 * cols + c];
    b += part[(s * 2 + 1) * cols + c];
  }
  if (dgamma) dgamma[c] = a;
  if (dbeta) dbeta[c] = b;
}

int64_t slices_of(int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>(kSlices, rows)); }

bool fits(int64_t rows, int64_t cols) { return rows < (1ll << 31) && cols <= (1 << 24); }

}  // namespace

extern "C" dmt_status dmt_layer_norm_fwd(const void* x, int64_t rows, int64_t cols, int64_t x_stride,
                                         int32_t dtype, const void* gamma, const void* beta,
                                         int32_t weight_dtype, float eps, void* y, int64_t y_stride,
                                         float* mean, float* rstd, void* stream) {
  if (rows < 0 || cols < 1 || x_stride < cols || y_stride < cols || !dmt_is_dtype(dtype)) return DMT_EINVAL;
  if ((gamma || beta) && weight_dtype != dtype && weight_dtype != DMT_F32) return DMT_EINVAL;
  const int64_t e = dmt_ebytes(dtype), we = dmt_ebytes(weight_dtype);
  if (!dmt_may_be_at(gamma, we) || !dmt_may_be_at(beta, we) || !dmt_may_be_at(mean, 4) || !dmt_may_be_at(rstd, 4))
    return DMT_EINVAL;
  if (!(eps >= 0.f)) return DMT_EINVAL;
  if (rows > 0 && (!dmt_is_at(x, e) || !dmt_is_at(y, e))) return DMT_EINVAL;
  if (x == y && x_stride != y_stride && rows > 1) return DMT_EINVAL;
  if (!fits(rows, cols)) return DMT_ENOTSUP;
  if (rows == 0) return DMT_OK;
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(kBlock), 0, s, (const char*)x, (int)cols, x_stride, gamma,
                       beta, weight_dtype, eps, (char*)y, y_stride, mean, rstd);
  };
  if (dtype == DMT_F32) go(norm_fwd<DMT_F32>);
  else if (dtype == DMT_F16) go(norm_fwd<DMT_F16>);
  else go(norm_fwd<DMT_BF16>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" size_t dmt_layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || !fits(rows, cols)) return 0;
  return sizeof(float) * 2 * (size_t)slices_of(rows) * (size_t)cols;
}

template <int XD, int GD>
static void bwd_run(const void* x, int64_t rows, int64_t cols, int64_t xs, const void* gamma, int32_t wdt,
                    const float* mean, const float* rstd, const void* dy, int64_t dys, void* dx, int64_t dxs,
                    float* dgamma, float* dbeta, float* part, hipStream_t s) {
  const int64_t per = (rows + kSlices - 1) / kSlices, slices = rows ? (rows + per - 1) / per : 0;
  const unsigned cb = (unsigned)((cols + kBlock - 1) / kBlock);
  // (before dx, which may stand in dy's place)
  if (dgamma || dbeta) {
    if (rows)
      hipLaunchKernelGGL((norm_bwd_slices<XD, GD>), dim3(cb, (unsigned)slices), dim3(kBlock), 0, s, (const char*)x, rows,
                         (int)cols, xs, mean, rstd, (const char*)dy, dys, per, part);
    hipLaunchKernelGGL(norm_bwd_sum, dim3(cb), dim3(kBlock), 0, s, part, slices, (int)cols, dgamma, dbeta);
  }
  if (rows)
    hipLaunchKernelGGL((norm_bwd_rows<XD, GD>), dim3((unsigned)rows), dim3(kBlock), 0, s, (const char*)x, (int)cols, xs,
                       gamma, wdt, mean, rstd, (const char*)dy, dys, (char*)dx, dxs);
}

extern "C" dmt_status dmt_layer_norm_bwd(const void* x, int64_t rows, int64_t cols, int64_t x_stride,
                                         int32_t dtype, const void* gamma, int32_t weight_dtype,
                                         const float* mean, const float* rstd, const void* dy,
                                         int64_t dy_stride, int32_t grad_dtype, void* dx, int64_t dx_stride,
                                         float* dgamma, float* dbeta, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  if (rows < 0 || cols < 1 || x_stride < cols || dy_stride < cols || dx_stride < cols || !dmt_is_dtype(dtype))
    return DMT_EINVAL;
  if (grad_dtype != dtype && grad_dtype != DMT_F32) return DMT_EINVAL;
  if (gamma && weight_dtype != dtype && weight_dtype != DMT_F32) return DMT_EINVAL;
  if (!dmt_may_be_at(gamma, dmt_ebytes(weight_dtype)) || !dmt_may_be_at(dgamma, 4) || !dmt_may_be_at(dbeta, 4))
    return DMT_EINVAL;
  const int64_t ge = dmt_ebytes(grad_dtype);
  if (rows > 0 && (!dmt_is_at(x, dmt_ebytes(dtype)) || !dmt_is_at(dy, ge) || !dmt_is_at(dx, ge) || !dmt_is_at(mean, 4) ||
                   !dmt_is_at(rstd, 4)))
    return DMT_EINVAL;
  if (dx == dy && dx_stride != dy_stride && rows > 1) return DMT_EINVAL;
  if (!fits(rows, cols)) return DMT_ENOTSUP;
  if (dgamma || dbeta) {
    if (!dmt_is_at(workspace, 256)) return DMT_EINVAL;
    if (workspace_bytes < dmt_layer_norm_bwd_workspace_bytes(rows, cols)) return DMT_ENOMEM;
  }
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto run) {
    run(x, rows, cols, x_stride, gamma, weight_dtype, mean, rstd, dy, dy_stride, dx, dx_stride, dgamma, dbeta,
        (float*)workspace, s);
  };
  if (dtype == DMT_F32) go(bwd_run<DMT_F32, DMT_F32>);
  else if (dtype == DMT_F16 && grad_dtype == DMT_F16) go(bwd_run<DMT_F16, DMT_F16>);
  else if (dtype == DMT_F16) go(bwd_run<DMT_F16, DMT_F32>);
  else if (grad_dtype == DMT_BF16) go(bwd_run<DMT_BF16, DMT_BF16>);
  else go(bwd_run<DMT_BF16, DMT_F32>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
