// dmt_dropout_fwd, dmt_dropout_bwd:  y = residual + (x where bits >= m, else 0) * 65536 / (65536 - m),  16 bits an element from
// Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten rounds on a
// counter of four words give the bits of eight elements of a row.  The mask is a function of (seed, step, site, row, col / 8), so
// the backward makes it again and nothing is stored.
//
// A thread has eight elements (16 bytes of a 16-bit type); rows start a new counter, so an odd width leaves a part of its last eight
// unused.  Bound by memory: the generator is some 20 wide products and 60 plain instructions for eight elements.  262144 x 256 bfloat16
// with the residual 71 us, 5.7 TB/s; 65536 x 1024 without 46, x 1021 in rows of 1026 55; 65536 x 333 float32 38, 4.7 TB/s.
#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kGroup = 8;

struct Drop {
  const char *x, *residual;
  char* y;
  int64_t x_stride, r_stride, y_stride;
  const int64_t* rng;
  int64_t rows;
  int cols, groups;             // groups of eight in a row
  uint32_t least, site;         // smallest half-word that stays; site * 2^21
  float scale;
};

// Four words from a counter and a key.
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
    c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
    c[1] = (uint32_t)b;
    c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
}

template <int DT, bool Residual>
__global__ __launch_bounds__(kBlock) void dropout(const Drop a, unsigned first) {
  constexpr int EB = dmt::EltBytes<DT>::value;
  const uint64_t at = (uint64_t)(first + blockIdx.x) * kBlock;             // this block's first group
  const int64_t row0 = (int64_t)(at / (uint32_t)a.groups);
  const uint32_t local = (uint32_t)(at - (uint64_t)row0 * (uint32_t)a.groups) + threadIdx.x;
  const uint32_t down = local / (uint32_t)a.groups;
  const int64_t row = row0 + down;
  if (row >= a.rows) return;
  const int group = (int)(local - down * (uint32_t)a.groups), col = group * kGroup, valid = min(kGroup, a.cols - col);
  const auto x = dmt::load_raw<DT, kGroup>(a.x + (row * a.x_stride + col) * EB, valid);
  dmt::Raw<DT, kGroup> r;
  if constexpr (Residual) r = dmt::load_raw<DT, kGroup>(a.residual + (row * a.r_stride + col) * EB, valid);
  const uint64_t seed = (uint64_t)a.rng[0], step = (uint64_t)a.rng[1];
  uint32_t c[4] = {a.site | (uint32_t)group, (uint32_t)row, (uint32_t)step, (uint32_t)(step >> 32)};
  philox(c, (uint32_t)seed, (uint32_t)(seed >> 32));
  float v[kGroup], w[kGroup];
  dmt::unpack<DT, kGroup>(x, v);
  if constexpr (Residual) dmt::unpack<DT, kGroup>(r, w);
#pragma unroll
  for (int q = 0; q < kGroup; ++q) {
    const uint32_t bits = q % 2 ? c[q / 2] >> 16 : c[q / 2] & 0xffffu;
    const float kept = bits >= a.least ? v[q] * a.scale : 0.f;
    v[q] = Residual ? w[q] + kept : kept;
  }
  dmt::store_elems<DT, kGroup>(a.y + (row * a.y_stride + col) * EB, valid, v);
}

dmt_status run(const void* x, int64_t rows, int64_t cols, int64_t x_stride, int32_t dtype, const void* residual,
               int64_t residual_stride, float p, const int64_t* rng, int32_t site, void* y, int64_t y_stride, void* stream) {
  if (rows < 0 || cols < 1 || x_stride < cols || y_stride < cols || !dmt_is_dtype(dtype)) return DMT_EINVAL;
  if (residual && residual_stride < cols) return DMT_EINVAL;
  if (!(p >= 0.f && p <= 1.f) || site < 0 || site > 2047 || !dmt_is_at(rng, 8)) return DMT_EINVAL;
  const int64_t e = dmt_ebytes(dtype);
  if (rows > 0 && (!dmt_is_at(x, e) || !dmt_is_at(y, e) || !dmt_may_be_at(residual, e))) return DMT_EINVAL;
  if (rows > 1 && ((x == y && x_stride != y_stride) || (residual && residual == y && residual_stride != y_stride))) return DMT_EINVAL;
  if (rows >= 1ll << 31 || cols > 1 << 24) return DMT_ENOTSUP;
  if (rows == 0) return DMT_OK;
  Drop a = {};
  a.x = (const char*)x, a.residual = (const char*)residual, a.y = (char*)y;
  a.x_stride = x_stride, a.r_stride = residual_stride, a.y_stride = y_stride;
  a.rng = rng, a.rows = rows, a.cols = (int)cols, a.groups = (int)((cols + kGroup - 1) / kGroup);
  a.least = (uint32_t)((double)p * 65536.0 + 0.5), a.site = (uint32_t)site << 21;
  a.scale = a.least < 65536 ? 65536.f / (float)(65536 - a.least) : 0.f;
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto kernel) {
    dmt_launches((rows * a.groups + kBlock - 1) / kBlock, kBlock,
                 [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, a, first); });
  };
  if (dtype == DMT_F32) residual ? go(dropout<DMT_F32, true>) : go(dropout<DMT_F32, false>);
  else if (dtype == DMT_F16) residual ? go(dropout<DMT_F16, true>) : go(dropout<DMT_F16, false>);
  else residual ? go(dropout<DMT_BF16, true>) : go(dropout<DMT_BF16, false>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

}  // namespace

extern "C" dmt_status dmt_dropout_fwd(const void* x, int64_t rows, int64_t cols, int64_t x_stride, int32_t dtype,
                                      const void* residual, int64_t residual_stride, float p, const int64_t* rng,
                                      int32_t site, void* y, int64_t y_stride, void* stream) {
  return run(x, rows, cols, x_stride, dtype, residual, residual_stride, p, rng, site, y, y_stride, stream);
}

extern "C" dmt_status dmt_dropout_bwd(const void* dy, int64_t rows, int64_t cols, int64_t dy_stride, int32_t dtype, float p,
                                      const int64_t* rng, int32_t site, void* dx, int64_t dx_stride, void* stream) {
  return run(dy, rows, cols, dy_stride, dtype, nullptr, 0, p, rng, site, dx, dx_stride, stream);
}
