// dmt_layer_norm_fwd, dmt_layer_norm_bwd:  h = (x - mean) r,  r = (var + eps)^-1/2,  y = h gamma + beta;  with g = dy gamma:
//   dx = r (g - mean g - h mean(g h)),  dgamma = sum over rows of dy h,  dbeta = sum of dy.
//
// A row is held in registers by a group of T lanes, NV pieces of 16 bytes a lane, so x (and dy) cross the memory once and the
// variance is a second pass over registers, not a difference of large sums.  Both are bound by memory: 65536 x 1052 bfloat16
// forward 58.5 us, 4.7 TB/s; 8192 x 2048, bfloat16 with float32 gradients, backward 35 + 4.8 us, 4.8 TB/s.  The backward walks
// rows with the weights' gradients of its columns in registers; a block's go to a row of partial sums, which
// a second launch adds up in the blocks' order.  Rows longer than registers hold are read again from memory.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;

// Sum over the T lanes that share a row; T of 64 and less inside a wave, else over the block of T threads.  Successive sums of a
// block alternate between the halves of `smem` [2][N][T / 64], so one barrier each suffices.
template <int T, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* smem, int& half) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = dmt::group_sum<T < 64 ? T : 64>(v[i]);
  if constexpr (T > 64) {
    constexpr int NW = T / 64;
    float* at = smem + half * N * NW;
    half ^= 1;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) at[i * NW + (threadIdx.x >> 6)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) v[i] += at[i * NW + w];
    }
  }
}

// E weights from column c on, as far as there are any; of the rows' type or float32.
template <int XD, int E>
__device__ __forceinline__ void load_weights(const void* w, int dt, int c, int valid, float (&x)[E]) {
  if (dt == DMT_F32) dmt::load_elems<DMT_F32, E>((const char*)w + (int64_t)c * 4, valid, x);
  else dmt::load_elems<XD, E>((const char*)w + (int64_t)c * dmt::EltBytes<XD>::value, valid, x);
}

// ------------------------------------------------------------------ forward

struct Fwd {
  const char* x;
  int64_t rows, x_stride;
  const void *gamma, *beta;
  char* y;
  int64_t y_stride;
  float *mean, *rstd;
  int cols, wdt;
  float eps;
};

// Where a lane's piece v of a row lies.  The last piece of a row that is no whole number of pieces starts earlier, so that it
// ends with the row: its first `skip` elements are the piece before's too, they count once in sums and are stored by both, alike.  (Element by
// element, such a piece was a third of the instructions of a row of 1052.)  Rows shorter than a piece have `valid` elements.
template <int E, int T> struct Place {
  int c, skip, valid;
  bool there;
  __device__ __forceinline__ Place(int v, int lane, int cols) {
    const int at = (v * T + lane) * E;
    there = at < cols;
    c = max(0, min(at, cols - E));
    skip = at - c;
    valid = min(E, cols);
  }
  __device__ __forceinline__ bool whole() const { return skip == 0 && valid == E; }
  __device__ __forceinline__ bool counts(int q) const { return q >= skip && q < valid; }
};

template <int XD, int T, int NV>
__global__ __launch_bounds__(T < kBlock ? kBlock : T) void norm_fwd(const Fwd a) {
  constexpr int E = dmt::ChunkElems<XD>::value, XB = dmt::EltBytes<XD>::value, G = (T < kBlock ? kBlock : T) / T;
  __shared__ float sm[2 * (T > 64 ? T / 64 : 1)];
  int half = 0;
  const int lane = threadIdx.x % T;
  const int64_t step = (int64_t)gridDim.x * G;
  int64_t r = (int64_t)blockIdx.x * G + threadIdx.x / T;
  dmt::Raw<XD, E> raw[NV], next[NV];
  auto load = [&](int64_t row) {
    if (row >= a.rows) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (p.there) next[v] = dmt::load_raw<XD, E>(a.x + (row * a.x_stride + p.c) * XB, p.valid);
    }
  };
  load(r);
  float gamma[NV][E], beta[NV][E];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Place<E, T> p(v, lane, a.cols);
#pragma unroll
    for (int q = 0; q < E; ++q) gamma[v][q] = 1.f, beta[v][q] = 0.f;
    if (a.gamma && p.there) load_weights<XD, E>(a.gamma, a.wdt, p.c, p.valid, gamma[v]);
    if (a.beta && p.there) load_weights<XD, E>(a.beta, a.wdt, p.c, p.valid, beta[v]);
  }
  for (; r < a.rows; r += step) {                           // (T > 64: the whole block has the same r)
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = next[v];
    load(r + step);
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (!p.there) continue;
      float x[E];
      dmt::unpack<XD, E>(raw[v], x);
      if (p.whole()) {
#pragma unroll
        for (int q = 0; q < E; ++q) s[0] += x[q];
      } else {
#pragma unroll
        for (int q = 0; q < E; ++q) s[0] += p.counts(q) ? x[q] : 0.f;
      }
    }
    row_sums<T, 1>(s, sm, half);
    const float m = s[0] / (float)a.cols;
    s[0] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (!p.there) continue;
      float x[E];
      dmt::unpack<XD, E>(raw[v], x);
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] -= m;
      if (!p.whole()) {
#pragma unroll
        for (int q = 0; q < E; ++q) x[q] = p.counts(q) ? x[q] : 0.f;
      }
#pragma unroll
      for (int q = 0; q < E; ++q) s[0] = fmaf(x[q], x[q], s[0]);
    }
    row_sums<T, 1>(s, sm, half);
    const float rs = 1.f / sqrtf(s[0] / (float)a.cols + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (!p.there) continue;
      float x[E];
      dmt::unpack<XD, E>(raw[v], x);
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] = fmaf((x[q] - m) * rs, gamma[v][q], beta[v][q]);
      dmt::store_elems<XD, E>(a.y + (r * a.y_stride + p.c) * XB, p.valid, x);
    }
    if (lane == 0) {
      if (a.mean) a.mean[r] = m;
      if (a.rstd) a.rstd[r] = rs;
    }
  }
}

// Rows of any length, a block each, read three times.
template <int XD>
__global__ __launch_bounds__(1024) void norm_fwd_long(const Fwd a, unsigned first_block) {
  constexpr int E = dmt::ChunkElems<XD>::value, XB = dmt::EltBytes<XD>::value, B = 1024;
  __shared__ float sm[2 * B / 64];
  int half = 0;
  const int64_t r = first_block + blockIdx.x;
  const char* xr = a.x + r * a.x_stride * XB;
  float s[1] = {0.f}, x[E], w[E];
  for (int c = threadIdx.x * E; c < a.cols; c += B * E) {
    dmt::load_elems<XD, E>(xr + (int64_t)c * XB, a.cols - c, x);
#pragma unroll
    for (int q = 0; q < E; ++q) s[0] += x[q];
  }
  row_sums<B, 1>(s, sm, half);
  const float m = s[0] / (float)a.cols;
  s[0] = 0.f;
  for (int c = threadIdx.x * E; c < a.cols; c += B * E) {
    dmt::load_elems<XD, E>(xr + (int64_t)c * XB, a.cols - c, x);
#pragma unroll
    for (int q = 0; q < E; ++q) s[0] += c + q < a.cols ? (x[q] - m) * (x[q] - m) : 0.f;
  }
  row_sums<B, 1>(s, sm, half);
  const float rs = 1.f / sqrtf(s[0] / (float)a.cols + a.eps);
  for (int c = threadIdx.x * E; c < a.cols; c += B * E) {
    const int valid = a.cols - c;
    dmt::load_elems<XD, E>(xr + (int64_t)c * XB, valid, x);
#pragma unroll
    for (int q = 0; q < E; ++q) x[q] = (x[q] - m) * rs;
    if (a.gamma) {
      load_weights<XD, E>(a.gamma, a.wdt, c, valid, w);
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] *= w[q];
    }
    if (a.beta) {
      load_weights<XD, E>(a.beta, a.wdt, c, valid, w);
#pragma unroll
      for (int q = 0; q < E; ++q) x[q] += w[q];
    }
    dmt::store_elems<XD, E>(a.y + (r * a.y_stride + c) * XB, valid, x);
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[r] = m;
    if (a.rstd) a.rstd[r] = rs;
  }
}

// ------------------------------------------------------------------ backward

struct Bwd {
  const char* x;
  int64_t rows, x_stride;
  const void* gamma;
  const float *mean, *rstd;
  const char* dy;
  int64_t dy_stride;
  char* dx;
  int64_t dx_stride;
  float* part;                                              // [blocks][2][cols], null where no second launch adds them up
  int cols, wdt;
  unsigned row_blocks;                                      // blocks behind them are few_columns()
  float *dgamma, *dbeta;
};

// The weights' gradients of few rows: 64 columns a block, its threads by 16, of which every group walks its share of the rows.  Beside
// the rows' own blocks instead of a launch behind them, which reads x and dy twice.
template <int XD, int GD, int B> __device__ __forceinline__ void few_columns(const Bwd& a, unsigned block) {
  constexpr int XB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value, U = B < 1024 ? 8 : 4, G = B / 16;
  __shared__ float s_cols[B / 64][2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)block * 64 + (lane & 15) * 4, valid = min(4, a.cols - c);
  float dg[4] = {0.f, 0.f, 0.f, 0.f}, db[4] = {0.f, 0.f, 0.f, 0.f};
  if (valid > 0)
    for (int64_t r0 = threadIdx.x / 16; r0 < a.rows; r0 += G * U) {
      dmt::Raw<XD, 4> x[U];
      dmt::Raw<GD, 4> dy[U];
      float m[U], rs[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * G;
        if (r >= a.rows) break;
        x[u] = dmt::load_raw<XD, 4>(a.x + (r * a.x_stride + c) * XB, valid);
        dy[u] = dmt::load_raw<GD, 4>(a.dy + (r * a.dy_stride + c) * GB, valid);
        m[u] = a.mean[r], rs[u] = a.rstd[r];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (r0 + u * G >= a.rows) break;
        float h[4], d[4];
        dmt::unpack<XD, 4>(x[u], h);
        dmt::unpack<GD, 4>(dy[u], d);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < valid) dg[q] = fmaf(d[q], (h[q] - m[u]) * rs[u], dg[q]), db[q] += d[q];
      }
    }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    dg[q] += dmt::lane_xor<16>(dg[q]);
    db[q] += dmt::lane_xor<16>(db[q]);
    dg[q] += dmt::lane_xor<32>(dg[q]);
    db[q] += dmt::lane_xor<32>(db[q]);
    if (lane < 16) s_cols[wave][0][lane * 4 + q] = dg[q], s_cols[wave][1][lane * 4 + q] = db[q];
  }
  __syncthreads();
  if (wave < 2) {
    float* out = wave == 0 ? a.dgamma : a.dbeta;
    const int at = (int)block * 64 + lane;
    float s = 0.f;
    for (int w = 0; w < B / 64; ++w) s += s_cols[w][wave][lane];
    if (out && at < a.cols) out[at] = s;
  }
}

template <int XD, int GD, int T, int NV>
__global__ __launch_bounds__(T < kBlock ? kBlock : T) void norm_bwd(const Bwd a) {
  constexpr int E = dmt::ChunkElems<XD>::value, XB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  constexpr int B = T < kBlock ? kBlock : T, G = B / T;     // groups of a block
  __shared__ float sm[2 * 2 * (T > 64 ? T / 64 : 1)];
  __shared__ float s_acc[G > 1 ? G - 1 : 1][G > 1 ? T * E : 1];
  if (blockIdx.x >= a.row_blocks) {
    few_columns<XD, GD, B>(a, blockIdx.x - a.row_blocks);
    return;
  }
  int half = 0;
  const int lane = threadIdx.x % T, group = threadIdx.x / T;
  float gamma[NV][E], dg[NV][E], db[NV][E];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const Place<E, T> p(v, lane, a.cols);
#pragma unroll
    for (int q = 0; q < E; ++q) gamma[v][q] = 1.f, dg[v][q] = 0.f, db[v][q] = 0.f;
    if (a.gamma && p.there) load_weights<XD, E>(a.gamma, a.wdt, p.c, p.valid, gamma[v]);
  }
  const float over = 1.f / (float)a.cols;
  dmt::Raw<XD, E> x[NV], next_x[NV];
  dmt::Raw<GD, E> dy[NV], next_dy[NV];
  float next_m = 0.f, next_rs = 0.f;
  auto load = [&](int64_t r) {
    if (r >= a.rows) return;
    next_m = a.mean[r], next_rs = a.rstd[r];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (!p.there) continue;
      next_x[v] = dmt::load_raw<XD, E>(a.x + (r * a.x_stride + p.c) * XB, p.valid);
      next_dy[v] = dmt::load_raw<GD, E>(a.dy + (r * a.dy_stride + p.c) * GB, p.valid);
    }
  };
  const int64_t step = (int64_t)a.row_blocks * G;
  int64_t r = (int64_t)blockIdx.x * G + group;
  load(r);
  for (; r < a.rows; r += step) {                           // (T > 64: the whole block has the same r)
    const float m = next_m, rs = next_rs;
#pragma unroll
    for (int v = 0; v < NV; ++v) x[v] = next_x[v], dy[v] = next_dy[v];
    load(r + step);
    float sums[2] = {0.f, 0.f};                             // of g and of g h
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (!p.there) continue;
      float h[E], d[E];
      dmt::unpack<XD, E>(x[v], h);
      dmt::unpack<GD, E>(dy[v], d);
      if (!p.whole()) {
#pragma unroll
        for (int q = 0; q < E; ++q) d[q] = p.counts(q) ? d[q] : 0.f, h[q] = p.counts(q) ? h[q] : m;
      }
#pragma unroll
      for (int q = 0; q < E; ++q) {
        h[q] = (h[q] - m) * rs;
        const float g = d[q] * gamma[v][q];
        sums[0] += g;
        sums[1] = fmaf(g, h[q], sums[1]);
        dg[v][q] = fmaf(d[q], h[q], dg[v][q]);
        db[v][q] += d[q];
      }
    }
    row_sums<T, 2>(sums, sm, half);
    const float mg = sums[0] * over, mgh = sums[1] * over;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Place<E, T> p(v, lane, a.cols);
      if (!p.there) continue;
      float h[E], d[E];
      dmt::unpack<XD, E>(x[v], h);
      dmt::unpack<GD, E>(dy[v], d);
#pragma unroll
      for (int q = 0; q < E; ++q) {
        h[q] = (h[q] - m) * rs;
        d[q] = rs * (fmaf(d[q], gamma[v][q], -mg) - h[q] * mgh);
      }
      dmt::store_elems<GD, E>(a.dx + (r * a.dx_stride + p.c) * GB, p.valid, d);
    }
  }
  if (!a.part) return;
  // the block's groups, in order, then one row of partial sums
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float (&acc)[E] = k == 0 ? dg[v] : db[v];
      if constexpr (G > 1) {
        __syncthreads();
        if (group > 0)
#pragma unroll
          for (int q = 0; q < E; ++q) s_acc[group - 1][q * T + lane] = acc[q];
        __syncthreads();
        if (group == 0)
          for (int o = 0; o < G - 1; ++o)
#pragma unroll
            for (int q = 0; q < E; ++q) acc[q] += s_acc[o][q * T + lane];
      }
      const Place<E, T> p(v, lane, a.cols);
      if (group > 0 || !p.there) continue;
      if (p.whole()) {
        dmt::store_elems<DMT_F32, E>((char*)(part + k * a.cols + p.c), E, acc);
      } else {
#pragma unroll
        for (int q = 0; q < E; ++q)
          if (p.counts(q)) part[k * a.cols + p.c + q] = acc[q];
      }
    }
  }
}

// Rows of any length: the rows' part and, a slice of the rows a block, the columns'.
template <int XD, int GD>
__global__ __launch_bounds__(1024) void norm_bwd_long(const Bwd a, unsigned first_block) {
  constexpr int E = dmt::ChunkElems<XD>::value, XB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value, B = 1024;
  __shared__ float sm[2 * 2 * B / 64];
  int half = 0;
  const int64_t r = first_block + blockIdx.x;
  const float m = a.mean[r], rs = a.rstd[r];
  float sums[2] = {0.f, 0.f}, h[E], d[E], w[E];
  for (int turn = 0; turn < 2; ++turn) {
    for (int c = threadIdx.x * E; c < a.cols; c += B * E) {
      const int valid = a.cols - c;
      dmt::load_elems<XD, E>(a.x + (r * a.x_stride + c) * XB, valid, h);
      dmt::load_elems<GD, E>(a.dy + (r * a.dy_stride + c) * GB, valid, d);
#pragma unroll
      for (int q = 0; q < E; ++q) w[q] = 1.f;
      if (a.gamma) load_weights<XD, E>(a.gamma, a.wdt, c, valid, w);
#pragma unroll
      for (int q = 0; q < E; ++q) {
        h[q] = (h[q] - m) * rs;
        d[q] *= w[q];
        if (turn == 0) sums[0] += d[q], sums[1] = fmaf(d[q], h[q], sums[1]);
        else d[q] = rs * (d[q] - sums[0] - h[q] * sums[1]);
      }
      if (turn == 1) dmt::store_elems<GD, E>(a.dx + (r * a.dx_stride + c) * GB, valid, d);
    }
    if (turn == 0) {
      row_sums<B, 2>(sums, sm, half);
      sums[0] /= (float)a.cols;
      sums[1] /= (float)a.cols;
    }
  }
}
template <int XD, int GD>
__global__ __launch_bounds__(kBlock) void norm_bwd_slices(const Bwd a, int64_t per) {
  constexpr int XB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  const int c = blockIdx.x * kBlock + threadIdx.x;
  if (c >= a.cols) return;
  const int64_t r0 = blockIdx.y * per, r1 = min(a.rows, r0 + per);
  float dg = 0.f, db = 0.f;
  for (int64_t r = r0; r < r1; ++r) {
    const float d = dmt::load1<GD>(a.dy + (r * a.dy_stride + c) * GB);
    dg = fmaf(d, (dmt::load1<XD>(a.x + (r * a.x_stride + c) * XB) - a.mean[r]) * a.rstd[r], dg);
    db += d;
  }
  a.part[(int64_t)blockIdx.y * 2 * a.cols + c] = dg;
  a.part[((int64_t)blockIdx.y * 2 + 1) * a.cols + c] = db;
}

// The partial rows, added up in order: a block has 64 columns of one of the two gradients, its 16 waves a share of the rows each.
__global__ __launch_bounds__(1024) void norm_bwd_sum(const float* __restrict__ part, int64_t n, int cols,
                                                     float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float sm[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, k = blockIdx.y;
  float* out = k == 0 ? dgamma : dbeta;
  if (!out) return;
  const int64_t per = (n + 15) / 16, i0 = wave * per, i1 = min(n, i0 + per);
  float s = 0.f;
  if (c < cols)
    for (int64_t i = i0; i < i1; i += 8) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = i + u < i1 ? part[((i + u) * 2 + k) * cols + c] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
  sm[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) {
    for (int w = 1; w < 16; ++w) s += sm[w][lane];
    out[c] = s;
  }
}

// ------------------------------------------------------------------ how a call is divided

// Lanes of a row and pieces of a lane, from the pieces of E elements of x a row has; run(T, NV) as types.  False: longer than the
// 128 registers of a thread of 1024 hold beside the weights (16384 columns; backward 8192).  Lanes that a row leaves idle cost as the
// others do: 262144 x 200 bfloat16 with 32 lanes a row 45 us, with 64 87; 229385 x 16, backward, with 8 lanes 21.8, with 16 30.
template <int V> struct Int { static constexpr int value = V; };
template <int E, typename Run> bool fwd_shape(int64_t pieces, Run run) {
  if (pieces <= 8) run(Int<8>(), Int<1>());
  else if (pieces <= 16) run(Int<16>(), Int<1>());
  else if (pieces <= 32) run(Int<32>(), Int<1>());
  else if (pieces <= 64) run(Int<64>(), Int<1>());
  else if (pieces <= 128) run(Int<64>(), Int<2>());
  else if (pieces <= 192) run(Int<64>(), Int<3>());
  else if (pieces <= 256) run(Int<64>(), Int<4>());
  else if (pieces <= 512) run(Int<256>(), Int<2>());
  else if (pieces <= 1024) run(Int<256>(), Int<4>());
  else if (pieces <= 2048) run(Int<1024>(), Int<2>());
  else if constexpr (E == 4) {
    if (pieces > 4096) return false;
    run(Int<1024>(), Int<4>());
  }
  else return false;
  return true;
}
template <int E, typename Run> bool bwd_shape(int64_t pieces, Run run) {
  if (pieces <= 8) run(Int<8>(), Int<1>());
  else if (pieces <= 16) run(Int<16>(), Int<1>());
  else if (pieces <= 32) run(Int<32>(), Int<1>());
  else if (pieces <= 64) run(Int<64>(), Int<1>());
  else if (pieces <= 128) run(Int<64>(), Int<2>());
  else if (pieces <= 256) run(Int<256>(), Int<1>());
  else if (pieces <= 512) run(Int<256>(), Int<2>());
  else if (pieces <= 1024) run(Int<1024>(), Int<1>());
  else if constexpr (E == 4) {
    if (pieces > 2048) return false;
    run(Int<1024>(), Int<2>());
  }
  else return false;
  return true;
}
// Blocks, at most; each walks rows with the weights in registers and the next row requested.  Forward, 65536 x 1052: 58.6 us with
// 1024, 85.8 with a block per four rows; 262144 x 128 (16 rows a block): 25.8 with 2048, 27.8 with 1024.  Backward: a row of
// partial sums a block, 8192 x 2048 35.4 + 4.3 us with 512, 34.7 + 6.8 with 1024; 8192 x 8192 (blocks of 1024 threads) 77.7 + 4.8 with
// 256, 82 + 6.6 with 512.
constexpr int64_t kBwdBlocks = 512;
constexpr int64_t fwd_blocks(int T) { return T <= 16 ? 2048 : 1024; }
constexpr int64_t bwd_blocks(int T) { return T >= 1024 ? 256 : kBwdBlocks; }
constexpr int64_t kSlices = 128;
// Rows up to which the weights' gradients are few_columns(): the whole call 9.0 us for 11.8 at 512 x 1024, 10.2 for 11.9 at 512 x 200, 17.8 for 11.9
// at 1000 x 200.
constexpr int64_t kFewRows = 512;

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
  Fwd a = {};
  a.x = (const char*)x, a.rows = rows, a.x_stride = x_stride, a.gamma = gamma, a.beta = beta;
  a.y = (char*)y, a.y_stride = y_stride, a.mean = mean, a.rstd = rstd, a.cols = (int)cols, a.wdt = weight_dtype, a.eps = eps;
  auto go = [&](auto xd) {
    constexpr int XD = decltype(xd)::value;
    const int64_t pieces = (cols + dmt::ChunkElems<XD>::value - 1) / dmt::ChunkElems<XD>::value;
    const bool done = fwd_shape<dmt::ChunkElems<XD>::value>(pieces, [&](auto t, auto nv) {
      constexpr int T = decltype(t)::value, B = T < kBlock ? kBlock : T;
      const int64_t blocks = std::min((rows + B / T - 1) / (B / T), fwd_blocks(T));
      hipLaunchKernelGGL((norm_fwd<XD, T, decltype(nv)::value>), dim3((unsigned)blocks), dim3(B), 0, s, a);
    });
    if (!done)
      dmt_launches(rows, 1024, [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(norm_fwd_long<XD>, grid, dim3(1024), 0, s, a, first); });
  };
  if (dtype == DMT_F32) go(Int<DMT_F32>());
  else if (dtype == DMT_F16) go(Int<DMT_F16>());
  else go(Int<DMT_BF16>());
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" size_t dmt_layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || !fits(rows, cols)) return 0;
  return sizeof(float) * 2 * (size_t)std::min(rows, kBwdBlocks) * (size_t)cols;
}

template <int XD, int GD>
static void bwd_run(Bwd a, hipStream_t s) {
  const int64_t pieces = (a.cols + dmt::ChunkElems<XD>::value - 1) / dmt::ChunkElems<XD>::value;
  int64_t parts = 0;
  bool sum = a.dgamma || a.dbeta;                           // whether partial sums are added up (no rows: none are, into zeros)
  const bool done = bwd_shape<dmt::ChunkElems<XD>::value>(pieces, [&](auto t, auto nv) {
    constexpr int T = decltype(t)::value, B = T < kBlock ? kBlock : T;
    parts = std::min((a.rows + B / T - 1) / (B / T), bwd_blocks(T));
    auto launch = [&](unsigned rows, unsigned columns) {
      a.row_blocks = rows;
      if (rows + columns > 0) hipLaunchKernelGGL((norm_bwd<XD, GD, T, decltype(nv)::value>), dim3(rows + columns), dim3(B), 0, s, a);
    };
    const unsigned columns = a.rows <= kFewRows && sum ? (unsigned)((a.cols + 63) / 64) : 0u;
    if (columns > 0) a.part = nullptr, sum = false;
    const bool ahead = (const char*)a.dx == a.dy || (const char*)a.dx == a.x;      // dx in the place of what the columns read
    if (columns > 0 && ahead) launch(0, columns);
    launch((unsigned)parts, ahead ? 0 : columns);
  });
  if (!done && a.rows > 0) {
    const int64_t per = (a.rows + kSlices - 1) / kSlices;
    parts = (a.rows + per - 1) / per;
    // (before dx, which may stand in dy's place)
    if (sum)
      hipLaunchKernelGGL((norm_bwd_slices<XD, GD>), dim3((unsigned)((a.cols + kBlock - 1) / kBlock), (unsigned)parts), dim3(kBlock), 0,
                         s, a, per);
    dmt_launches(a.rows, 1024,
                 [&](unsigned first, dim3 grid) { hipLaunchKernelGGL((norm_bwd_long<XD, GD>), grid, dim3(1024), 0, s, a, first); });
  }
  if (sum)
    hipLaunchKernelGGL(norm_bwd_sum, dim3((unsigned)((a.cols + 63) / 64), 2), dim3(1024), 0, s, a.part, parts, a.cols, a.dgamma, a.dbeta);
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
    const size_t need = dmt_layer_norm_bwd_workspace_bytes(rows, cols);      // (0: none, of no rows)
    if (need > 0 && !dmt_is_at(workspace, 256)) return DMT_EINVAL;
    if (workspace_bytes < need) return DMT_ENOMEM;
  }
  hipStream_t s = (hipStream_t)stream;
  Bwd a = {};
  a.x = (const char*)x, a.rows = rows, a.x_stride = x_stride, a.gamma = gamma, a.mean = mean, a.rstd = rstd;
  a.dy = (const char*)dy, a.dy_stride = dy_stride, a.dx = (char*)dx, a.dx_stride = dx_stride;
  a.part = dgamma || dbeta ? (float*)workspace : nullptr, a.dgamma = dgamma, a.dbeta = dbeta, a.cols = (int)cols, a.wdt = weight_dtype;
  if (dtype == DMT_F32) bwd_run<DMT_F32, DMT_F32>(a, s);
  else if (dtype == DMT_F16 && grad_dtype == DMT_F16) bwd_run<DMT_F16, DMT_F16>(a, s);
  else if (dtype == DMT_F16) bwd_run<DMT_F16, DMT_F32>(a, s);
  else if (grad_dtype == DMT_BF16) bwd_run<DMT_BF16, DMT_BF16>(a, s);
  else bwd_run<DMT_BF16, DMT_F32>(a, s);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
