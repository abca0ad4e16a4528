// dmt_gated_scan_fwd, dmt_gated_scan_bwd, dmt_gated_scan_step, dmt_sequence_rows:  h_t = f_t h_{t-1} + u_t,  f = sigmoid(gate),
// u = (1 - f) value or value; and backwards  l_t = dh_t + m_{t+1},  m_t = f_t l_t,  dvalue = l (1 - f),  dgate = l (h_{t-1} - value) f (1 - f).
//
// Both are first-order recurrences, so a stretch of rows maps the state before it to the one behind it by h -> A h + S, with A the
// product of its f; a stretch that holds a sequence's first row (backwards: its last) forgets what came before.  Rows are cut
// into chunks, a block's each (for the channels of a group of lanes), and chunks into the stretches of `walkers`: lane
// groups that go through their rows one after another, 16 at a time.  Where sequences are as long as stretches, or
// so many that a walker can have whole ones, nothing else is needed.  Otherwise a first launch takes every stretch's (A, S), reading only
// the rows that matter to the next one (behind its last first row), and the second starts each walker from what those before
// it lead to.  One chunk does both in one launch.
//
// The backward needs h_{t-1}: the forward keeps the state in front of every 16th row in float32, from which a walker goes through
// its 16 rows again, so neither h nor a rounded h is read.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 512, kTile = 16;

// How rows are cut.
struct Cut {
  int group;           // lanes of a walker: 16, 32 or 64
  int tiles;           // groups' widths of channels
  int64_t sub;         // rows of a walker, a multiple of 16 unless `whole`
  int64_t chunk;       // rows of a chunk
  int64_t chunks;
  bool whole;          // every walker starts with a sequence's first row
  bool one;            // no state passes between chunks
};

struct Scan {
  const char *gate, *value, *dh;
  char *h, *dgate, *dvalue;
  int64_t gate_stride, value_stride, h_stride, dh_stride, dgate_stride, dvalue_stride, rows;
  const int32_t* seq;
  const float *initial, *dfinal;
  float *final, *dinitial, *kept;
  float2 *stretch, *chunk;         // (A, S) [chunks * walkers][cols], [chunks][cols]; A = -1: forgets what came before
  int* forgets;                    // [chunks]
  unsigned long long* first_bad;
  int sequences, length, cols, tiles;
  bool free, whole;
  int64_t sub, chunk_rows, chunks;
};

template <int G> __device__ __forceinline__ int uniform(int v) {
  if constexpr (G == 64) return __builtin_amdgcn_readfirstlane(v);
  else return v;
}

// First row of walker w of a chunk (of the chunk's end, for the walkers' number).
template <int G> __device__ __forceinline__ int begin_of(const Scan& a, int64_t chunk, int w) {
  const int64_t c0 = chunk * a.chunk_rows, c1 = min(c0 + a.chunk_rows, a.rows);
  if (w == 0) return (int)c0;
  if (w == kBlock / G) return (int)c1;
  const int64_t at = c0 + w * a.sub;
  return (int)min(c1, a.whole ? at : at & ~(int64_t)(kTile - 1));
}

__device__ __forceinline__ int id_of(const Scan& a, int row) {
  const int id = a.seq[row];
  return (uint32_t)id < (uint32_t)a.sequences ? id : -1;
}
__device__ __forceinline__ int sequence_of(const Scan& a, int row) { return a.seq ? id_of(a, row) : row / a.length; }

// Bits of the 16 rows from r0 on that lie in [lo, hi): whether a row is of a sequence, is its first, its last.
struct Bits { uint32_t there, first, last; };

template <int G, bool Report = false>
__device__ __forceinline__ Bits bits_of(const Scan& a, int r0, int lo, int hi) {
  const int lane = threadIdx.x & 63, row = r0 + (lane & 15);
  bool there = row >= lo && row < hi, first = false, last = false;
  if (there) {
    if (a.seq) {
      const int raw = a.seq[row], id = (uint32_t)raw < (uint32_t)a.sequences ? raw : -1;
      if (Report && raw >= a.sequences && a.first_bad) atomicMin(a.first_bad, (unsigned long long)row);
      there = id >= 0;
      first = there && (row == 0 || id_of(a, row - 1) != id);
      last = there && (row + 1 == (int)a.rows || id_of(a, row + 1) != id);
    } else {
      const int at = row % a.length;
      first = at == 0;
      last = at == a.length - 1;
    }
  }
  const int shift = G == 64 ? 0 : lane & 48;
  Bits b;
  b.there = (uint32_t)(__ballot(there) >> shift) & 0xffffu;
  b.first = (uint32_t)(__ballot(first) >> shift) & 0xffffu;
  b.last = (uint32_t)(__ballot(last) >> shift) & 0xffffu;
  return b;
}

// Channels of a lane: 4 bytes of the rows' type.
template <int XD> struct Width { static constexpr int value = XD == DMT_F32 ? 1 : 2; };

// V elements of type D in as few words; of a single column only the first is there.
template <int D, int V> struct Word { uint32_t w[V * dmt::EltBytes<D>::value / 4 > 0 ? V * dmt::EltBytes<D>::value / 4 : 1]; };

template <int D, int V> __device__ __forceinline__ Word<D, V> load_word(const char* p, bool both) {
  typedef uint32_t __attribute__((aligned(2))) u32;
  Word<D, V> r;
  if constexpr (D == DMT_F32) {
    r.w[0] = *(const DMT_GLOBAL uint32_t*)p;
    if constexpr (V == 2) r.w[1] = both ? *(const DMT_GLOBAL uint32_t*)(p + 4) : 0u;
  } else {
    r.w[0] = both ? *(const DMT_GLOBAL u32*)p : (uint32_t) * (const DMT_GLOBAL uint16_t*)p;
  }
  return r;
}
template <int D, int V> __device__ __forceinline__ void unpack_word(const Word<D, V>& r, float (&x)[V]) {
  if constexpr (D == DMT_F32) {
#pragma unroll
    for (int q = 0; q < V; ++q) x[q] = __uint_as_float(r.w[q]);
  } else {
    dmt::unpack2<D>(r.w[0], x[0], x[1]);
  }
}
template <int D, int V> __device__ __forceinline__ void store_word(char* p, const float (&x)[V], bool both) {
  typedef uint32_t __attribute__((aligned(2))) u32;
  if constexpr (D == DMT_F32) {
    *(DMT_GLOBAL float*)p = x[0];
    if constexpr (V == 2) {
      if (both) *(DMT_GLOBAL float*)(p + 4) = x[1];
    }
  } else {
    const uint32_t w = dmt::round2<D>(x[0], x[1]);
    if (both) *(DMT_GLOBAL u32*)p = w;
    else *(DMT_GLOBAL uint16_t*)p = (uint16_t)w;
  }
}

// f = sigmoid(x) and 1 - f, each to a few units of its last place: e = exp(-|x|) by 2^t with t's rounding put back, then 1 / (1 + e).
__device__ __forceinline__ void sigmoids(float x, float& f, float& rest) {
  float z = -fabsf(x);
  z = z < -100.f ? -100.f : z;                              // (keeps a NaN)
  const float t = z * 1.44269504088896341f;
  const float lo = fmaf(z, 1.44269504088896341f, -t) + z * 1.92596299e-8f;
  const float p = __builtin_amdgcn_exp2f(t);
  const float e = fmaf(p, lo * 0.693147180559945309f, p);
  const float r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;
  f = x >= 0.f ? r : er;
  rest = x >= 0.f ? er : r;
}

struct Map { float a, s; };
__device__ __forceinline__ Map after(Map l, Map r) {         // l, then r
  if (r.a < 0.f) return r;
  return {l.a < 0.f ? -1.f : l.a * r.a, fmaf(r.a, l.s, r.s)};
}
__device__ __forceinline__ float applied(Map m, float h) { return m.a < 0.f ? m.s : fmaf(m.a, h, m.s); }

// What a lane knows about its channels.
template <int G, int XD> struct Lane {
  static constexpr int V = Width<XD>::value;
  int w, at, c;            // walker, lane of it, first channel
  bool on, both;
  __device__ __forceinline__ Lane(int tile, int cols) {
    w = uniform<G>(threadIdx.x / G);
    at = threadIdx.x % G;
    const int c0 = (tile * G + at) * V;
    on = c0 < cols;
    c = max(0, min(c0, cols - V));        // the last pair of an odd width holds the channel before too: both lanes find the same
    both = cols >= V;
  }
};

// ---- what a stretch makes of the state before it

template <int G, int XD, int V>
__device__ __forceinline__ void stretch_fwd(const Scan& a, const Lane<G, XD>& l, int lo, int hi, Map (&m)[V]) {
  constexpr int EB = dmt::EltBytes<XD>::value;
#pragma unroll
  for (int q = 0; q < V; ++q) m[q] = {1.f, 0.f};
  if (lo >= hi) return;
  bool needed = hi < (int)a.rows;                                 // by the row behind
  if (needed) needed = a.seq ? id_of(a, hi) >= 0 && id_of(a, hi) == id_of(a, hi - 1) : hi % a.length != 0;
  if (!needed) {
#pragma unroll
    for (int q = 0; q < V; ++q) m[q] = {-1.f, 0.f};
    return;
  }
  int from = lo;
  if (!a.seq) {
    const int begin = hi - 1 - (hi - 1) % a.length;
    from = max(lo, begin);
    if (begin >= lo) {
#pragma unroll
      for (int q = 0; q < V; ++q) m[q] = {-1.f, 0.f};
    }
  } else {
    for (int r0 = (hi - 1) & ~(kTile - 1); r0 + kTile > lo; r0 -= kTile) {
      const uint32_t first = bits_of<G>(a, r0, lo, hi).first;
      if (first) {
        from = r0 + 31 - __builtin_clz(first);
#pragma unroll
        for (int q = 0; q < V; ++q) m[q] = {-1.f, 0.f};
        break;
      }
    }
  }
  if (m[0].a < 0.f && a.initial) {
    const float* at = a.initial + (int64_t)sequence_of(a, from) * a.cols + l.c;
#pragma unroll
    for (int q = 0; q < V; ++q) m[q].s = q == 0 || l.both ? at[q] : 0.f;
  }
  if (!l.on) return;
  const char *gp = a.gate + ((int64_t)from * a.gate_stride + l.c) * EB, *vp = a.value + ((int64_t)from * a.value_stride + l.c) * EB;
  const int64_t gs = a.gate_stride * EB, vs = a.value_stride * EB;
  for (int r0 = from; r0 < hi; r0 += kTile) {
    Word<XD, V> g[kTile], v[kTile];
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      const int j = min(i, hi - 1 - r0);
      g[i] = load_word<XD, V>(gp + j * gs, l.both);
      v[i] = load_word<XD, V>(vp + j * vs, l.both);
    }
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      if (r0 + i >= hi) continue;
      float x[V], u[V];
      unpack_word<XD, V>(g[i], x);
      unpack_word<XD, V>(v[i], u);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float f, rest;
        sigmoids(x[q], f, rest);
        m[q].s = fmaf(f, m[q].s, a.free ? u[q] : rest * u[q]);
        m[q].a = m[q].a < 0.f ? -1.f : m[q].a * f;
      }
    }
    gp += kTile * gs;
    vp += kTile * vs;
  }
}

template <int G, int XD, int GD, int V>
__device__ __forceinline__ void stretch_bwd(const Scan& a, const Lane<G, XD>& l, int lo, int hi, Map (&m)[V]) {
  constexpr int EB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
#pragma unroll
  for (int q = 0; q < V; ++q) m[q] = {1.f, 0.f};
  if (lo >= hi) return;
  bool needed = lo > 0;                                           // by the row before
  if (needed) needed = a.seq ? id_of(a, lo) >= 0 && id_of(a, lo) == id_of(a, lo - 1) : lo % a.length != 0;
  if (!needed) {
#pragma unroll
    for (int q = 0; q < V; ++q) m[q] = {-1.f, 0.f};
    return;
  }
  int to = hi - 1;
  bool ends = false;
  if (!a.seq) {
    const int last = lo - lo % a.length + a.length - 1;
    ends = last < hi;
    to = min(last, hi - 1);
  } else {
    for (int r0 = lo & ~(kTile - 1); r0 < hi; r0 += kTile) {
      const uint32_t last = bits_of<G>(a, r0, lo, hi).last;
      if (last) {
        to = r0 + __builtin_ctz(last);
        ends = true;
        break;
      }
    }
  }
  if (ends) {
    const float* at = a.dfinal ? a.dfinal + (int64_t)sequence_of(a, to) * a.cols + l.c : nullptr;
#pragma unroll
    for (int q = 0; q < V; ++q) m[q] = {-1.f, at && (q == 0 || l.both) ? at[q] : 0.f};
  }
  if (!l.on) return;
  const char *gp = a.gate + ((int64_t)to * a.gate_stride + l.c) * EB, *dp = a.dh + ((int64_t)to * a.dh_stride + l.c) * GB;
  const int64_t gs = a.gate_stride * EB, ds = a.dh_stride * GB;
  for (int r0 = to; r0 >= lo; r0 -= kTile) {
    Word<XD, V> g[kTile];
    Word<GD, V> d[kTile];
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      const int j = min(i, r0 - lo);
      g[i] = load_word<XD, V>(gp - j * gs, l.both);
      d[i] = load_word<GD, V>(dp - j * ds, l.both);
    }
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      if (r0 - i < lo) continue;
      float x[V], y[V];
      unpack_word<XD, V>(g[i], x);
      unpack_word<GD, V>(d[i], y);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float f, rest;
        sigmoids(x[q], f, rest);
        m[q].s = f * (y[q] + m[q].s);
        m[q].a = m[q].a < 0.f ? -1.f : m[q].a * f;
      }
    }
    gp -= kTile * gs;
    dp -= kTile * ds;
  }
}

template <int G, int XD, int GD, bool Back, int V>
__device__ __forceinline__ void stretch_of(const Scan& a, const Lane<G, XD>& l, int lo, int hi, Map (&m)[V]) {
  if constexpr (Back) stretch_bwd<G, XD, GD, V>(a, l, lo, hi, m);
  else stretch_fwd<G, XD, V>(a, l, lo, hi, m);
}

template <int G, int XD, int GD, bool Back> __global__ __launch_bounds__(kBlock) void scan_stretches(const Scan a, unsigned first) {
  constexpr int V = Width<XD>::value, W = kBlock / G;
  __shared__ Map maps[W][G * V];
  const uint32_t at = first + blockIdx.x;
  const int64_t chunk = at / (uint32_t)a.tiles;
  const Lane<G, XD> l((int)(at % (uint32_t)a.tiles), a.cols);
  Map m[V];
  stretch_of<G, XD, GD, Back, V>(a, l, begin_of<G>(a, chunk, l.w), begin_of<G>(a, chunk, l.w + 1), m);
#pragma unroll
  for (int q = 0; q < V; ++q) maps[l.w][l.at * V + q] = m[q];
  const int forgets = __syncthreads_or(m[0].a < 0.f);
  if (l.on)
#pragma unroll
    for (int q = 0; q < V; ++q)
      if (q == 0 || l.both) a.stretch[(chunk * W + l.w) * a.cols + l.c + q] = make_float2(m[q].a, m[q].s);
  if (l.w == 0 && l.on) {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      Map all = {1.f, 0.f};
      for (int w = 0; w < W; ++w) all = after(all, maps[Back ? W - 1 - w : w][l.at * V + q]);
      if (q == 0 || l.both) a.chunk[chunk * a.cols + l.c + q] = make_float2(all.a, all.s);
    }
  }
  if (threadIdx.x == 0 && at % (uint32_t)a.tiles == 0) a.forgets[chunk] = forgets;
}

// The state in front of (behind) a walker's rows: from all chunks since the last one that forgets, then the chunk's walkers.
template <int G, int XD, int GD, bool Back, bool One, int V>
__device__ __forceinline__ void state_before(const Scan& a, const Lane<G, XD>& l, int64_t chunk, int lo, int hi, float (&h)[V]) {
  constexpr int W = kBlock / G;
  __shared__ Map maps[2][W][G * V];
  __shared__ int nearest;
#pragma unroll
  for (int q = 0; q < V; ++q) h[q] = 0.f;
  if constexpr (One) {
    if (a.whole) return;
    Map m[V];
    stretch_of<G, XD, GD, Back, V>(a, l, lo, hi, m);
#pragma unroll
    for (int q = 0; q < V; ++q) maps[0][l.w][l.at * V + q] = m[q];
    __syncthreads();
  } else {
    // chunks between the nearest that forgets (it too) and this one; counted from here on, backwards or forwards
    const int64_t before = Back ? a.chunks - 1 - chunk : chunk;
    int64_t many = before;
    for (int64_t base = 0; base < before; base += kBlock) {
      if (threadIdx.x == 0) nearest = kBlock;
      __syncthreads();
      const int64_t i = base + threadIdx.x;
      if (i < before && a.forgets[Back ? chunk + 1 + i : chunk - 1 - i]) atomicMin(&nearest, (int)threadIdx.x);
      __syncthreads();
      const int n = nearest;
      __syncthreads();
      if (n < kBlock) {
        many = base + n + 1;
        break;
      }
    }
    // farthest first, a share a walker
    const int64_t share = (many + W - 1) / W, from = min(many, l.w * share), to = min(many, from + share);
    Map m[V];
#pragma unroll
    for (int q = 0; q < V; ++q) m[q] = {1.f, 0.f};
#pragma unroll 4
    for (int64_t i = from; i < to; ++i) {
      const int64_t c = Back ? chunk + many - i : chunk - many + i;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float2 x = a.chunk[c * a.cols + l.c + (l.both ? q : 0)];
        m[q] = after(m[q], {x.x, x.y});
      }
    }
#pragma unroll
    for (int q = 0; q < V; ++q) {
      maps[1][l.w][l.at * V + q] = m[q];
      const float2 x = a.stretch[(chunk * W + l.w) * a.cols + l.c + (l.both ? q : 0)];
      maps[0][l.w][l.at * V + q] = {x.x, x.y};
    }
    __syncthreads();
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int q = 0; q < V; ++q) h[q] = applied(maps[1][w][l.at * V + q], h[q]);
  }
  if constexpr (Back) {
    for (int w = W - 1; w > l.w; --w)
#pragma unroll
      for (int q = 0; q < V; ++q) h[q] = applied(maps[0][w][l.at * V + q], h[q]);
  } else {
    for (int w = 0; w < l.w; ++w)
#pragma unroll
      for (int q = 0; q < V; ++q) h[q] = applied(maps[0][w][l.at * V + q], h[q]);
  }
}

// ---- the rows

// Row i of a tile, or a row of the walker's own for rows that are not there (read and not used).
__device__ __forceinline__ int64_t row_at(const Bits& b, int i, int r0, int lo) { return b.there >> i & 1 ? r0 + i : lo; }

template <int G, int XD, bool One> __global__ __launch_bounds__(kBlock) void scan_fwd(const Scan a, unsigned first) {
  constexpr int V = Width<XD>::value, EB = dmt::EltBytes<XD>::value;
  const uint32_t at = first + blockIdx.x;
  const int64_t chunk = a.chunks - 1 - at / (uint32_t)a.tiles;    // what was read last comes first
  const Lane<G, XD> l((int)(at % (uint32_t)a.tiles), a.cols);
  const int lo = begin_of<G>(a, chunk, l.w), hi = begin_of<G>(a, chunk, l.w + 1);
  float h[V];
  state_before<G, XD, XD, false, One, V>(a, l, chunk, lo, hi, h);
  const char *gate = a.gate + (int64_t)l.c * EB, *value = a.value + (int64_t)l.c * EB;
  char* out = a.h + (int64_t)l.c * EB;
  for (int r0 = lo & ~(kTile - 1); r0 < hi && lo < hi; r0 += kTile) {
    const Bits b = at % (uint32_t)a.tiles == 0 ? bits_of<G, true>(a, r0, lo, hi) : bits_of<G>(a, r0, lo, hi);
    if (!l.on) continue;
    Word<XD, V> g[kTile], v[kTile];
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      const int64_t r = row_at(b, i, r0, lo);
      g[i] = load_word<XD, V>(gate + r * a.gate_stride * EB, l.both);
      v[i] = load_word<XD, V>(value + r * a.value_stride * EB, l.both);
    }
    if (a.kept && r0 >= lo)
#pragma unroll
      for (int q = 0; q < V; ++q)
        if (q == 0 || l.both) a.kept[(int64_t)(r0 / kTile) * a.cols + l.c + q] = h[q];
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      const int r = r0 + i;
      if (r < lo || r >= hi) continue;
      float y[V] = {};
      if (b.there >> i & 1) {
        if (b.first >> i & 1) {
          const float* from = a.initial ? a.initial + (int64_t)sequence_of(a, r) * a.cols + l.c : nullptr;
#pragma unroll
          for (int q = 0; q < V; ++q) h[q] = from && (q == 0 || l.both) ? from[q] : 0.f;
        }
        float x[V], u[V];
        unpack_word<XD, V>(g[i], x);
        unpack_word<XD, V>(v[i], u);
#pragma unroll
        for (int q = 0; q < V; ++q) {
          float f, rest;
          sigmoids(x[q], f, rest);
          y[q] = h[q] = fmaf(f, h[q], a.free ? u[q] : rest * u[q]);
        }
        if ((b.last >> i & 1) && a.final) {
          float* to = a.final + (int64_t)sequence_of(a, r) * a.cols + l.c;
#pragma unroll
          for (int q = 0; q < V; ++q)
            if (q == 0 || l.both) to[q] = h[q];
        }
      }
      store_word<XD, V>(out + (int64_t)r * a.h_stride * EB, y, l.both);
    }
  }
}

template <int G, int XD, int GD, bool One> __global__ __launch_bounds__(kBlock) void scan_bwd(const Scan a, unsigned first) {
  constexpr int V = Width<XD>::value, EB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  const uint32_t at = first + blockIdx.x;
  const int64_t chunk = a.chunks - 1 - at / (uint32_t)a.tiles;
  const Lane<G, XD> l((int)(at % (uint32_t)a.tiles), a.cols);
  const int lo = begin_of<G>(a, chunk, l.w), hi = begin_of<G>(a, chunk, l.w + 1);
  float m[V];
  state_before<G, XD, GD, true, One, V>(a, l, chunk, lo, hi, m);
  const char *gate = a.gate + (int64_t)l.c * EB, *value = a.value + (int64_t)l.c * EB, *dh = a.dh + (int64_t)l.c * GB;
  char *dgate = a.dgate + (int64_t)l.c * GB, *dvalue = a.dvalue + (int64_t)l.c * GB;
  for (int r0 = (hi - 1) & ~(kTile - 1); r0 + kTile > lo && lo < hi; r0 -= kTile) {
    const Bits b = bits_of<G>(a, r0, lo, hi);
    if (!l.on) continue;
    Word<XD, V> g[kTile], v[kTile];
    Word<GD, V> d[kTile];
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      const int64_t r = row_at(b, i, r0, lo);
      g[i] = load_word<XD, V>(gate + r * a.gate_stride * EB, l.both);
      v[i] = load_word<XD, V>(value + r * a.value_stride * EB, l.both);
      d[i] = load_word<GD, V>(dh + r * a.dh_stride * GB, l.both);
    }
    float h[V] = {};
    if (r0 >= lo)
#pragma unroll
      for (int q = 0; q < V; ++q) h[q] = a.kept[(int64_t)(r0 / kTile) * a.cols + l.c + (l.both ? q : 0)];
    // f, 1 - f (free: 1) and (h_{t-1} - value) f (1 - f) of the 16 rows
    float f[kTile][V], share[kTile][V], slope[kTile][V];
#pragma unroll
    for (int i = 0; i < kTile; ++i) {
      if (b.first >> i & 1) {
        const float* from = a.initial ? a.initial + (int64_t)sequence_of(a, r0 + i) * a.cols + l.c : nullptr;
#pragma unroll
        for (int q = 0; q < V; ++q) h[q] = from && (q == 0 || l.both) ? from[q] : 0.f;
      }
      float x[V], u[V];
      unpack_word<XD, V>(g[i], x);
      unpack_word<XD, V>(v[i], u);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float rest;
        sigmoids(x[q], f[i][q], rest);
        slope[i][q] = (a.free ? h[q] : h[q] - u[q]) * f[i][q] * rest;
        share[i][q] = a.free ? 1.f : rest;
        h[q] = fmaf(f[i][q], h[q], a.free ? u[q] : rest * u[q]);
      }
    }
#pragma unroll
    for (int i = kTile - 1; i >= 0; --i) {
      const int r = r0 + i;
      if (r < lo || r >= hi) continue;
      float dg[V] = {}, dv[V] = {};
      if (b.there >> i & 1) {
        if (b.last >> i & 1) {
          const float* from = a.dfinal ? a.dfinal + (int64_t)sequence_of(a, r) * a.cols + l.c : nullptr;
#pragma unroll
          for (int q = 0; q < V; ++q) m[q] = from && (q == 0 || l.both) ? from[q] : 0.f;
        }
        float y[V];
        unpack_word<GD, V>(d[i], y);
#pragma unroll
        for (int q = 0; q < V; ++q) {
          const float lam = y[q] + m[q];
          dg[q] = lam * slope[i][q];
          dv[q] = lam * share[i][q];
          m[q] = f[i][q] * lam;
        }
        if ((b.first >> i & 1) && a.dinitial) {
          float* to = a.dinitial + (int64_t)sequence_of(a, r) * a.cols + l.c;
#pragma unroll
          for (int q = 0; q < V; ++q)
            if (q == 0 || l.both) to[q] = m[q];
        }
      }
      store_word<GD, V>(dgate + (int64_t)r * a.dgate_stride * GB, dg, l.both);
      store_word<GD, V>(dvalue + (int64_t)r * a.dvalue_stride * GB, dv, l.both);
    }
  }
}

// ------------------------------------------------------------------ one more row

struct Step {
  const char *gate, *value;
  char* h;
  int64_t gate_stride, value_stride, h_stride;
  const int32_t* slots;
  const float* state;
  float* new_state;
  unsigned long long* first_bad;
  int64_t rows, states;
  int cols;
  bool free;
};

constexpr int kStepBlock = 256;

template <int XD> __global__ __launch_bounds__(kStepBlock) void scan_step(const Step a, unsigned first) {
  constexpr int EB = dmt::EltBytes<XD>::value, E = 4;
  const int64_t i = (int64_t)first + blockIdx.x;
  int64_t slot = i;
  if (a.slots) {
    slot = a.slots[i];
    bool taken = false;                                       // by an earlier row
    for (int64_t j = threadIdx.x; j < i; j += kStepBlock) taken |= a.slots[j] == slot;
    const bool bad = slot >= 0 && (slot >= a.states || __syncthreads_or(taken));
    if (bad && threadIdx.x == 0 && a.first_bad) atomicMin(a.first_bad, (unsigned long long)i);
    if (bad) slot = -1;
  }
  for (int c = threadIdx.x * E; c < a.cols; c += kStepBlock * E) {
    const int valid = min(E, a.cols - c);
    float y[E] = {};
    if (slot >= 0) {
      float x[E], u[E];
      dmt::load_elems<XD, E>(a.gate + (i * a.gate_stride + c) * EB, valid, x);
      dmt::load_elems<XD, E>(a.value + (i * a.value_stride + c) * EB, valid, u);
      dmt::load_elems<DMT_F32, E>((const char*)(a.state + slot * a.cols + c), valid, y);
#pragma unroll
      for (int q = 0; q < E; ++q) {
        float f, rest;
        sigmoids(x[q], f, rest);
        y[q] = fmaf(f, y[q], a.free ? u[q] : rest * u[q]);
      }
      dmt::store_elems<DMT_F32, E>((char*)(a.new_state + slot * a.cols + c), valid, y);
    }
    dmt::store_elems<XD, E>(a.h + (i * a.h_stride + c) * EB, valid, y);
  }
}

// ------------------------------------------------------------------ rows' sequences

__global__ __launch_bounds__(256) void sequence_rows(const int64_t* offsets, int64_t sequences, int64_t rows, int32_t* out,
                                                     unsigned long long* first_bad) {
  const int64_t step = (int64_t)gridDim.x * 256, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t r = at; r < rows; r += step) {
    int64_t lo = 0, hi = sequences + 1;                        // offsets before lo are <= r, from hi on > r
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (offsets[mid] <= r) lo = mid + 1;
      else hi = mid;
    }
    out[r] = lo <= sequences ? (int)(lo - 1) : -1;
  }
  if (first_bad)
    for (int64_t b = at; b < sequences; b += step)
      if (offsets[b + 1] < offsets[b]) atomicMin(first_bad, (unsigned long long)b);
}

// ------------------------------------------------------------------ host

constexpr int64_t kMost = 1ll << 30;          // rows and sequences: a tile past the last row is still a 32-bit row

// Waves that fill the chip with enough rows requested at once.
constexpr int64_t kWaves = 2048;

Cut cut_of(int64_t rows, int64_t cols, int v, bool dense, int64_t sequences) {
  Cut c = {};
  const int64_t lanes = (cols + v - 1) / v;
  c.group = lanes <= 16 ? 16 : lanes <= 32 ? 32 : 64;
  c.tiles = (int)((lanes + c.group - 1) / c.group);
  const int64_t walkers = kBlock / c.group;
  auto waves = [&](int64_t sub) { return (rows + sub - 1) / sub * c.tiles * c.group / 64; };
  if (dense && rows > 0) {
    const int64_t length = rows / sequences, many = std::max<int64_t>(1, 32 / length);
    if (waves(length * many) >= kWaves) {
      c.sub = length * many, c.chunk = c.sub * walkers, c.whole = c.one = true;
      c.chunks = (rows + c.chunk - 1) / c.chunk;
      return c;
    }
  }
  c.sub = 64;
  while (c.sub > 16 && waves(c.sub) < kWaves) c.sub /= 2;
  if (rows <= walkers * 64) c.sub = std::max<int64_t>(16, (rows + walkers * 16 - 1) / (walkers * 16) * 16);
  c.chunk = c.sub * walkers;
  c.chunks = std::max<int64_t>(1, (rows + c.chunk - 1) / c.chunk);
  c.one = c.chunks == 1;
  return c;
}

template <int V> struct Int { static constexpr int value = V; };

size_t stretch_bytes(const Cut& c, int64_t cols) { return c.one ? 0 : sizeof(float2) * (size_t)(c.chunks * (kBlock / c.group) * cols); }
size_t chunk_bytes(const Cut& c, int64_t cols) { return c.one ? 0 : sizeof(float2) * (size_t)(c.chunks * cols); }
size_t scratch_bytes(const Cut& c, int64_t cols) {
  return c.one ? 0 : stretch_bytes(c, cols) + chunk_bytes(c, cols) + sizeof(int) * (size_t)c.chunks;
}

bool fits(int64_t rows, int64_t cols) { return rows <= kMost && cols <= 1 << 24; }

// Checks that the forward and the backward share.
dmt_status checked(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride, int64_t rows, int64_t cols,
                   int32_t dtype, int32_t form, const int32_t* sequence_of, int64_t sequences, const float* initial) {
  if (rows < 0 || cols < 1 || sequences < 0 || gate_stride < cols || value_stride < cols || !dmt_is_dtype(dtype)) return DMT_EINVAL;
  if (form != DMT_SCAN_COUPLED && form != DMT_SCAN_FREE) return DMT_EINVAL;
  const int64_t e = dmt_ebytes(dtype);
  if (rows > 0 && (!dmt_is_at(gate, e) || !dmt_is_at(value, e))) return DMT_EINVAL;
  if (!dmt_may_be_at(sequence_of, 4) || !dmt_may_be_at(initial, 4)) return DMT_EINVAL;
  if (!sequence_of && rows > 0 && (sequences < 1 || rows % sequences != 0)) return DMT_EINVAL;
  if (!fits(rows, cols) || sequences > kMost) return DMT_ENOTSUP;
  return DMT_OK;
}

// Fills in how the rows are cut; where the workspace is too small or misplaced, says so.
dmt_status place(Scan& a, const Cut& c, void* workspace, size_t workspace_bytes) {
  const size_t need = scratch_bytes(c, a.cols);
  if (need > 0 && !dmt_is_at(workspace, 256)) return DMT_EINVAL;
  if (workspace_bytes < need) return DMT_ENOMEM;
  a.tiles = c.tiles, a.sub = c.sub, a.chunk_rows = c.chunk, a.chunks = c.chunks, a.whole = c.whole;
  a.stretch = (float2*)workspace;
  a.chunk = (float2*)((char*)workspace + stretch_bytes(c, a.cols));
  a.forgets = (int*)((char*)a.chunk + chunk_bytes(c, a.cols));
  return DMT_OK;
}

template <typename Kernel> void launch(Kernel kernel, const Scan& a, hipStream_t s) {
  dmt_launches(a.chunks * a.tiles, kBlock,
               [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, a, first); });
}

template <int G, int XD> void run_fwd(const Scan& a, const Cut& c, hipStream_t s) {
  if (c.one) {
    launch(scan_fwd<G, XD, true>, a, s);
  } else {
    launch(scan_stretches<G, XD, XD, false>, a, s);
    launch(scan_fwd<G, XD, false>, a, s);
  }
}
template <int G, int XD, int GD> void run_bwd(const Scan& a, const Cut& c, hipStream_t s) {
  if (c.one) {
    launch(scan_bwd<G, XD, GD, true>, a, s);
  } else {
    launch(scan_stretches<G, XD, GD, true>, a, s);
    launch(scan_bwd<G, XD, GD, false>, a, s);
  }
}
template <typename Run> void by_group(int group, Run run) {
  if (group == 16) run(Int<16>());
  else if (group == 32) run(Int<32>());
  else run(Int<64>());
}

}  // namespace

extern "C" dmt_status dmt_sequence_rows(const int64_t* offsets, int64_t sequences, int64_t rows, int32_t* sequence_of,
                                        int64_t* first_bad, void* stream) {
  if (sequences < 0 || rows < 0 || !dmt_is_at(offsets, 8) || !dmt_may_be_at(first_bad, 8)) return DMT_EINVAL;
  if (rows > 0 && !dmt_is_at(sequence_of, 4)) return DMT_EINVAL;
  if (rows > kMost || sequences > kMost) return DMT_ENOTSUP;
  const int64_t n = std::max(rows, sequences);
  if (n == 0) return DMT_OK;
  hipLaunchKernelGGL(sequence_rows, dim3((unsigned)std::min<int64_t>(4096, (n + 255) / 256)), dim3(256), 0, (hipStream_t)stream, offsets,
                     sequences, rows, sequence_of, (unsigned long long*)first_bad);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" size_t dmt_gated_scan_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || !fits(rows, cols)) return 0;
  return std::max(scratch_bytes(cut_of(rows, cols, 1, false, 0), cols), scratch_bytes(cut_of(rows, cols, 2, false, 0), cols));
}

extern "C" size_t dmt_gated_scan_kept_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || !fits(rows, cols)) return 0;
  return sizeof(float) * (size_t)((rows + kTile - 1) / kTile * cols);
}

extern "C" dmt_status dmt_gated_scan_fwd(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride,
                                         int64_t rows, int64_t cols, int32_t dtype, int32_t form,
                                         const int32_t* sequence_of, int64_t sequences, const float* initial, void* h,
                                         int64_t h_stride, float* final, void* kept, size_t kept_bytes,
                                         int64_t* first_bad, void* workspace, size_t workspace_bytes, void* stream) {
  const dmt_status bad = checked(gate, gate_stride, value, value_stride, rows, cols, dtype, form, sequence_of, sequences, initial);
  if (bad != DMT_OK) return bad;
  if (h_stride < cols || (rows > 0 && !dmt_is_at(h, dmt_ebytes(dtype)))) return DMT_EINVAL;
  if (!dmt_may_be_at(final, 4) || (final && final == initial) || !dmt_may_be_at(kept, 256) || !dmt_may_be_at(first_bad, 8)) return DMT_EINVAL;
  if (kept && kept_bytes < dmt_gated_scan_kept_bytes(rows, cols)) return DMT_ENOMEM;
  if (rows == 0) return DMT_OK;
  Scan a = {};
  a.gate = (const char*)gate, a.value = (const char*)value, a.h = (char*)h;
  a.gate_stride = gate_stride, a.value_stride = value_stride, a.h_stride = h_stride, a.rows = rows, a.cols = (int)cols;
  a.seq = sequence_of, a.sequences = (int)sequences, a.length = sequence_of ? 1 : (int)(rows / sequences);
  a.initial = initial, a.final = final, a.kept = (float*)kept, a.free = form == DMT_SCAN_FREE, a.first_bad = (unsigned long long*)first_bad;
  const Cut c = cut_of(rows, cols, dtype == DMT_F32 ? 1 : 2, !sequence_of, sequences);
  const dmt_status room = place(a, c, workspace, workspace_bytes);
  if (room != DMT_OK) return room;
  by_group(c.group, [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (dtype == DMT_F32) run_fwd<G, DMT_F32>(a, c, (hipStream_t)stream);
    else if (dtype == DMT_F16) run_fwd<G, DMT_F16>(a, c, (hipStream_t)stream);
    else run_fwd<G, DMT_BF16>(a, c, (hipStream_t)stream);
  });
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" dmt_status dmt_gated_scan_bwd(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride,
                                         int64_t rows, int64_t cols, int32_t dtype, int32_t form,
                                         const int32_t* sequence_of, int64_t sequences, const float* initial,
                                         const void* kept, size_t kept_bytes, const void* dh, int64_t dh_stride,
                                         int32_t grad_dtype, const float* dfinal, void* dgate, int64_t dgate_stride,
                                         void* dvalue, int64_t dvalue_stride, float* dinitial, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  const dmt_status bad = checked(gate, gate_stride, value, value_stride, rows, cols, dtype, form, sequence_of, sequences, initial);
  if (bad != DMT_OK) return bad;
  if (grad_dtype != dtype && grad_dtype != DMT_F32) return DMT_EINVAL;
  if (dh_stride < cols || dgate_stride < cols || dvalue_stride < cols) return DMT_EINVAL;
  const int64_t ge = dmt_ebytes(grad_dtype);
  if (rows > 0 && (!dmt_is_at(dh, ge) || !dmt_is_at(dgate, ge) || !dmt_is_at(dvalue, ge) || !dmt_is_at(kept, 256))) return DMT_EINVAL;
  if (!dmt_may_be_at(dfinal, 4) || !dmt_may_be_at(dinitial, 4) || (dfinal && dfinal == dinitial)) return DMT_EINVAL;
  if (kept_bytes < dmt_gated_scan_kept_bytes(rows, cols)) return DMT_ENOMEM;
  if (rows == 0) return DMT_OK;
  Scan a = {};
  a.gate = (const char*)gate, a.value = (const char*)value, a.dh = (const char*)dh, a.dgate = (char*)dgate, a.dvalue = (char*)dvalue;
  a.gate_stride = gate_stride, a.value_stride = value_stride, a.dh_stride = dh_stride, a.dgate_stride = dgate_stride;
  a.dvalue_stride = dvalue_stride, a.rows = rows, a.cols = (int)cols;
  a.seq = sequence_of, a.sequences = (int)sequences, a.length = sequence_of ? 1 : (int)(rows / sequences);
  a.initial = initial, a.dfinal = dfinal, a.dinitial = dinitial, a.kept = (float*)kept, a.free = form == DMT_SCAN_FREE;
  const Cut c = cut_of(rows, cols, dtype == DMT_F32 ? 1 : 2, !sequence_of, sequences);
  const dmt_status room = place(a, c, workspace, workspace_bytes);
  if (room != DMT_OK) return room;
  hipStream_t s = (hipStream_t)stream;
  by_group(c.group, [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (dtype == DMT_F32) run_bwd<G, DMT_F32, DMT_F32>(a, c, s);
    else if (dtype == DMT_F16 && grad_dtype == DMT_F16) run_bwd<G, DMT_F16, DMT_F16>(a, c, s);
    else if (dtype == DMT_F16) run_bwd<G, DMT_F16, DMT_F32>(a, c, s);
    else if (grad_dtype == DMT_BF16) run_bwd<G, DMT_BF16, DMT_BF16>(a, c, s);
    else run_bwd<G, DMT_BF16, DMT_F32>(a, c, s);
  });
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}

extern "C" dmt_status dmt_gated_scan_step(const void* gate, int64_t gate_stride, const void* value, int64_t value_stride,
                                          int64_t rows, int64_t cols, int32_t dtype, int32_t form, const int32_t* slots,
                                          const float* state, float* new_state, int64_t states, void* h,
                                          int64_t h_stride, int64_t* first_bad, void* stream) {
  if (rows < 0 || cols < 1 || states < 0 || gate_stride < cols || value_stride < cols || h_stride < cols || !dmt_is_dtype(dtype))
    return DMT_EINVAL;
  if (form != DMT_SCAN_COUPLED && form != DMT_SCAN_FREE) return DMT_EINVAL;
  const int64_t e = dmt_ebytes(dtype);
  if (rows > 0 && (!dmt_is_at(gate, e) || !dmt_is_at(value, e) || !dmt_is_at(h, e))) return DMT_EINVAL;
  if (states > 0 && (!dmt_is_at(state, 4) || !dmt_is_at(new_state, 4))) return DMT_EINVAL;
  if (!dmt_may_be_at(slots, 4) || !dmt_may_be_at(first_bad, 8) || (!slots && states < rows)) return DMT_EINVAL;
  if (rows > kMost || (slots && rows > 65536) || states > kMost || cols > 1 << 24) return DMT_ENOTSUP;
  if (rows == 0) return DMT_OK;
  Step a = {};
  a.gate = (const char*)gate, a.value = (const char*)value, a.h = (char*)h;
  a.gate_stride = gate_stride, a.value_stride = value_stride, a.h_stride = h_stride, a.slots = slots;
  a.state = state, a.new_state = new_state, a.first_bad = (unsigned long long*)first_bad, a.rows = rows, a.states = states;
  a.cols = (int)cols, a.free = form == DMT_SCAN_FREE;
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto kernel) {
    dmt_launches(rows, kStepBlock, [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kStepBlock), 0, s, a, first); });
  };
  if (dtype == DMT_F32) go(scan_step<DMT_F32>);
  else if (dtype == DMT_F16) go(scan_step<DMT_F16>);
  else go(scan_step<DMT_BF16>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
