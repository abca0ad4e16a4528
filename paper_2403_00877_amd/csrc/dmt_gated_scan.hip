// dmt_gated_scan_fwd, dmt_gated_scan_bwd, dmt_gated_scan_step, dmt_sequence_rows:  h_t = f_t h_{t-1} + u_t,  f = sigmoid(gate),
// u = (1 - f) value or value; and backwards  l_t = dh_t + m_{t+1},  m_t = f_t l_t,  dvalue = l (1 - f),  dgate = l (h_{t-1} - value) f (1 - f).
//
// Both are first-order recurrences, so a stretch of rows maps the state before it to the one behind it by h -> A h + S, with A the
// product of its f; a stretch that holds a sequence's first row (backwards: its last) forgets what came before.  Rows are cut
// into chunks, a block's each (for the channels of a group of lanes), and chunks into the stretches of `walkers`: lane
// groups that go through their rows one after another, 8 at a time, with a lane's channels in registers.  A stretch begins where a
// sequence does, if one begins near its nominal place; so short sequences are walked whole and only long ones are cut.  Where any
// is cut, a first launch takes every stretch's (A, S), reading only the rows that a next stretch continues, and the second starts each
// walker from what those before it lead to.  One chunk does both in one launch, and so do equal sequences that are no longer than a stretch.
//
// The backward needs h_{t-1}: the forward keeps the state in front of every 8th row in float32, from which a walker goes through
// its 8 rows again, so neither h nor a rounded h is read.
//
// Bound by memory where sequences are long: two of 65536 x 512 bfloat16, forward 80 + 86 us (the rows are read twice, 268 MB each time,
// and 168 MB written), backward 65 + 141 (705 MB in the second launch, 5.0 TB/s).  4096 ragged ones, 131072 x 256 bfloat16, forward 22 + 51 us, backward
// 25 + 94.  2048 padded ones, 102400 x 201 float32, forward 6 + 51 us, backward 5 + 69.  4096 of 64 x 256 bfloat16 whole, one launch each, 90 + 141 (4.8 and
// 5.0 TB/s).  A later chunk looks through the maps of all earlier ones of its sequence: (chunks)^2 / 2 of 8 bytes a channel.  2^18 rows of 512 bfloat16 as one
// sequence for 16: second launches 192 + 300 us for 185 + 284; 2^20 as one for 64: 938 + 1366 for 743 + 1203; 2^24 of 16 channels as one for 256: 491 + 940 for 411 + 851.
#include <algorithm>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

// Threads of a block; rows of a tile, of a turn of the first launch; the longest stretch's; channels of a lane.  (Two channels a lane: backward of 102400 x 201
// float32 111 us for 88, one: 120.  Eight of bfloat16: forward of 131072 x 512 no faster, of 131072 x 256 ragged 59 for 50: twice the registers.)
constexpr int kBlock = 512, kTile = 8, kRun = 16, kSub = 64, kRoom = 32, V = 4;
constexpr uint32_t kAll = (1u << kTile) - 1;

// How rows are cut.
struct Cut {
  int group;           // lanes of a walker: 8, 16, 32 or 64
  int tiles;           // groups' widths of channels
  int64_t sub;         // rows of a walker nominally
  int64_t chunk;       // rows of a chunk
  int64_t chunks;
  bool whole;          // every walker starts with a sequence's first row: equal ones, none longer than a stretch
  bool one;            // no state passes between chunks
  bool narrow;         // fewer channels than a lane has
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
  bool whole, one;
  int64_t sub, chunk_rows, chunks;
};

// Lanes of a walker.  0 stands for rows of fewer channels than a lane has (a walker has 8 lanes then, and one of them has them).
template <int G> struct Lanes { static constexpr int value = G == 0 ? 8 : G; };

template <int G> __device__ __forceinline__ int uniform(int v) {
  if constexpr (G == 64) return __builtin_amdgcn_readfirstlane(v);
  else return v;
}

__device__ __forceinline__ int id_of(const Scan& a, int row) {
  const int id = a.seq[row];
  return (uint32_t)id < (uint32_t)a.sequences ? id : -1;
}
__device__ __forceinline__ int sequence_of(const Scan& a, int row) { return a.seq ? id_of(a, row) : row / a.length; }

// Where the rows of the walker whose nominal first row is b begin: where the sequence changes next, if it does within the stretch, else at
// b's tile, in front of whose first row the state is kept.  So walkers have whole sequences where those are short, and only long ones are cut.
// (The stretch is looked through up to the next one's tile, so that beginnings ascend.)
template <int G> __device__ __forceinline__ int begin_of(const Scan& a, int64_t nominal) {
  constexpr int N = Lanes<G>::value, Steps = kSub / N;
  if (nominal >= a.rows) return (int)a.rows;
  const int64_t past = (nominal + a.sub) & ~(int64_t)(kTile - 1);
  const int b = (int)nominal, end = (int)min(a.rows, past), lane = threadIdx.x & 63;
  if (!a.seq) {
    const int next = (b + a.length - 1) / a.length * a.length;
    return next < past ? next : b & ~(kTile - 1);
  }
  int here[Steps], before[Steps];
#pragma unroll
  for (int i = 0; i < Steps; ++i) {
    const int row = min(b + i * N + lane % N, end - 1);
    here[i] = id_of(a, row);
    before[i] = id_of(a, max(row - 1, 0));
  }
  int found = b & ~(kTile - 1);
#pragma unroll
  for (int i = Steps - 1; i >= 0; --i) {
    const int row = b + i * N + lane % N;
    uint64_t change = __ballot(row < end && (row == 0 || here[i] != before[i])) >> (N == 64 ? 0 : lane & ~(N - 1));
    if (N < 64) change &= (1ull << (N & 63)) - 1;
    if (change) found = b + i * N + __builtin_ctzll(change);
  }
  return uniform<G>(found);
}

// Bits of the kTile rows from r0 on that lie in [lo, hi): whether a row is of a sequence, is its first, its last; and the
// sequence of row r0 + (lane mod kTile).
struct Bits {
  uint32_t there, first, last;
  int id;
  // Row i's sequence.
  __device__ __forceinline__ int id_at(int i) const { return __shfl(id, (threadIdx.x & 63 & ~(kTile - 1)) + i); }
};

// What the bits of a tile are made of, requested ahead: raw ids of a lane's row and of its neighbours.
struct Ids { int before, here, behind; };

__device__ __forceinline__ Ids ids_of(const Scan& a, int r0, int lo, int hi) {
  Ids x = {-1, -1, -1};
  const int row = r0 + (threadIdx.x & (kTile - 1));
  if (a.seq && row >= lo && row < hi) {
    x.before = a.seq[max(row - 1, 0)];
    x.here = a.seq[row];
    x.behind = a.seq[min(row + 1, (int)a.rows - 1)];
  }
  return x;
}

template <int G> __device__ __forceinline__ Bits bits_of(const Scan& a, Ids x, int r0, int lo, int hi) {
  const int lane = threadIdx.x & 63, row = r0 + (lane & (kTile - 1));
  bool there = row >= lo && row < hi, first, last;
  Bits b;
  if (a.seq) {
    const auto valid = [&](int id) { return (uint32_t)id < (uint32_t)a.sequences ? id : -1; };
    b.id = valid(x.here);
    first = row == 0 || valid(x.before) != b.id;
    last = row + 1 == (int)a.rows || valid(x.behind) != b.id;
    there = there && b.id >= 0;
  } else {
    b.id = (int)((uint32_t)max(row, 0) / (uint32_t)a.length);
    const int at = row - b.id * a.length;
    first = at == 0;
    last = at == a.length - 1;
  }
  const int shift = G == 64 ? 0 : lane & ~(kTile - 1);
  b.there = (uint32_t)(__ballot(there) >> shift) & kAll;
  b.first = (uint32_t)(__ballot(there && first) >> shift) & kAll;
  b.last = (uint32_t)(__ballot(there && last) >> shift) & kAll;
  return b;
}

// Lowers first_bad to the first of rows [lo, hi) whose id is none; the walker's lanes look at its rows.
__device__ __forceinline__ void report_bad(const Scan& a, int lo, int hi, int at, int lanes) {
  for (int row = lo + at; row < hi; row += lanes)
    if (a.seq[row] >= a.sequences) {
      atomicMin(a.first_bad, (unsigned long long)row);
      break;
    }
}

// f = sigmoid(x) and 1 - f from e = exp(-x): f = 1 / (1 + e), 1 - f = e f.  The product x log2 e is rounded, so e is off by up to 1.25 |x|
// units of 2^-24 and two more; f and 1 - f then by f (1 - f) times that, at most 0.65 units, and by a few units of their own.  The reciprocal
// gives 0 where its result is below 2^-126, so f is 0 from e = 2^126 on, and e f with it: 1 - f is taken as 1 where it is that to half a unit, from 2^25 on.
// A NaN is in f and in 1 - f (the comparison is false; a minimum would take the number).
__device__ __forceinline__ float exp_minus(float x) { return __builtin_amdgcn_exp2f(x * -1.44269504088896341f); }
__device__ __forceinline__ void from_exp(float e, float& f, float& rest) {
  f = __builtin_amdgcn_rcpf(1.f + e);
  rest = e >= 0x1p25f ? 1.f : e * f;
}
__device__ __forceinline__ void sigmoids(float x, float& f, float& rest) { from_exp(exp_minus(x), f, rest); }

// Which chunk and channels a block has.  Blocks go to the eight XCDs in turn; the tiles of a chunk go to one, so that a line that two
// tiles share (rows of no whole number of lines) is read once and written whole from its L2.
struct Block {
  int64_t chunk;
  int tile;
  __device__ __forceinline__ Block(const Scan& a, unsigned first) {
    const uint32_t at = first + blockIdx.x, tiles = (uint32_t)a.tiles, many = (uint32_t)(a.chunks / 8 * 8) * tiles;
    if (at < many) {
      chunk = at / 8 / tiles * 8 + at % 8;
      tile = (int)(at / 8 % tiles);
    } else {
      chunk = at / tiles;
      tile = (int)(at % tiles);
    }
  }
};

struct Map { float a, s; };
__device__ __forceinline__ Map after(Map l, Map r) {         // l, then r
  if (r.a < 0.f) return r;
  return {l.a < 0.f ? -1.f : l.a * r.a, fmaf(r.a, l.s, r.s)};
}
__device__ __forceinline__ float applied(Map m, float h) { return m.a < 0.f ? m.s : fmaf(m.a, h, m.s); }

// What a lane knows about its channels.
template <int G> struct Lane {
  static constexpr int N = Lanes<G>::value;
  int w, at, c, valid;     // walker, lane of it, first channel, how many there are
  __device__ __forceinline__ Lane(int tile, int cols) {
    w = uniform<G>(threadIdx.x / N);
    at = threadIdx.x % N;
    // the last lane of an odd width has channels of the one before too, and lanes past the width have the last ones: all find, and
    // store, the same
    c = G == 0 ? 0 : min((tile * N + at) * V, cols - V);
    valid = G == 0 ? cols : V;
  }
};

// A lane's channels of a row of a float32 [rows][cols] (null: zeros); and back.
__device__ __forceinline__ void load_state(const float* p, int64_t row, int cols, int c, int valid, float (&x)[V]) {
#pragma unroll
  for (int q = 0; q < V; ++q) x[q] = 0.f;
  if (p) dmt::load_elems<DMT_F32, V>((const char*)(p + row * cols) + (uint32_t)c * 4u, valid, x);
}
__device__ __forceinline__ void store_state(float* p, int64_t row, int cols, int c, int valid, const float (&x)[V]) {
  dmt::store_elems<DMT_F32, V>((char*)(p + row * cols) + (uint32_t)c * 4u, valid, x);
}

// ---- maps of a block's walkers, in the rows' order (Back: against it)

// m: the walker's own -> of all walkers of the wave up to it.
template <int G, bool Back> __device__ __forceinline__ void join_wave(Map (&m)[V]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = Lanes<G>::value; o < 64; o <<= 1)
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const Map t = {Back ? __shfl_down(m[q].a, o) : __shfl_up(m[q].a, o), Back ? __shfl_down(m[q].s, o) : __shfl_up(m[q].s, o)};
      if (Back ? lane + o < 64 : lane >= o) m[q] = after(t, m[q]);
    }
}
// From there: of all walkers of the wave before it.
template <int G, bool Back> __device__ __forceinline__ void before_in_wave(Map (&m)[V]) {
  constexpr int N = Lanes<G>::value;
  const int lane = threadIdx.x & 63;
  const bool none = Back ? lane + N >= 64 : lane < N;
#pragma unroll
  for (int q = 0; q < V; ++q) {
    const Map t = {Back ? __shfl_down(m[q].a, N) : __shfl_up(m[q].a, N), Back ? __shfl_down(m[q].s, N) : __shfl_up(m[q].s, N)};
    m[q] = none ? Map{1.f, 0.f} : t;
  }
}
// The wave's own map, of its last walker, to all.
template <int G, bool Back, int C> __device__ __forceinline__ void tell_wave(const Map (&m)[V], Map (&waves)[kBlock / 64][C]) {
  constexpr int N = Lanes<G>::value;
  const int lane = threadIdx.x & 63;
  if (Back ? lane < N : lane >= 64 - N)
#pragma unroll
    for (int q = 0; q < V; ++q) waves[threadIdx.x >> 6][lane % N * V + q] = m[q];
}

// ---- what a stretch makes of the state before it

// Rows [from, hi) in their order: A and S.
template <int XD, bool Free>
__device__ __forceinline__ void map_fwd(const Scan& a, int c, int valid, int from, int hi, float (&A)[V], float (&S)[V]) {
  constexpr int EB = dmt::EltBytes<XD>::value;
  const int64_t gs = a.gate_stride * EB, vs = a.value_stride * EB;
  const char *gp = a.gate + from * gs, *vp = a.value + from * vs;
  const uint32_t off = (uint32_t)c * EB;
  for (int r0 = from; r0 < hi; r0 += kRun) {
    dmt::Raw<XD, V> g[kRun], v[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const int j = min(i, hi - 1 - r0);
      g[i] = dmt::load_raw<XD, V>(gp + j * gs + off, valid);
      v[i] = dmt::load_raw<XD, V>(vp + j * vs + off, valid);
    }
    const auto row = [&](int i) {
      float x[V], u[V];
      dmt::unpack<XD, V>(g[i], x);
      dmt::unpack<XD, V>(v[i], u);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float f, rest;
        sigmoids(x[q], f, rest);
        S[q] = fmaf(f, S[q], Free ? u[q] : rest * u[q]);
        A[q] *= f;
      }
    };
    if (r0 + kRun <= hi) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) row(i);
    } else {
#pragma unroll
      for (int i = 0; i < kRun - 1; ++i)
        if (r0 + i < hi) row(i);
    }
    gp += kRun * gs;
    vp += kRun * vs;
  }
}

// Rows [lo, to] against their order: m -> A m + S.
template <int XD, int GD>
__device__ __forceinline__ void map_bwd(const Scan& a, int c, int valid, int lo, int to, float (&A)[V], float (&S)[V]) {
  constexpr int EB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  const int64_t gs = a.gate_stride * EB, ds = a.dh_stride * GB;
  const char *gp = a.gate + to * gs, *dp = a.dh + to * ds;
  const uint32_t off = (uint32_t)c * EB, off_g = (uint32_t)c * GB;
  for (int r0 = to; r0 >= lo; r0 -= kRun) {
    dmt::Raw<XD, V> g[kRun];
    dmt::Raw<GD, V> d[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const int j = min(i, r0 - lo);
      g[i] = dmt::load_raw<XD, V>(gp - j * gs + off, valid);
      d[i] = dmt::load_raw<GD, V>(dp - j * ds + off_g, valid);
    }
    const auto row = [&](int i) {
      float x[V], y[V];
      dmt::unpack<XD, V>(g[i], x);
      dmt::unpack<GD, V>(d[i], y);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float f = __builtin_amdgcn_rcpf(1.f + exp_minus(x[q]));
        S[q] = f * (y[q] + S[q]);
        A[q] *= f;
      }
    };
    if (r0 - kRun >= lo - 1) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) row(i);
    } else {
#pragma unroll
      for (int i = 0; i < kRun - 1; ++i)
        if (r0 - i >= lo) row(i);
    }
    gp -= kRun * gs;
    dp -= kRun * ds;
  }
}

// The map of rows [lo, hi) (backwards: against their order).  Only what the next (the previous) row continues is read: nothing
// where a sequence starts there, else from the last first (to the first last) row on.
template <int G, int XD, int GD, bool Back, bool Free>
__device__ __forceinline__ void stretch_of(const Scan& a, const Lane<G>& l, int lo, int hi, Map (&m)[V]) {
  constexpr int N = Lanes<G>::value;
  float A[V], S[V];
#pragma unroll
  for (int q = 0; q < V; ++q) A[q] = 1.f, S[q] = 0.f;
  bool forgets = false;
  if (lo < hi) {
    const int edge = Back ? lo : hi, inner = Back ? lo : hi - 1, outer = Back ? lo - 1 : hi;     // rows inner and outer: of one sequence?
    int at = Back ? hi - 1 : lo;                           // the row from which (to which) on the map is made
    bool on = edge > 0 && edge < (int)a.rows;
    if (on && a.seq) {
      const int id = id_of(a, inner), next = id_of(a, outer);
      const int there = Back ? hi - 1 : lo, past = Back ? min(hi, (int)a.rows - 1) : max(lo - 1, 0);
      const bool ends = id_of(a, there) != id_of(a, past) || (Back ? hi == (int)a.rows : lo == 0);
      on = id >= 0 && id == next;
      forgets = ends;                                      // unless a row in between says so nearer
      for (int i = 0; on && i < hi - lo; i += N) {
        const int row = Back ? lo + i + l.at : hi - 1 - i - l.at;
        const bool other = row >= lo && row < hi && id_of(a, row) != id;
        uint64_t found = __ballot(other) >> (N == 64 ? 0 : (threadIdx.x & 63 & ~(N - 1)));
        if (N < 64) found &= (1ull << (N & 63)) - 1;
        if (found) {
          const int k = i + __builtin_ctzll(found);        // rows from the inner one on
          at = Back ? lo + k - 1 : hi - k;
          forgets = true;
          break;
        }
      }
    } else if (on) {
      on = edge % a.length != 0;
      const int begin = Back ? lo - lo % a.length + a.length - 1 : hi - 1 - (hi - 1) % a.length;
      forgets = Back ? begin < hi : begin >= lo;
      if (forgets) at = begin;
    }
    if (on) {
      if (forgets) load_state(Back ? a.dfinal : a.initial, sequence_of(a, inner), a.cols, l.c, l.valid, S);
      if constexpr (Back) map_bwd<XD, GD>(a, l.c, l.valid, lo, at, A, S);
      else map_fwd<XD, Free>(a, l.c, l.valid, at, hi, A, S);
    } else {
      forgets = true;
    }
  }
#pragma unroll
  for (int q = 0; q < V; ++q) m[q] = {forgets ? -1.f : A[q], S[q]};
}

template <int G, int XD, int GD, bool Back, bool Free>
__global__ __launch_bounds__(kBlock) void scan_stretches(const Scan a, unsigned first) {
  constexpr int N = Lanes<G>::value, W = kBlock / N;
  __shared__ Map waves[kBlock / 64][N * V];
  const Block block(a, first);
  const int64_t chunk = block.chunk;
  const Lane<G> l(block.tile, a.cols);
  Map m[V];
  const int64_t nominal = chunk * a.chunk_rows + l.w * a.sub;
  stretch_of<G, XD, GD, Back, Free>(a, l, begin_of<G>(a, nominal), begin_of<G>(a, nominal + a.sub), m);
#pragma unroll
  for (int q = 0; q < V; ++q)
    if (q < l.valid) a.stretch[(chunk * W + l.w) * a.cols + l.c + q] = make_float2(m[q].a, m[q].s);
  const bool mine = m[0].a < 0.f;
  join_wave<G, Back>(m);
  tell_wave<G, Back>(m, waves);
  const int forgets = __syncthreads_or(mine);
  if (l.w == 0) {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      Map all = {1.f, 0.f};
#pragma unroll
      for (int w = 0; w < kBlock / 64; ++w) all = after(all, waves[Back ? kBlock / 64 - 1 - w : w][l.at * V + q]);
      if (q < l.valid) a.chunk[chunk * a.cols + l.c + q] = make_float2(all.a, all.s);
    }
  }
  if (threadIdx.x == 0 && block.tile == 0) a.forgets[chunk] = forgets;
}

// The state in front of (behind) a walker's rows: from all chunks since the last one that forgets, then the chunk's walkers.
template <int G, int XD, int GD, bool Back, bool Free>
__device__ __forceinline__ void state_before(const Scan& a, const Lane<G>& l, int64_t chunk, int lo, int hi, float (&h)[V]) {
  constexpr int N = Lanes<G>::value, W = kBlock / N, Waves = kBlock / 64;
  __shared__ Map waves[2][Waves][N * V];
  __shared__ int nearest;
#pragma unroll
  for (int q = 0; q < V; ++q) h[q] = 0.f;
  if (a.whole) return;
  bool goes_on = lo < hi && (Back ? hi < (int)a.rows : lo > 0);
  if (goes_on) {
    const int edge = Back ? hi : lo;
    goes_on = a.seq ? id_of(a, edge) >= 0 && id_of(a, edge) == id_of(a, edge - 1) : edge % a.length != 0;
  }
  if (!__syncthreads_or(goes_on)) return;
  Map m[V];
  if (a.one) {
    stretch_of<G, XD, GD, Back, Free>(a, l, lo, hi, m);
  } else {
    float2 own[V];
#pragma unroll
    for (int q = 0; q < V; ++q) own[q] = a.stretch[(chunk * W + l.w) * a.cols + l.c + min(q, l.valid - 1)];
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
#pragma unroll
    for (int q = 0; q < V; ++q) m[q] = {1.f, 0.f};
#pragma unroll 4
    for (int64_t i = from; i < to; ++i) {
      const int64_t c = Back ? chunk + many - i : chunk - many + i;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float2 x = a.chunk[c * a.cols + l.c + min(q, l.valid - 1)];
        m[q] = after(m[q], {x.x, x.y});
      }
    }
    join_wave<G, false>(m);
    tell_wave<G, false>(m, waves[1]);
#pragma unroll
    for (int q = 0; q < V; ++q) m[q] = {own[q].x, own[q].y};
  }
  join_wave<G, Back>(m);
  tell_wave<G, Back>(m, waves[0]);
  before_in_wave<G, Back>(m);
  __syncthreads();
  const int wave = uniform<64>(threadIdx.x >> 6);
#pragma unroll
  for (int q = 0; q < V; ++q) {
    if (!a.one)
      for (int w = 0; w < Waves; ++w) h[q] = applied(waves[1][w][l.at * V + q], h[q]);
    if constexpr (Back) {
      for (int w = Waves - 1; w > wave; --w) h[q] = applied(waves[0][w][l.at * V + q], h[q]);
    } else {
      for (int w = 0; w < wave; ++w) h[q] = applied(waves[0][w][l.at * V + q], h[q]);
    }
    h[q] = applied(m[q], h[q]);
  }
}

// ---- the rows

// The tile's rows of a matrix, p the first and a lane's channels `off` bytes in; where a row is not there a row of the walker's own,
// `own` rows on (read and not used).  (A walker of a whole wave has p in scalar registers, and a load is one instruction.)
template <int D> __device__ __forceinline__ void load_tile(const char* p, int64_t stride, bool all, uint32_t there, int own, uint32_t off,
                                                                  int valid, dmt::Raw<D, V> (&x)[kTile]) {
  if (all) {
#pragma unroll
    for (int i = 0; i < kTile; ++i) x[i] = dmt::load_raw<D, V>(p + i * stride + off, valid);
  } else {
    const char* instead = p + own * stride;
#pragma unroll
    for (int i = 0; i < kTile; ++i) x[i] = dmt::load_raw<D, V>((there >> i & 1 ? p + i * stride : instead) + off, valid);
  }
}
// Whether every walker of the wave says so.
template <int G> __device__ __forceinline__ bool every(bool x) {
  if constexpr (G == 64) return x;
  else return __ballot(!x) == 0;
}
// A stride of the loop's turn: its multiples are made there, not held for all rows of every matrix over the loop.
__device__ __forceinline__ int64_t here(int64_t stride) {
  asm volatile("" : "+s"(stride));
  return stride;
}
// Bits of the tile's rows in [lo, hi).
__device__ __forceinline__ uint32_t own_bits(int r0, int lo, int hi) {
  uint32_t b = kAll;
  if (r0 < lo) b &= kAll << (lo - r0);
  if (r0 + kTile > hi) b &= kAll >> (r0 + kTile - hi);
  return b;
}

template <int G, int XD, bool Free> __global__ __launch_bounds__(kBlock) void scan_fwd(const Scan a, unsigned first) {
  constexpr int EB = dmt::EltBytes<XD>::value;
  const Block block(a, first);
  const int64_t chunk = a.chunks - 1 - block.chunk;               // what was read last comes first
  const Lane<G> l(block.tile, a.cols);
  const int64_t nominal = chunk * a.chunk_rows + l.w * a.sub;
  const int lo = begin_of<G>(a, nominal), hi = begin_of<G>(a, nominal + a.sub);
  const int64_t gate_bytes = a.gate_stride * EB, value_bytes = a.value_stride * EB, h_bytes = a.h_stride * EB;
  const uint32_t off = (uint32_t)l.c * EB;
  int r0 = lo & ~(kTile - 1);
  Bits b = bits_of<G>(a, ids_of(a, r0, lo, hi), r0, lo, hi);
  float h[V];
  state_before<G, XD, XD, false, Free>(a, l, chunk, lo, hi, h);
  if (lo >= hi) return;
  if (a.seq && a.first_bad && block.tile == 0) report_bad(a, lo, hi, l.at, Lanes<G>::value);
  for (Bits next; r0 < hi; r0 += kTile, b = next) {
    const Ids ahead = ids_of(a, r0 + kTile, lo, hi);
    const uint32_t own = own_bits(r0, lo, hi);
    if (every<G>(b.there == 0)) {
      const float zero[V] = {};
      for (int i = 0; i < kTile; ++i)
        if (own >> i & 1) dmt::store_elems<XD, V>(a.h + (r0 + i) * h_bytes + off, l.valid, zero);
      next = bits_of<G>(a, ahead, r0 + kTile, lo, hi);
      continue;
    }
    const int64_t gs = here(gate_bytes), vs = here(value_bytes), hs = here(h_bytes);
    const bool all = every<G>(b.there == kAll);
    dmt::Raw<XD, V> g[kTile], v[kTile];
    float start[V];                                       // what the tile's first sequence starts from
    const int i0 = __builtin_ctz(b.first | 1u << kTile);
    load_tile<XD>(a.gate + r0 * gs, gs, all, b.there, max(lo - r0, 0), off, l.valid, g);
    load_tile<XD>(a.value + r0 * vs, vs, all, b.there, max(lo - r0, 0), off, l.valid, v);
    load_state(b.first ? a.initial : nullptr, b.id_at(i0), a.cols, l.c, l.valid, start);
    next = bits_of<G>(a, ahead, r0 + kTile, lo, hi);
    if (a.kept && r0 >= lo) store_state(a.kept, r0 / kTile, a.cols, l.c, l.valid, h);
    const auto step = [&](const dmt::Raw<XD, V>& gi, const dmt::Raw<XD, V>& vi) {
      float s[V], u[V];
      dmt::unpack<XD, V>(gi, s);
      dmt::unpack<XD, V>(vi, u);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float f, rest;
        sigmoids(s[q], f, rest);
        h[q] = fmaf(f, h[q], Free ? u[q] : rest * u[q]);
        asm volatile("" : "+v"(h[q]));                    // rounded to float32 before it is to 16 bits, whichever way the tile takes
      }
    };
    const auto row = [&](int i) { step(g[i], v[i]); };
    char* to = a.h + r0 * hs;
    const uint32_t ends = a.final ? b.last : 0u;
    if (all && every<G>(b.first == 0 && ends == 0)) {
#pragma unroll
      for (int i = 0; i < kTile; ++i) {
        row(i);
        dmt::store_elems<XD, V>(to + i * hs + off, l.valid, h);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kTile; ++i) {
        if (!(own >> i & 1)) continue;
        float out[V] = {};
        if (b.there >> i & 1) {
          if (b.first >> i & 1) {
            if (i != i0) load_state(a.initial, b.id_at(i), a.cols, l.c, l.valid, start);
#pragma unroll
            for (int q = 0; q < V; ++q) h[q] = start[q];
          }
          row(i);
#pragma unroll
          for (int q = 0; q < V; ++q) out[q] = h[q];
          if (ends >> i & 1) store_state(a.final, b.id_at(i), a.cols, l.c, l.valid, h);
        }
        dmt::store_elems<XD, V>(to + i * hs + off, l.valid, out);
      }
    }
  }
}

template <int G, int XD, int GD, bool Free>
__global__ __launch_bounds__(kBlock) void scan_bwd(const Scan a, unsigned first) {
  constexpr int EB = dmt::EltBytes<XD>::value, GB = dmt::EltBytes<GD>::value;
  const Block block(a, first);
  const int64_t chunk = a.chunks - 1 - block.chunk;
  const Lane<G> l(block.tile, a.cols);
  const int64_t nominal = chunk * a.chunk_rows + l.w * a.sub;
  const int lo = begin_of<G>(a, nominal), hi = begin_of<G>(a, nominal + a.sub);
  int r0 = (hi - 1) & ~(kTile - 1);
  Bits b = bits_of<G>(a, ids_of(a, r0, lo, hi), r0, lo, hi);
  float m[V];
  state_before<G, XD, GD, true, Free>(a, l, chunk, lo, hi, m);
  const int64_t gate_bytes = a.gate_stride * EB, value_bytes = a.value_stride * EB, dh_bytes = a.dh_stride * GB;
  const int64_t dgate_bytes = a.dgate_stride * GB, dvalue_bytes = a.dvalue_stride * GB;
  const uint32_t off = (uint32_t)l.c * EB, off_g = (uint32_t)l.c * GB;
  if (lo >= hi) return;
  for (Bits next; r0 + kTile > lo; r0 -= kTile, b = next) {
    const Ids ahead = ids_of(a, r0 - kTile, lo, hi);
    if (every<G>(b.there == 0)) {
      const uint32_t own = own_bits(r0, lo, hi);
      const float zero[V] = {};
      for (int i = 0; i < kTile; ++i)
        if (own >> i & 1) {
          dmt::store_elems<GD, V>(a.dgate + (r0 + i) * dgate_bytes + off_g, l.valid, zero);
          dmt::store_elems<GD, V>(a.dvalue + (r0 + i) * dvalue_bytes + off_g, l.valid, zero);
        }
      next = bits_of<G>(a, ahead, r0 - kTile, lo, hi);
      continue;
    }
    const int64_t gs = here(gate_bytes), vs = here(value_bytes), ds = here(dh_bytes), dgs = here(dgate_bytes), dvs = here(dvalue_bytes);
    const bool all = every<G>(b.there == kAll);
    dmt::Raw<XD, V> g[kTile], v[kTile];
    dmt::Raw<GD, V> d[kTile];
    // the state before the tile, what its first sequence starts from and the gradient that its last one ends with
    float h[V], start[V], end[V];
    const int i0 = __builtin_ctz(b.first | 1u << kTile), i1 = 31 - __builtin_clz(b.last | 1u), id0 = b.id_at(i0), id1 = b.id_at(i1);
    load_tile<XD>(a.gate + r0 * gs, gs, all, b.there, max(lo - r0, 0), off, l.valid, g);
    load_tile<XD>(a.value + r0 * vs, vs, all, b.there, max(lo - r0, 0), off, l.valid, v);
    load_tile<GD>(a.dh + r0 * ds, ds, all, b.there, max(lo - r0, 0), off_g, l.valid, d);
    load_state(r0 >= lo ? a.kept : nullptr, r0 / kTile, a.cols, l.c, l.valid, h);
    load_state(b.first ? a.initial : nullptr, id0, a.cols, l.c, l.valid, start);
    load_state(b.last ? a.dfinal : nullptr, id1, a.cols, l.c, l.valid, end);
    next = bits_of<G>(a, ahead, r0 - kTile, lo, hi);
    float prev[kTile][V];                                 // the state before each row, forwards; the gradients from them, backwards
    const auto there = [&](int i) {
      __builtin_amdgcn_sched_barrier(0);                  // one row after another, or the rows' f and 1 - f are all held at once
      float x[V], u[V];
      dmt::unpack<XD, V>(g[i], x);
      dmt::unpack<XD, V>(v[i], u);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float f, rest;
        sigmoids(x[q], f, rest);
        prev[i][q] = h[q];
        h[q] = fmaf(f, h[q], Free ? u[q] : rest * u[q]);
      }
    };
    const auto back = [&](int i, float (&dg)[V], float (&dv)[V]) {
      // f and 1 - f are made again: kept over the tile they take 64 registers, and with them a third of the waves
      dmt::Raw<XD, V> gi = g[i], vi = v[i];
#pragma unroll
      for (int q = 0; q < dmt::Raw<XD, V>::kWords; ++q) asm volatile("" : "+v"(gi.w[q]), "+v"(vi.w[q]));
      float x[V], u[V], y[V];
      dmt::unpack<XD, V>(gi, x);
      dmt::unpack<XD, V>(vi, u);
      dmt::unpack<GD, V>(d[i], y);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        float f, rest;
        sigmoids(x[q], f, rest);
        const float lam = y[q] + m[q], shut = lam * rest;
        dv[q] = Free ? lam : shut;
        dg[q] = (Free ? prev[i][q] : prev[i][q] - u[q]) * f * shut;
        m[q] = f * lam;
      }
    };
    char *to_g = a.dgate + r0 * dgs, *to_v = a.dvalue + r0 * dvs;
    if (all && every<G>((b.first | b.last) == 0)) {
#pragma unroll
      for (int i = 0; i < kTile; ++i) there(i);
#pragma unroll
      for (int i = kTile - 1; i >= 0; --i) {
        float dg[V], dv[V];
        back(i, dg, dv);
        dmt::store_elems<GD, V>(to_g + i * dgs + off_g, l.valid, dg);
        dmt::store_elems<GD, V>(to_v + i * dvs + off_g, l.valid, dv);
      }
    } else {
      const uint32_t own = own_bits(r0, lo, hi);
#pragma unroll
      for (int i = 0; i < kTile; ++i) {
        if (b.first >> i & 1) {
          if (i != i0) load_state(a.initial, b.id_at(i), a.cols, l.c, l.valid, start);
#pragma unroll
          for (int q = 0; q < V; ++q) h[q] = start[q];
        }
        there(i);                                         // (of no sequence: the next first row forgets it)
      }
#pragma unroll
      for (int i = kTile - 1; i >= 0; --i) {
        if (!(own >> i & 1)) continue;
        float dg[V] = {}, dv[V] = {};
        if (b.there >> i & 1) {
          if (b.last >> i & 1) {
            if (i != i1) load_state(a.dfinal, b.id_at(i), a.cols, l.c, l.valid, end);
#pragma unroll
            for (int q = 0; q < V; ++q) m[q] = end[q];
          }
          back(i, dg, dv);
          if ((b.first >> i & 1) && a.dinitial) store_state(a.dinitial, b.id_at(i), a.cols, l.c, l.valid, m);
        }
        dmt::store_elems<GD, V>(to_g + i * dgs + off_g, l.valid, dg);
        dmt::store_elems<GD, V>(to_v + i * dvs + off_g, l.valid, dv);
      }
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

constexpr int kStepBlock = 256, kStepRows = 64, kStepBits = 1 << 17;

// A block has `per` rows (Many) or one.  Whether an earlier row of the call names a row's slot too: one slot is compared with all
// earlier ones; several set bits (slot mod 2^17), the earlier ones are looked up there, and the few that hit are compared.  (One row a
// block: 8192 x 64 float16 17 us, 65536 x 64 580.)
template <int XD, bool Many> __global__ __launch_bounds__(kStepBlock) void scan_step(const Step a, int per, unsigned first) {
  constexpr int EB = dmt::EltBytes<XD>::value, E = 4;
  __shared__ int slots[kStepRows], taken[kStepRows];
  __shared__ uint32_t bits[Many ? kStepBits / 32 : 1];
  const int64_t i0 = (int64_t)(first + blockIdx.x) * per;
  const int m = (int)min((int64_t)per, a.rows - i0), t = threadIdx.x;
  if (a.slots) {
    int raw = -1;
    if (t < m) {
      raw = a.slots[i0 + t];
      slots[t] = raw < a.states ? raw : -1;
      taken[t] = 0;
    }
    if constexpr (Many) {
      for (int w = t; w < kStepBits / 32; w += kStepBlock) bits[w] = 0;
      __syncthreads();
      if (t < m && slots[t] >= 0) atomicOr(&bits[slots[t] % kStepBits / 32], 1u << (slots[t] & 31));
    }
    __syncthreads();
#pragma unroll 4
    for (int64_t j = t * 4; j < i0; j += kStepBlock * 4) {
      const int many = (int)min((int64_t)4, i0 - j);
      const auto ids = dmt::load_raw<DMT_F32, 4>((const char*)(a.slots + j), many);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int id = (int)ids.w[q];
        if (q >= many || id < 0) continue;
        if constexpr (Many) {
          if (bits[id % kStepBits / 32] >> (id & 31) & 1)
            for (int r = 0; r < m; ++r)
              if (slots[r] == id) taken[r] = 1;
        } else {
          if (slots[0] == id) taken[0] = 1;
        }
      }
    }
    __syncthreads();
    bool bad = false;
    if (t < m) {
      bad = raw >= a.states || taken[t];
      for (int r = 0; r < t; ++r) bad |= raw >= 0 && slots[r] == raw;
      if (bad && a.first_bad) atomicMin(a.first_bad, (unsigned long long)(i0 + t));
    }
    __syncthreads();
    if (bad) slots[t] = -1;
    __syncthreads();
  }
  const int pieces = (a.cols + E - 1) / E;
  for (int64_t at = t; at < (int64_t)m * pieces; at += kStepBlock) {
    const int r = (int)((uint64_t)at / (uint32_t)pieces), c = (int)(at - (int64_t)r * pieces) * E, valid = min(E, a.cols - c);
    const int64_t i = i0 + r, slot = a.slots ? slots[r] : i;
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

// Longer equal sequences are whole too where that leaves kWhole waves: bfloat16, forward and backward, 2048 of 128 x 256 93 + 145 us (2048 waves), cut
// 42 + 82 + 36 + 138; 256 of 256 x 1024 126 + 195 (1024 waves), cut 66 + 82 + 51 + 140; 128 of 512 x 1024 220 + 345 (512), cut 78 + 83 + 58 + 138.
constexpr int64_t kWhole = 1024;

// Waves that fill the chip with enough rows requested at once; stretches are as long as leaves so many, since a longer one is more
// often whole sequences, and then the first launch has nothing to read.  Equal sequences of up to kSub rows are always a walker's, one or some:
// 4096 of 64 x 64 bfloat16, forward and backward, 37 + 53 us, cut in four 49 + 68; one of 50 x 128 alone 13, in seven of eight rows 8.3 us.  131072 x 256 bfloat16 in 4096 ragged sequences: stretches of 32
// rows 21 + 48 us, of 64 20 + 64.  102400 x 201 float32 in 2048 padded ones (a lane has twice the bytes): of 64 6 + 65, of 32 16 + 64, of 16 26 + 62.
constexpr int64_t waves_for(int elem_bytes) { return elem_bytes == 4 ? 1536 : 4096; }

Cut cut_of(int64_t rows, int64_t cols, int elem_bytes, bool dense, int64_t sequences) {
  Cut c = {};
  const int64_t lanes = (cols + V - 1) / V;
  c.group = lanes <= 8 ? 8 : lanes <= 16 ? 16 : lanes <= 32 ? 32 : 64;
  c.tiles = (int)((lanes + c.group - 1) / c.group);
  c.narrow = cols < V;
  const int64_t walkers = kBlock / c.group;
  auto waves = [&](int64_t sub) { return (rows + sub - 1) / sub * c.tiles * c.group / 64; };
  const int64_t length = dense && rows > 0 ? rows / sequences : kSub + 1;
  const bool few = rows <= walkers * kSub;                 // one chunk holds all
  c.whole = dense && rows > 0 && (length <= (few ? 2 * kTile : kSub) || waves(length) >= kWhole);
  if (c.whole) {
    c.sub = length * std::max<int64_t>(1, 2 * kTile / length);
  } else if (few) {
    c.sub = std::max<int64_t>(kTile, (rows + walkers * kTile - 1) / (walkers * kTile) * kTile);
  } else {
    c.sub = kSub;
    while (c.sub > 2 * kTile && waves(c.sub) < waves_for(elem_bytes)) c.sub /= 2;
    // rooms of a padded batch begin where stretches of their length do, forward + backward on one state, half of the rooms' rows there: 2048 of 50 x 201 float32 36 +
    // 68 us for 45 + 92, 1024 of 64 x 256 bfloat16 32 + 48 for 39 + 61, 4096 of 50 56 + 105 for 82 + 147.  A ragged batch whose mean length is such a whole number cannot be
    // told from it: 4096 of 50 on average 106 + 167 for 118 + 194, 1400 61 + 86 for 57 + 88, but 1024 of 64, the fewest waves that are let, 68 + 103 for 44 + 67;
    // with fewer still it costs more (262144 x 16 bfloat16 in 4096 ragged sequences, 512 waves: 91 + 131 for 40 + 52)
    const int64_t room = !dense && sequences > 0 && rows % sequences == 0 ? rows / sequences : 0;
    if (room >= kRoom && room <= kSub && waves(room) >= 1024) c.sub = room;
  }
  c.chunk = c.sub * walkers;
  c.chunks = std::max<int64_t>(1, (rows + c.chunk - 1) / c.chunk);
  c.one = c.chunks == 1 || c.whole;
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
  a.tiles = c.tiles, a.sub = c.sub, a.chunk_rows = c.chunk, a.chunks = c.chunks, a.whole = c.whole, a.one = c.one;
  a.stretch = (float2*)workspace;
  a.chunk = (float2*)((char*)workspace + stretch_bytes(c, a.cols));
  a.forgets = (int*)((char*)a.chunk + chunk_bytes(c, a.cols));
  return DMT_OK;
}

template <typename Kernel> void launch(Kernel kernel, const Scan& a, hipStream_t s) {
  dmt_launches(a.chunks * a.tiles, kBlock,
               [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, a, first); });
}

template <int G, int XD> void run_fwd(const Scan& a, bool free, hipStream_t s) {
  if (free) {
    if (!a.one) launch(scan_stretches<G, XD, XD, false, true>, a, s);
    launch(scan_fwd<G, XD, true>, a, s);
  } else {
    if (!a.one) launch(scan_stretches<G, XD, XD, false, false>, a, s);
    launch(scan_fwd<G, XD, false>, a, s);
  }
}
template <int G, int XD, int GD> void run_bwd(const Scan& a, bool free, hipStream_t s) {
  if (!a.one) launch(scan_stretches<G, XD, GD, true, false>, a, s);      // (l does not depend on u)
  if (free) launch(scan_bwd<G, XD, GD, true>, a, s);
  else launch(scan_bwd<G, XD, GD, false>, a, s);
}
template <typename Run> void by_group(const Cut& c, Run run) {
  if (c.narrow) run(Int<0>());
  else if (c.group == 8) run(Int<8>());
  else if (c.group == 16) run(Int<16>());
  else if (c.group == 32) run(Int<32>());
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
  // of either type, and with the shortest stretch that rooms can bring
  size_t most = 0;
  for (int elem_bytes : {2, 4}) {
    Cut c = cut_of(rows, cols, elem_bytes, false, 0);
    if (!c.one && c.sub > kRoom) {
      c.chunk = c.chunk / c.sub * kRoom;
      c.chunks = (rows + c.chunk - 1) / c.chunk;
    }
    most = std::max(most, scratch_bytes(c, cols));
  }
  return most;
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
  a.initial = initial, a.final = final, a.kept = (float*)kept, a.first_bad = (unsigned long long*)first_bad;
  const Cut c = cut_of(rows, cols, (int)dmt_ebytes(dtype), !sequence_of, sequences);
  const dmt_status room = place(a, c, workspace, workspace_bytes);
  if (room != DMT_OK) return room;
  by_group(c, [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (dtype == DMT_F32) run_fwd<G, DMT_F32>(a, form == DMT_SCAN_FREE, (hipStream_t)stream);
    else if (dtype == DMT_F16) run_fwd<G, DMT_F16>(a, form == DMT_SCAN_FREE, (hipStream_t)stream);
    else run_fwd<G, DMT_BF16>(a, form == DMT_SCAN_FREE, (hipStream_t)stream);
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
  a.initial = initial, a.dfinal = dfinal, a.dinitial = dinitial, a.kept = (float*)kept;
  const Cut c = cut_of(rows, cols, (int)dmt_ebytes(dtype), !sequence_of, sequences);
  const dmt_status room = place(a, c, workspace, workspace_bytes);
  if (room != DMT_OK) return room;
  hipStream_t s = (hipStream_t)stream;
  by_group(c, [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (dtype == DMT_F32) run_bwd<G, DMT_F32, DMT_F32>(a, form == DMT_SCAN_FREE, s);
    else if (dtype == DMT_F16 && grad_dtype == DMT_F16) run_bwd<G, DMT_F16, DMT_F16>(a, form == DMT_SCAN_FREE, s);
    else if (dtype == DMT_F16) run_bwd<G, DMT_F16, DMT_F32>(a, form == DMT_SCAN_FREE, s);
    else if (grad_dtype == DMT_BF16) run_bwd<G, DMT_BF16, DMT_BF16>(a, form == DMT_SCAN_FREE, s);
    else run_bwd<G, DMT_BF16, DMT_F32>(a, form == DMT_SCAN_FREE, s);
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
    // without slots as many rows as give every thread four pieces
    const int64_t want = slots ? rows / 512 : 4 * kStepBlock * 4 / cols;
    const int per = (int)std::min<int64_t>(kStepRows, std::max<int64_t>(1, slots ? want : std::min(want, rows / 512)));
    dmt_launches((rows + per - 1) / per, kStepBlock,
                 [&](unsigned first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kStepBlock), 0, s, a, per, first); });
  };
  const bool many = slots && rows >= 1024;
  if (dtype == DMT_F32) many ? go(scan_step<DMT_F32, true>) : go(scan_step<DMT_F32, false>);
  else if (dtype == DMT_F16) many ? go(scan_step<DMT_F16, true>) : go(scan_step<DMT_F16, false>);
  else many ? go(scan_step<DMT_BF16, true>) : go(scan_step<DMT_BF16, false>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
