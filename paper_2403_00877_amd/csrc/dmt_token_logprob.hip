// dmt_token_logprob_fwd, dmt_token_logprob_bwd: rows of scores as distributions.
//   M = max x, S = sum exp(x - M), T = sum exp(x - M) (x - M):  log p_j = x_j - M - log S,  H = log S - T / S.
//
// Forward, one pass over the scores.  A block takes a span of a row, 8 KB at a time in registers; every lane keeps a maximum, S
// and T of its own and rescales them when its maximum grows.  Exponents are kept to the base 2: z = x log2 e - M log2 e is one
// fused multiply-add; M's product is rounded once and the same in every term (and in the backward), at most 1/16 from what it should
// be, so its error cancels.  Beyond |M| = 2^20, where it would grow, z = (x - M) log2 e, and a sum that crosses that line is
// brought to the other side's terms.
// The top k: each wave holds its 64 best so far, sorted, one a lane, and looks singly at few scores only, those above a bound that at
// least k scores reach.  The bound is the k-th largest of 64 maxima, the columns of all waves' running maxima, taken after pieces
// 1, 2, 4, 8 ... of a span: of 13 pieces and k = 20 some 25 scores of a wave are looked at, where each wave's own k-th best let 75 through
// (512 x 100003 float16: 34.8 us for 41.1, 2.9 TB/s; 622 x 107750 float32, k = 1: 52 for 71).  What is left is mostly arithmetic: the
// sums of 16-bit scores take some 16 of the 35 us.
// Rows are cut into spans when they are too few to fill the chip; a second launch joins the spans.
#include <algorithm>
#include <type_traits>

#include "dmt_internal.h"
#include "dmt_rows.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;
constexpr int kVecs = 2;                                   // 16-byte pieces of a lane under way
constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.693147180559945f;
constexpr float kFar = 0x1p20f;                            // |M| beyond which M log2 e is not rounded but taken after the difference
constexpr float kApart = 1e30f;                            // distances (and gradients) beyond which a few products may overflow
constexpr float kNone = -200.f;                            // 2^kNone is 0: stands for exponents down to -inf

// of W waves
template <int DT, int W = kWaves> constexpr int piece_elems() { return W * 64 * kVecs * dmt::ChunkElems<DT>::value; }

// The largest float below x (x itself, where that is -inf).
__device__ __forceinline__ float just_below(float x) {
  const uint32_t u = __float_as_uint(x);
  return x == -kInf ? x : x == 0.f ? -__uint_as_float(1u) : __uint_as_float(x > 0.f ? u - 1 : u + 1);
}

// (x - m) log2 e + residue(m);  m is not -inf.
__device__ __forceinline__ float exponent(float x, float m) {
  return fabsf(m) > kFar ? (x - m) * kLog2e : fmaf(x, kLog2e, -(m * kLog2e));
}
// What the rounding of m's product adds to every exponent, exactly; |residue| <= 1/16.
__device__ __forceinline__ float residue(float m) { return fabsf(m) > kFar ? 0.f : fmaf(m, kLog2e, -(m * kLog2e)); }
__device__ __forceinline__ float or_zero(float m) { return m == -kInf ? 0.f : m; }

// log p of score x;  ls = log2 S.  (Far below M, exponents of 2 would overflow before natural ones do.)
__device__ __forceinline__ float log_prob(float x, float m, float ls) {
  return fabsf(x - m) > kApart ? x - m - ls * kLn2 : (exponent(x, m) - ls) * kLn2;
}

struct Sum {
  float m, s, t;                                           // t in units of ln 2
};

// What `a` is with the maximum m (>= a.m).  Its terms hold a.m's residue and get m's; equal maxima leave the sums as they are.
__device__ __forceinline__ void rescale(Sum& a, float m) {
  const float by = (a.m - m) * kLog2e + (residue(m) - residue(a.m));
  const float d = a.m == -kInf ? kNone : by, f = __builtin_amdgcn_exp2f(d);
  a.t = f == 0.f ? 0.f : f * fmaf(d, a.s, a.t);
  a.s *= f;                                                // (a NaN stays)
  a.m = m;
}

// ------------------------------------------------------------------ sorted lists, one entry a lane

// An entry orders by score, then by the lower item: larger entries are better, 0 is none.  Between spans it is the float32 score
// and the item, 64 bits; inside a span of 16-bit scores the score itself and the item's distance from the span's begin, 32 bits.
__device__ __forceinline__ uint64_t entry(float v, uint32_t item) {
  const uint32_t u = __float_as_uint(v == 0.f ? 0.f : v);  // (zeros of both signs tie)
  return (uint64_t)((u >> 31) ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - item);
}
__device__ __forceinline__ float entry_score(uint64_t e) {
  const uint32_t u = (uint32_t)(e >> 32);
  return e == 0 ? -kInf : __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint32_t entry_item(uint64_t e) { return 0xffffffffu - (uint32_t)e; }

template <int DT> struct Local {                           // inside a span
  static constexpr int kMost = 65536;                      // scores of a span, at most
  using type = uint32_t;
  static __device__ __forceinline__ type make(float v, int at) {
    uint32_t u = v == 0.f ? 0u : dmt::round2<DT>(v, 0.f) & 0xffffu;
    return ((u >> 15) ? ~u & 0xffffu : u | 0x8000u) << 16 | (0xffffu - (uint32_t)at);
  }
  static __device__ __forceinline__ float score(type e) {
    const uint32_t u = e >> 16, bits = (u >> 15) ? u & 0x7fffu : ~u & 0xffffu;
    if (e == 0) return -kInf;
    if constexpr (DT == DMT_BF16) return dmt::bf16_lo(bits);
    else return dmt::f16_bits_to_f32(bits);
  }
  static __device__ __forceinline__ uint64_t wide(type e, int begin) {
    return e ? entry(score(e), (uint32_t)begin + 0xffffu - (e & 0xffffu)) : 0;
  }
};
template <> struct Local<DMT_F32> {
  static constexpr int kMost = 1 << 30;
  using type = uint64_t;
  static __device__ __forceinline__ type make(float v, int at) { return entry(v, (uint32_t)at); }
  static __device__ __forceinline__ float score(type e) { return entry_score(e); }
  static __device__ __forceinline__ uint64_t wide(type e, int begin) { return e ? e - (uint32_t)begin : 0; }
};

template <typename V> __device__ __forceinline__ V larger(V a, V b) { return a > b ? a : b; }

// One step of a bitonic network: lanes O apart, those with KEEP's bit set take the larger value.
template <int O, uint64_t KEEP, typename V> __device__ __forceinline__ V exchange(V v) {
  const V w = dmt::lane_xor<O>(v);
  return __builtin_amdgcn_inverse_ballot_w64(KEEP) == (v > w) ? v : w;
}
// The lanes whose bit N is 0.
constexpr uint64_t lanes_without(int n) {
  uint64_t m = 0;
  for (int i = 0; i < 64; ++i) m |= (uint64_t)((i & n) == 0) << i;
  return m;
}
// A sequence that rises, then falls (or the other way round) into falling order.
template <int O = 32, typename V> __device__ __forceinline__ V merge_falling(V v) {
  v = exchange<O, lanes_without(O)>(v);
  if constexpr (O > 1) v = merge_falling<O / 2>(v);
  return v;
}
// Blocks of N lanes (rising and falling by turns) into such blocks of 2 N ... 64.
template <bool Falling, int N, int O, typename V> __device__ __forceinline__ V sort_steps(V v) {
  constexpr uint64_t up = Falling ? lanes_without(N) : ~lanes_without(N);
  v = exchange<O, ~(lanes_without(O) ^ up)>(v);
  if constexpr (O > 1) return sort_steps<Falling, N, O / 2>(v);
  else if constexpr (N < 64) return sort_steps<Falling, N * 2, N>(v);
  else return v;
}
template <typename V, bool Falling> __device__ __forceinline__ V sort64(V v) { return sort_steps<Falling, 2, 1>(v); }
// The 64 best of a falling list and of 64 entries in any order.
template <typename V> __device__ __forceinline__ V add64(V list, V more) {
  return merge_falling(larger(list, sort64<V, false>(more)));
}

// The waves' lists into one, in wave 0.  lds [kWaves][64].
template <typename V> __device__ __forceinline__ V join_lists(V list, V (*lds)[64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  lds[wave][lane] = list;
  __syncthreads();
  if (wave == 0)
    for (int w = 1; w < kWaves; ++w) list = merge_falling(larger(list, lds[w][63 - lane]));
  return list;
}

// A wave's sums into one, the same in every lane.
__device__ __forceinline__ Sum join_lanes(Sum a) {
  rescale(a, dmt::group_max<64>(a.m));
  a.s = dmt::group_sum<64>(a.s);
  a.t = dmt::group_sum<64>(a.t);
  return a;
}
// The block's threads' into one, the same in every thread.  Ends with a barrier.
__device__ __forceinline__ Sum join_sums(Sum a, float (*lds)[3]) {
  a = join_lanes(a);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) lds[wave][0] = a.m, lds[wave][1] = a.s, lds[wave][2] = a.t;
  __syncthreads();
  Sum all = {-kInf, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) all.m = fmaxf(all.m, lds[w][0]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Sum b = {lds[w][0], lds[w][1], lds[w][2]};
    rescale(b, all.m);
    all.s += b.s;
    all.t += b.t;
  }
  __syncthreads();
  return all;
}

// ------------------------------------------------------------------ forward

struct Fwd {
  const char* x;
  int64_t stride, rows;
  int vocab, k, spans, span;                               // span: elements, a multiple of the piece
  unsigned first_block;                                    // of the launch, among the call's
  const int32_t* targets;
  float *logprob, *entropy, *stats;
  int32_t* top_ids;
  float* top_logprobs;
  unsigned long long* first_bad;
  float4* part;                                            // [row][span] sums
  uint64_t* lists;                                         // [row][span][k]
};

// A row's answers from its sums (known to every thread) and its list (its first wave's), by the threads `tid` from 0 on.
template <int DT>
__device__ __forceinline__ void finish(const Fwd& a, int64_t row, int tid, const Sum& all, uint64_t list) {
  constexpr int EB = dmt::EltBytes<DT>::value;
  const bool empty = all.s == 0.f;
  const float m = or_zero(all.m), ls = log2f(all.s);
  if (tid == 0) {
    const int32_t at = a.targets ? a.targets[row] : -1;
    if (at >= a.vocab && a.first_bad) atomicMin(a.first_bad, (unsigned long long)row);
    if (a.logprob)
      a.logprob[row] = at < 0 || at >= a.vocab ? 0.f
                       : empty                 ? -kInf
                                               : log_prob(dmt::load1<DT>(a.x + (row * a.stride + at) * EB), m, ls);
    if (a.entropy) a.entropy[row] = empty ? 0.f : (ls - all.t / all.s) * kLn2;
    if (a.stats) a.stats[2 * row] = all.m, a.stats[2 * row + 1] = all.s * __builtin_amdgcn_exp2f(-residue(m));
  }
  if (tid < a.k) {
    a.top_ids[row * a.k + tid] = list ? (int32_t)entry_item(list) : -1;
    if (a.top_logprobs) a.top_logprobs[row * a.k + tid] = list ? log_prob(entry_score(list), m, ls) : -kInf;
  }
}

// A piece of a row (8 KB for a block) from element j on, -inf behind `end`.
template <int DT, bool Once = false, int W = kWaves>
__device__ __forceinline__ void load_piece(const char* row, int j, int end, dmt::Raw<DT, dmt::ChunkElems<DT>::value> (&r)[kVecs]) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value, kWords = dmt::Raw<DT, E>::kWords;
  constexpr uint32_t kMasked = DT == DMT_F32 ? 0xff800000u : DT == DMT_F16 ? 0xfc00fc00u : 0xff80ff80u;
  const int tid = (int)threadIdx.x % (W * 64);
  if (j + piece_elems<DT, W>() <= end) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
      r[v] = dmt::load_raw<DT, E, Once>(row + ((int64_t)j + (v * W * 64 + tid) * E) * EB, E);
    return;
  }
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    const int at = j + (v * W * 64 + tid) * E, valid = end - at;
    if (valid > 0) r[v] = dmt::load_raw<DT, E>(row + (int64_t)at * EB, valid);
    if (valid < E) {
#pragma unroll
      for (int q = 0; q < kWords; ++q) {
        if constexpr (DT == DMT_F32) {
          if (q >= valid) r[v].w[q] = kMasked;
        } else {
          if (q * 2 >= valid) r[v].w[q] = kMasked;
          else if (q * 2 + 1 >= valid) r[v].w[q] = (r[v].w[q] & 0xffffu) | (kMasked & 0xffff0000u);
        }
      }
    }
  }
}

// Once: the scores pass the caches by.  W: waves of a row; with one a block takes four whole rows, and nothing crosses waves.
template <int DT, bool Top, bool Once, int W>
__global__ __launch_bounds__(kBlock, Top ? 4 : 5) void logprob_spans(const Fwd a) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value;
  __shared__ float s_sum[kWaves][3];
  using Entry = typename Local<DT>::type;
  __shared__ Entry s_list[Top ? kWaves : 1][64];
  __shared__ int s_buf[Top ? kWaves : 1][128];             // each wave's candidates, by their distance from `begin`: less than 64, and 64
  constexpr int kPiece = piece_elems<DT, W>();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const unsigned block = a.first_block + blockIdx.x;
  const int64_t row = W == 1 ? (int64_t)block * kWaves + wave : block / (unsigned)a.spans;
  const int span = W == 1 ? 0 : (int)(block % (unsigned)a.spans);
  if (W == 1 && row >= a.rows) return;
  const int tid = (int)threadIdx.x % (W * 64);
  const char* x = a.x + row * a.stride * EB;
  const int begin = span * a.span, end = min(a.vocab, begin + a.span);
  Sum sum = {-kInf, 0.f, 0.f};
  Entry list = 0;
  float cut = -kInf;                                       // scores up to it are not among the k best
  int waiting = 0;
  int* buf = s_buf[Top ? wave : 0];
  __shared__ float s_best[Top ? 2 : 1][kWaves][64];        // the lanes' maxima; two sets by turns, so that one barrier does
  // (one piece: each wave by itself, 6.1 us for 6.5; but k = 50 8192 x 1000 48 for 38)
  const bool shared = W == 1 || end - begin > kPiece || a.k > 32;
  int piece = 0;
  // the next piece is requested ahead (without: 319 x 209950 float16, k = 5: 43.9 us for 41.8; 512 x 100003, k = 20: 35.6 for 34.8)
  dmt::Raw<DT, E> r[kVecs], next[kVecs];
  load_piece<DT, Once, W>(x, begin, end, next);
  for (int j = begin; j < end; j += kPiece) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) r[v] = next[v];
    if (j + kPiece < end) load_piece<DT, Once, W>(x, j + kPiece, end, next);
    float pm = -kInf;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      float e[E];
      dmt::unpack<DT, E>(r[v], e);
#pragma unroll
      for (int q = 0; q < E; ++q) pm = fmaxf(pm, e[q]);
    }
    if (pm > sum.m) rescale(sum, pm);
    const float m = or_zero(sum.m), m2 = m * kLog2e;
    auto add = [&](auto z) {
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        float e[E];
        dmt::unpack<DT, E>(r[v], e);
#pragma unroll
        for (int q = 0; q < E; ++q) {
          const float d = z(e[q]), p = __builtin_amdgcn_exp2f(d);
          sum.s += p;
          sum.t = fmaf(p, fmaxf(d, kNone), sum.t);
        }
      }
    };
    if (__any(fabsf(m) > kFar)) add([&](float v) { return exponent(v, m); });
    else add([&](float v) { return fmaf(v, kLog2e, -m2); });
    if constexpr (Top) {
      const bool last = j + kPiece >= end;
      float low = cut;                                     // of this piece, candidates are above it
      if (shared && (piece & (piece + 1)) == 0) {
        // after pieces 1, 2, 4, 8 ...: at least k scores of the span so far reach the k-th largest of 64 maxima, each of a lane of
        // every wave; in this piece equal ones may have lower items
        float of = sum.m;
        if constexpr (W > 1) {
          float(*best)[64] = s_best[__popc((uint32_t)piece) & 1];
          best[wave][lane] = sum.m;
          __syncthreads();
          of = best[0][lane];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) of = fmaxf(of, best[w][lane]);
        }
        const float bound = __shfl(sort64<float, true>(of), a.k - 1);
        low = fmaxf(low, just_below(bound));
        cut = fmaxf(cut, bound);
      }
      ++piece;
      const uint64_t over = __ballot(pm > low);
      if (over || (last && waiting > 0)) {
        if (__popcll(over) >= max(a.k, 12)) low = fmaxf(low, just_below(__shfl(sort64<float, true>(pm), a.k - 1)));
        uint32_t found = 0;                                // which of the lane's scores are above it
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
          float e[E];
          dmt::unpack<DT, E>(r[v], e);
#pragma unroll
          for (int q = 0; q < E; ++q) found |= (uint32_t)(e[q] > low) << (v * E + q);
        }
        // one of each lane's at a time (few lanes have one, fewer two: taking them from the registers, a ballot and a branch for
        // each of those, was most of the kernel's instructions); the scores are read again when they go into the list
        for (;;) {
          const uint64_t mask = __ballot(found != 0);
          if (found) {
            const int slot = __builtin_ctz(found);
            found &= found - 1;
            buf[waiting + __popcll(mask & ((1ull << lane) - 1))] = j - begin + (slot / E * W * 64 + tid) * E + slot % E;
          }
          __builtin_amdgcn_wave_barrier();
          waiting += __popcll(mask);
          // a full wave of them goes into the list, or what there is after the last piece
          if (waiting >= 64 || (!mask && last && waiting > 0)) {
            const int from = max(0, waiting - 64);
            const int at = buf[min(from + lane, 127)];
            const Entry e = from + lane < waiting ? Local<DT>::make(dmt::load1<DT>(x + ((int64_t)begin + at) * EB), at) : 0;
            __builtin_amdgcn_wave_barrier();
            waiting = from;
            list = add64(list, e);
          }
          if (!mask) break;
        }
        // later pieces hold later items only: a score has to beat the k-th
        cut = fmaxf(cut, __shfl(Local<DT>::score(list), a.k - 1));
      }
    }
  }
  if constexpr (W == 1) {
    sum = join_lanes(sum);
  } else {
    sum = join_sums(sum, s_sum);
    if constexpr (Top) list = join_lists(list, s_list);
  }
  if (W == 1 || a.spans == 1) {
    finish<DT>(a, row, tid, sum, Local<DT>::wide(list, begin));
  } else {
    const int64_t at = row * a.spans + span;
    if (tid == 0) a.part[at] = make_float4(sum.m, sum.s, sum.t, 0.f);
    if (Top && tid < a.k) a.lists[at * a.k + tid] = Local<DT>::wide(list, begin);
  }
}

// A row's spans into one.
template <int DT, bool Top>
__global__ __launch_bounds__(kBlock) void logprob_join(const Fwd a) {
  __shared__ float s_sum[kWaves][3];
  __shared__ uint64_t s_list[kWaves][64];
  const int64_t row = a.first_block + blockIdx.x;
  Sum sum = {-kInf, 0.f, 0.f};
  for (int i = threadIdx.x; i < a.spans; i += kBlock) {
    const float4 p = a.part[row * a.spans + i];
    Sum b = {p.x, p.y, p.z};
    const float m = fmaxf(sum.m, b.m);
    rescale(sum, m);
    rescale(b, m);
    sum.s += b.s;
    sum.t += b.t;
  }
  uint64_t list = 0;
  if constexpr (Top) {
    const int count = a.spans * a.k, lane = threadIdx.x & 63;
    const uint64_t* from = a.lists + row * a.spans * a.k;
    for (int i = (int)(threadIdx.x >> 6) * 64; i < count; i += kBlock) {
      const uint64_t e = i + lane < count ? from[i + lane] : 0;
      if (__any(e > __shfl(list, a.k - 1))) list = add64(list, e);
    }
    list = join_lists(list, s_list);
  }
  sum = join_sums(sum, s_sum);
  finish<DT>(a, row, (int)threadIdx.x, sum, list);
}

// ------------------------------------------------------------------ backward

// dx = p (A + B z) with p = exp2(z) / S, z to the base 2:  A = -g_lp - g_H (H - log S),  B = -g_H ln 2, S with the residue that
// the terms here have and the kept sum has not.  A block takes a piece of a row; bound by memory: 8192 x 65536 bfloat16 355 us,
// 6.0 TB/s, behind a forward of 176 (6.1, from past the caches); in a train of twenty passes 363 and 190 to 225.
template <int DT>
__global__ __launch_bounds__(kBlock) void logprob_bwd(unsigned first_block, const char* x, int vocab, int64_t stride, int pieces,
                                                      const int32_t* __restrict__ targets,
                                                      const float* __restrict__ stats,
                                                      const float* __restrict__ entropy,
                                                      const float* __restrict__ grad_logprob,
                                                      const float* __restrict__ grad_entropy, char* dx,
                                                      int64_t dx_stride) {
  constexpr int E = dmt::ChunkElems<DT>::value, EB = dmt::EltBytes<DT>::value;
  const unsigned block = first_block + blockIdx.x;
  const int64_t row = block / (unsigned)pieces;
  const int j = (int)(block % (unsigned)pieces) * piece_elems<DT>();
  const char* xr = x + row * stride * EB;
  char* dr = dx + row * dx_stride * EB;
  dmt::Raw<DT, E> r[kVecs];
  load_piece<DT>(xr, j, vocab, r);
  const float m = or_zero(stats[2 * row]), s = stats[2 * row + 1] * __builtin_amdgcn_exp2f(residue(m)), inv = s == 0.f ? 0.f : 1.f / s;
  const int32_t at = targets ? targets[row] : -1;
  const float gl = grad_logprob && at >= 0 && at < vocab ? grad_logprob[row] : 0.f;
  const float gh = grad_entropy && s != 0.f ? grad_entropy[row] : 0.f, h = grad_entropy ? entropy[row] : 0.f;
  const float A = s == 0.f ? 0.f : (-gl - gh * (h - logf(s))) * inv, B = -gh * kLn2 * inv, m2 = m * kLog2e;
  auto grads = [&](auto z, auto masks) {
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int c = j + (v * kBlock + (int)threadIdx.x) * E;
      if (c >= vocab) break;
      float e[E], d[E];
      dmt::unpack<DT, E>(r[v], e);
#pragma unroll
      for (int q = 0; q < E; ++q) {
        const float w = z(e[q]);
        d[q] = __builtin_amdgcn_exp2f(w) * fmaf(B, fmaxf(w, kNone), A);
        if (decltype(masks)::value && e[q] == -kInf) d[q] = 0.f;
      }
      if (gl != 0.f && (uint32_t)(at - c) < (uint32_t)E) {
#pragma unroll
        for (int q = 0; q < E; ++q)
          if (c + q == at && e[q] != -kInf) d[q] += gl;
      }
      dmt::store_elems<DT, E>(dr + (int64_t)c * EB, min(E, vocab - c), d);
    }
  };
  // a masked score's exponential is 0, which is its gradient as long as the other factor is finite
  if (!(fabsf(A) < kApart && fabsf(B) < kApart)) grads([&](float v) { return exponent(v, m); }, std::true_type());
  else if (fabsf(m) > kFar) grads([&](float v) { return exponent(v, m); }, std::false_type());
  else grads([&](float v) { return fmaf(v, kLog2e, -m2); }, std::false_type());
}

// A row is cut into equal spans of whole pieces while the blocks are fewer than fit the chip at once: eight of a CU, with the lists four
// (512 x 100003, k = 20: 35 us with 1024 blocks, 40 with 2048), and then as near to that as whole spans come (1003 x 12000, k = 20: 14.9 us
// in one span each, 18.2 + 5.3 in two).  Short rows stay whole, which saves the second launch, the time of some 4.5 pieces with lists (60 x
// 12000 bfloat16, k = 20, 3 pieces: 8.9 us for 10.6; 400 x 12000 float32, 6 pieces, three spans: 12.6 for 16.7; 60 x 12000 float32, six spans:
// 11.5 for 11.1) and of some 16 without (12000 float32: 7 us for 10; 60 x 30000 float32, 15 pieces: 7.7 for 10.0; 60 x 60000 bfloat16, 15:
// 10.7 for 9.8; 400: 15.5 for 17.1).  And a row's lists stay below kMostEntries, which the second launch sorts:
// 262144 scores, k = 50: 10 + 10 us in 32 spans, 7 + 17 in 64.
struct Spans {
  int spans, span;
};
constexpr int64_t kFillBlocks = 2048, kFillTop = 1024, kLeastPieces = 4, kMostEntries = 2048;
constexpr int64_t kCacheBytes = 256 << 20;
Spans spans_of(int64_t rows, int64_t vocab, int64_t piece, int k, int64_t most) {
  const int64_t pieces = (vocab + piece - 1) / piece, fill = k > 0 ? kFillTop : kFillBlocks;
  int64_t want = std::min(pieces, k > 0 ? std::max<int64_t>(1, (fill + rows / 2) / rows) : (fill + rows - 1) / rows);
  if (k > 0) want = std::min(want, kMostEntries / k);
  int64_t per = (pieces + want - 1) / want;
  if (2 * pieces * (want - 1) <= (k > 0 ? 9 : 32) * want) per = pieces;      // (the spans would save less than 4.5 pieces' time, or 16)
  else if (k == 0) per = std::max(per, std::min(kLeastPieces, pieces));
  per = std::min(per, most / piece);
  const int64_t spans = (pieces + per - 1) / per;
  return {(int)spans, (int)((pieces + spans - 1) / spans * piece)};
}

// Whole rows, a wave each: nothing to join across waves, but fewer loads of a row under way and coarser shares.  Rows of a wave's own piece, and
// while there are waves for half the chip (lists) or all of it: 8192 x 1000 float32, k = 10 17.7 us for 36.7; 2500 x 4000, k = 10 13.9 for
// 15.8, no lists 16.8 for 15.4; 8192 x 8000 bfloat16, k = 10 42.6 for 55.0, no lists 83.0 for 85.5 with the backward; lists of long rows: 9000 x
// 30000 123 for 137, but 2500 x 30000 60 for 51; long rows without: 8192 x 65536 187 for 168.
bool wave_a_row(int64_t rows, int64_t vocab, int64_t piece, int k) {
  const int64_t pieces = rows >= 4096 ? (k > 0 ? 16 : 4) : rows >= 2048 && k > 0 ? 4 : 0;
  return vocab <= std::max(piece / kWaves, pieces * piece);
}

// Sums and lists of so many spans.
size_t part_bytes(int64_t spans, int k) {
  return dmt_align_up(sizeof(float4) * (size_t)spans, 256) + sizeof(uint64_t) * (size_t)spans * (size_t)k;
}

bool fits(int64_t rows, int64_t vocab) { return rows < (1ll << 31) && vocab <= (1ll << 30); }

}  // namespace

extern "C" size_t dmt_token_logprob_workspace_bytes(int64_t rows, int64_t vocab, int32_t k) {
  if (rows < 0 || vocab < 1 || k < 0 || k > DMT_TOP_MAX || !fits(rows, vocab)) return 0;
  // the most that any type, and any fewer rows, can need
  const int64_t pieces = (vocab + piece_elems<DMT_F32>() - 1) / piece_elems<DMT_F32>();
  const int64_t least = (vocab + Local<DMT_BF16>::kMost - 1) / Local<DMT_BF16>::kMost;
  return part_bytes(std::min(rows * pieces, kFillBlocks + rows * least), k);
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
  const int64_t piece = dtype == DMT_F32 ? piece_elems<DMT_F32>() : piece_elems<DMT_BF16>();
  if (rows == 0) return DMT_OK;
  const Spans sp = spans_of(rows, vocab, piece, k, k > 0 && dtype != DMT_F32 ? Local<DMT_BF16>::kMost : 1 << 30);
  if (rows * sp.spans >= (1ll << 31)) return DMT_ENOTSUP;
  if (sp.spans > 1) {
    if (!dmt_is_at(workspace, 256)) return DMT_EINVAL;
    if (workspace_bytes < part_bytes(rows * sp.spans, k)) return DMT_ENOMEM;
  }
  Fwd a = {};
  a.x = (const char*)x, a.stride = x_stride, a.rows = rows, a.vocab = (int)vocab, a.k = k, a.spans = sp.spans, a.span = sp.span;
  a.targets = targets, a.logprob = logprob, a.entropy = entropy, a.stats = stats;
  a.top_ids = top_ids, a.top_logprobs = top_logprobs, a.first_bad = (unsigned long long*)first_bad;
  a.part = (float4*)workspace;
  a.lists = (uint64_t*)((char*)workspace + dmt_align_up(sizeof(float4) * (size_t)rows * sp.spans, 256));
  const bool narrow = sp.spans == 1 && wave_a_row(rows, vocab, piece, k);
  auto launch = [&](auto kernel, int64_t blocks) {
    dmt_launches(blocks, kBlock, [&](unsigned first, dim3 grid) {
      a.first_block = first;
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, (hipStream_t)stream, a);
    });
  };
  auto go = [&](auto spans, auto spans_narrow, auto join) {
    if (narrow) launch(spans_narrow, (rows + kWaves - 1) / kWaves);
    else launch(spans, rows * sp.spans);
    if (sp.spans > 1) launch(join, rows);
  };
  auto type = [&](auto top, auto once) {
    constexpr bool Top = decltype(top)::value, Once = decltype(once)::value;
    auto of = [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      go(logprob_spans<DT, Top, Once, kWaves>, logprob_spans<DT, Top, Once, 1>, logprob_join<DT, Top>);
    };
    if (dtype == DMT_F32) of(std::integral_constant<int, DMT_F32>());
    else if (dtype == DMT_F16) of(std::integral_constant<int, DMT_F16>());
    else of(std::integral_constant<int, DMT_BF16>());
  };
  // Scores that the Infinity Cache does not hold for the backward need not pass through it: 1 GiB, forward 239 -> 212 us (its
  // backward 348 -> 363); 64 MiB would be 17.0 for 17.0 and the backward 22.8 for 21.6.
  const bool once = (double)rows * (double)vocab * (double)dmt_ebytes(dtype) > (double)kCacheBytes;
  if (k > 0) type(std::true_type(), std::false_type());
  else if (once) type(std::false_type(), std::true_type());
  else type(std::false_type(), std::false_type());
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
  const int64_t piece = dtype == DMT_F32 ? piece_elems<DMT_F32>() : piece_elems<DMT_BF16>();
  const int64_t pieces = (vocab + piece - 1) / piece;
  if (rows * pieces >= (1ll << 31)) return DMT_ENOTSUP;
  auto go = [&](auto kernel) {
    dmt_launches(rows * pieces, kBlock, [&](unsigned first, dim3 grid) {
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, (hipStream_t)stream, first, (const char*)x, (int)vocab, x_stride, (int)pieces,
                         targets, stats, entropy, grad_logprob, grad_entropy, (char*)dx, dx_stride);
    });
  };
  if (dtype == DMT_F32) go(logprob_bwd<DMT_F32>);
  else if (dtype == DMT_F16) go(logprob_bwd<DMT_F16>);
  else go(logprob_bwd<DMT_BF16>);
  return hipGetLastError() == hipSuccess ? DMT_OK : DMT_EHIP;
}
