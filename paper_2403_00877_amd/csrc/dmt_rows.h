// Rows of matrices with any stride and alignment: pieces of up to 16 bytes a lane from any
// element on, float32 values in between, one rounding on the way out.
#pragma once

#include "dmt_device_utils.h"

namespace dmt {

// gfx950 reads and writes a global 16-byte piece at any address; the types only tell the compiler
// that an address is a multiple of the element alone.
template <int EB> struct Piece;
template <> struct Piece<4> {
  typedef dmt_u32x4 __attribute__((aligned(4))) v4;
  typedef dmt_u32x2 __attribute__((aligned(4))) v2;
};
template <> struct Piece<2> {
  typedef dmt_u32x4 __attribute__((aligned(2))) v4;
  typedef dmt_u32x2 __attribute__((aligned(2))) v2;
};

template <int DT> __device__ __forceinline__ uint32_t round2(float a, float b) {
  if constexpr (DT == DMT_BF16) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const dmt_f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  } else {
    return pack2<DT>(a, b);
  }
}

template <int DT> __device__ __forceinline__ float load1(const char* p) {
  if constexpr (DT == DMT_F32) {
    return *(const DMT_GLOBAL float*)p;
  } else {
    const uint32_t u = *(const DMT_GLOBAL uint16_t*)p;
    if constexpr (DT == DMT_BF16) return bf16_lo(u);
    else return f16_bits_to_f32(u);
  }
}

template <int DT> __device__ __forceinline__ void store1(char* p, float v) {
  if constexpr (DT == DMT_F32) *(DMT_GLOBAL float*)p = v;
  else *(DMT_GLOBAL uint16_t*)p = (uint16_t)round2<DT>(v, 0.f);
}

// A lane's E consecutive elements as they lie in memory.
template <int DT, int E> struct Raw {
  static constexpr int kWords = E * EltBytes<DT>::value / 4;
  uint32_t w[kWords];
};

// The first `valid` of them are there (valid >= 1 .. E; the others read as zero).  Once: the line is not read again soon.
template <int DT, int E, bool Once = false>
__device__ __forceinline__ Raw<DT, E> load_raw(const char* p, int valid) {
  constexpr int EB = EltBytes<DT>::value, W = Raw<DT, E>::kWords;
  Raw<DT, E> r;
  if (valid >= E) {
    if constexpr (W == 2) {
      const dmt_u32x2 v = *(const DMT_GLOBAL typename Piece<EB>::v2*)p;
      r.w[0] = v.x, r.w[1] = v.y;
    } else {
#pragma unroll
      for (int q = 0; q < W; q += 4) {
        const DMT_GLOBAL typename Piece<EB>::v4* at = (const DMT_GLOBAL typename Piece<EB>::v4*)(p + q * 4);
        const dmt_u32x4 v = Once ? __builtin_nontemporal_load(at) : *at;
        r.w[q] = v.x, r.w[q + 1] = v.y, r.w[q + 2] = v.z, r.w[q + 3] = v.w;
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < W; ++q) r.w[q] = 0;
#pragma unroll
    for (int i = 0; i < E - 1; ++i) {
      if (i < valid) {
        if constexpr (EB == 4) r.w[i] = *(const DMT_GLOBAL uint32_t*)(p + i * 4);
        else r.w[i / 2] |= (uint32_t) * (const DMT_GLOBAL uint16_t*)(p + i * 2) << (i % 2 * 16);
      }
    }
  }
  return r;
}

template <int DT, int E>
__device__ __forceinline__ void unpack(const Raw<DT, E>& r, float (&x)[E]) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if constexpr (DT == DMT_F32) {
      x[i] = __uint_as_float(r.w[i]);
    } else {
      float a, b;
      unpack2<DT>(r.w[i / 2], a, b);
      x[i] = i % 2 ? b : a;
    }
  }
}

template <int DT, int E>
__device__ __forceinline__ void load_elems(const char* p, int valid, float (&x)[E]) {
  unpack<DT, E>(load_raw<DT, E>(p, valid), x);
}

template <int DT, int E>
__device__ __forceinline__ void store_elems(char* p, int valid, const float (&x)[E]) {
  constexpr int EB = EltBytes<DT>::value, W = Raw<DT, E>::kWords;
  if (valid >= E) {
    uint32_t w[W];
#pragma unroll
    for (int q = 0; q < W; ++q) {
      if constexpr (DT == DMT_F32) w[q] = __float_as_uint(x[q]);
      else w[q] = round2<DT>(x[q * 2], x[q * 2 + 1]);
    }
    if constexpr (W == 2) {
      const dmt_u32x2 v = {w[0], w[1]};
      *(DMT_GLOBAL typename Piece<EB>::v2*)p = v;
    } else {
#pragma unroll
      for (int q = 0; q < W; q += 4) {
        const dmt_u32x4 v = {w[q], w[q + 1], w[q + 2], w[q + 3]};
        *(DMT_GLOBAL typename Piece<EB>::v4*)(p + q * 4) = v;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < E - 1; ++i)
      if (i < valid) store1<DT>(p + i * EB, x[i]);
  }
}

// The first `valid` of E float32 zeros, past the caches.
template <int E> __device__ __forceinline__ void clear_elems(char* p, int valid) {
  const dmt_u32x4 zero = {0, 0, 0, 0};
  if (valid >= E) {
#pragma unroll
    for (int q = 0; q < E; q += 4) __builtin_nontemporal_store(zero, (DMT_GLOBAL Piece<4>::v4*)(p + q * 4));
  } else {
#pragma unroll
    for (int i = 0; i < E - 1; ++i)
      if (i < valid) store1<DMT_F32>(p + i * 4, 0.f);
  }
}

// Lane ^ O's value, O a power of two below 64: by DPP inside a row of 16 lanes, by gfx950's row and half swaps
// across them (no trip through LDS, which a shuffle is).
template <int O> __device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (O == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);         // quad_perm 1 0 3 2
  else if constexpr (O == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);    // quad_perm 2 3 0 1
  else if constexpr (O == 4)                                                              // ^ 7, then ^ 3
    return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);
  else if constexpr (O == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);   // row_ror 8
  else if constexpr (O == 16) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);                  // rows 0 0 2 2, 1 1 3 3
    return threadIdx.x & 16 ? p[0] : p[1];
  } else {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);                  // low low, high high
    return threadIdx.x & 32 ? p[0] : p[1];
  }
}
template <int O> __device__ __forceinline__ float lane_xor(float v) {
  return __uint_as_float(lane_xor<O>(__float_as_uint(v)));
}
template <int O> __device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  return (uint64_t)lane_xor<O>((uint32_t)(v >> 32)) << 32 | lane_xor<O>((uint32_t)v);
}

// Sum (maximum) over the lanes of an aligned group of G lanes, the same in each of them.
template <int G> __device__ __forceinline__ float group_sum(float v) {
  if constexpr (G > 1) {
    v = group_sum<G / 2>(v);
    v += lane_xor<G / 2>(v);
  }
  return v;
}
template <int G> __device__ __forceinline__ float group_max(float v) {
  if constexpr (G > 1) {
    v = group_max<G / 2>(v);
    v = fmaxf(v, lane_xor<G / 2>(v));
  }
  return v;
}

}  // namespace dmt

// Host side: whether `dtype` is one of the three, and p aligned to it.
static inline bool dmt_is_dtype(int32_t t) { return t == DMT_F32 || t == DMT_F16 || t == DMT_BF16; }
static inline int64_t dmt_ebytes(int32_t t) { return t == DMT_F32 ? 4 : 2; }
static inline bool dmt_is_at(const void* p, int64_t align) { return p && ((uintptr_t)p & (uintptr_t)(align - 1)) == 0; }
// Whether an optional pointer is absent or aligned.
static inline bool dmt_may_be_at(const void* p, int64_t align) { return ((uintptr_t)p & (uintptr_t)(align - 1)) == 0; }

// Calls go(first block, grid) for the launches that `blocks` blocks of `threads` threads take: one is of fewer than 2^32 threads (the
// runtime starts some of the blocks of a larger one, and reports nothing).
template <typename Go> static inline void dmt_launches(int64_t blocks, int64_t threads, Go go) {
  const int64_t most = ((1ll << 32) - 1) / threads;
  for (int64_t first = 0; first < blocks; first += most)
    go((unsigned)first, dim3((unsigned)(blocks - first < most ? blocks - first : most)));
}
