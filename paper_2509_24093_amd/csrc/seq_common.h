// Device helpers of the sequence kernels: typed vector loads and stores, sums
// over groups of lanes, the 8-bit checkpoint format.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "seq.h"

namespace cgconv {
namespace seqdev {

template <int B>
struct Word;
template <>
struct Word<1> { typedef uint8_t type; };
template <>
struct Word<2> { typedef uint16_t type; };
template <>
struct Word<4> { typedef uint32_t type; };
template <>
struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <>
struct Word<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

typedef __bf16 bf16;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return (float)v; }
__device__ __forceinline__ float widen(int8_t v) { return (float)v; }

// Words of V elements at an address that is a multiple of one element only (the
// hardware's global accesses take any address).
template <class T, int V>
struct Words {
  static constexpr int kBytes = V * (int)sizeof(T), kWord = kBytes < 16 ? kBytes : 16, kWords = kBytes / kWord;
  typedef typename Word<kWord>::type W;
  typedef W Unaligned __attribute__((aligned(alignof(T))));
};

// V consecutive elements (a power of two), in accesses of at most 16 bytes.  NT:
// nontemporal, for what nobody reads again soon.
template <bool NT = false, class T, int V>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[V]) {
  typedef Words<T, V> S;
  T t[V];
#pragma unroll
  for (int i = 0; i < S::kWords; ++i) {
    const typename S::Unaligned* q = reinterpret_cast<const typename S::Unaligned*>(p) + i;
    const typename S::W w = NT ? __builtin_nontemporal_load(q) : *q;
    __builtin_memcpy(t + i * S::kWord / (int)sizeof(T), &w, sizeof w);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = widen(t[i]);
}

// The first n of V elements, zeros behind them (TAIL; else all V).
template <bool TAIL, bool NT = false, class T, int V>
__device__ __forceinline__ void load_part(const T* p, int n, float (&v)[V]) {
  if (!TAIL || n >= V) {
    load_vec<NT>(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = i < n ? widen(p[i]) : 0.f;
}

// V elements as they are stored, to be widened later: loads kept in flight take
// the registers of the storage type only.
template <class T, int V>
struct Raw {
  typedef Words<T, V> S;
  typename S::W w[S::kWords];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < S::kWords; ++i) w[i] = reinterpret_cast<const typename S::Unaligned*>(p)[i];
  }
  template <bool TAIL>
  __device__ __forceinline__ void load_part(const T* p, int n) {
    if (!TAIL || n >= V) {
      load(p);
      return;
    }
    T t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = i < n ? p[i] : (T)0;
    __builtin_memcpy(w, t, S::kBytes);
  }
  __device__ __forceinline__ void widen_to(float (&v)[V]) const {
    T t[V];
    __builtin_memcpy(t, w, S::kBytes);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = widen(t[i]);
  }
};

// Rounds to T to nearest, ties to even (nothing to round for float).
template <bool NT = false, class T, int V>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[V]) {
  typedef Words<T, V> S;
  T t[V];
#pragma unroll
  for (int i = 0; i < V; ++i) t[i] = (T)v[i];
#pragma unroll
  for (int i = 0; i < S::kWords; ++i) {
    typename S::W w;
    __builtin_memcpy(&w, t + i * S::kWord / (int)sizeof(T), sizeof w);
    typename S::Unaligned* q = reinterpret_cast<typename S::Unaligned*>(p) + i;
    if (NT)
      __builtin_nontemporal_store(w, q);
    else
      *q = w;
  }
}

template <bool TAIL, bool NT = false, class T, int V>
__device__ __forceinline__ void store_part(T* p, int n, const float (&v)[V]) {
  if (!TAIL || n >= V) {
    store_vec<NT>(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) p[i] = (T)v[i];
}

// x as a number the compiler knows nothing of: what is computed from it stays where it is,
// instead of waiting in registers for every turn of a loop.
__device__ __forceinline__ int afresh(int x) {
  asm volatile("" : "+s"(x));
  return x;
}
__device__ __forceinline__ int afresh_lane(int x) {  // x differs from lane to lane
  asm volatile("" : "+v"(x));
  return x;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

// Combines v over aligned groups of `lanes` lanes (a power of two, uniform):
// every lane of a group ends with the same value.  The partners within 16
// lanes come by DPP: quad_perm (1, 0, 3, 2), quad_perm (2, 3, 0, 1), half-row
// mirror, row mirror; after each step all lanes of a half agree, so a mirror is
// as good as an exchange.
template <class Op>
__device__ __forceinline__ float group_reduce(float v, int lanes, Op op) {
  if (lanes > 1) v = op(v, dpp<0xB1>(v));
  if (lanes > 2) v = op(v, dpp<0x4E>(v));
  if (lanes > 4) v = op(v, dpp<0x141>(v));
  if (lanes > 8) v = op(v, dpp<0x140>(v));
  if (lanes > 16) v = op(v, __shfl_xor(v, 16));
  if (lanes > 32) v = op(v, __shfl_xor(v, 32));
  return v;
}
__device__ __forceinline__ float group_sum(float v, int lanes) {
  return group_reduce(v, lanes, [](float a, float b) { return a + b; });
}

// ---- 8-bit checkpoint format -----------------------------------------------------
//
// Of every 32 channels of a row (the last group shorter) the scale s = 2^e is
// the smallest power of two, at least 2^-126, with max |x| <= 127 s; its byte is
// e + 127.  A value's code is x / s to the nearest whole number, ties to even,
// so that |x - code s| <= s / 2 <= max |x| / 127, or 2^-127 where s is the
// smallest.  Every step is exact: the codes do not depend on who computes them,
// and a bfloat16 tensor's values come back as bfloat16 without another rounding
// (7 bits of a code fit its 8).  A group that holds an infinity or NaN gets the
// byte 255 and comes back as NaN.

// bits: of max |x|.  127 s = (127/64) 2^(e + 6): a mantissa above 63/64 (0x7E0000
// of 2^23) carries into the exponent.
__device__ __forceinline__ uint32_t pack_scale(uint32_t bits) {
  const int e = (int)((bits + 0x1FFFFu) >> 23) - 6;
  return bits >= 0x7F800000u ? 255u : (uint32_t)(e < 1 ? 1 : e);
}
__device__ __forceinline__ float pack_inverse(uint32_t scale) { return __uint_as_float((254u - scale) << 23); }
__device__ __forceinline__ float unpack_scale(uint32_t scale) {
  return __uint_as_float(scale == 255u ? 0x7FC00000u : scale << 23);
}

// max over a group as bit patterns of |x| (NaN above infinity above all numbers)
__device__ __forceinline__ uint32_t group_max_bits(uint32_t v, int lanes) {
  auto step = [](uint32_t a, int b) { return a > (uint32_t)b ? a : (uint32_t)b; };
  if (lanes > 1) v = step(v, __builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  if (lanes > 2) v = step(v, __builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
  if (lanes > 4) v = step(v, __builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
  if (lanes > 8) v = step(v, __builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));
  if (lanes > 16) v = step(v, __shfl_xor((int)v, 16));
  return v;
}

template <int V>
__device__ __forceinline__ uint32_t max_bits(const float (&v)[V]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
    m = b > m ? b : m;
  }
  return m;
}

// Codes of the first n of V values under the scale byte (zeros under byte 255).
template <bool TAIL, int V>
__device__ __forceinline__ void store_codes(int8_t* p, int n, const float (&v)[V], uint32_t scale) {
  const float inv = pack_inverse(scale);
  int8_t t[V];
#pragma unroll
  for (int i = 0; i < V; ++i) t[i] = scale == 255u ? (int8_t)0 : (int8_t)(int)__builtin_rintf(v[i] * inv);
  if (!TAIL || n >= V) {
    typename Words<int8_t, V>::W w;
    __builtin_memcpy(&w, t, sizeof w);
    *reinterpret_cast<typename Words<int8_t, V>::Unaligned*>(p) = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) p[i] = t[i];
}

template <int V>
__device__ __forceinline__ void unpack_codes(const Raw<int8_t, V>& codes, uint32_t scale, float (&v)[V]) {
  codes.widen_to(v);
  const float s = unpack_scale(scale);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] *= s;
}

template <bool TAIL, int V>
__device__ __forceinline__ void load_codes(const int8_t* p, int n, uint32_t scale, float (&v)[V]) {
  Raw<int8_t, V> codes;
  codes.template load_part<TAIL>(p, n);
  unpack_codes(codes, scale, v);
}

}  // namespace seqdev

// Widest vector that divides a row of C elements, at most 16 bytes.
inline int seq_vec(int type, int64_t C) {
  int v = type == SEQ_BF16 ? 8 : 4;
  while (C % v) v /= 2;
  return v;
}

}  // namespace cgconv
