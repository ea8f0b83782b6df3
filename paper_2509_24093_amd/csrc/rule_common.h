// Device helpers and the workspace of the gated delta rule (delta_rule.hip,
// delta_rule_bwd.hip).
//
// Products in 32 bits on the bfloat16 matrix cores: a float is the sum of three
// bfloat16, x = h + m + l, each the leading 8 bits of what is left (24 bits in
// all: exact, but for parts below the smallest normal).  Of the nine products of
// two such sums the three smallest are left out: the parts are cut, m is below 2^-7
// and l below 2^-15 of the leading bit, so what is left out is below 2^-21 of the
// product (7.8 x 2^-24 at the worst found, 0.7 x 2^-24 on average over normal numbers)
// and always has its sign.  A bfloat16 operand is its own first part, and nothing is
// left out.  Outputs and gradients are off as those of plain sums in 32 bits are,
// 1e-7 to 5e-7 in a chunk's 2-norm (tests/test_delta_rule_precision.py).  Six
// v_mfma_f32_16x16x32_bf16 take 96 cycles where the fp32 instructions of the same
// product take 256.
//
// Lanes: m = lane & 15, q = lane >> 4.  Accumulators hold column m, rows 4 q .. 4 q + 3
// of a 16 x 16 tile.  The order of the products' inner index is free as long as
// both operands keep to it: element e of lane group q is index 4 q + e (e < 4) of
// the first 16 and 4 q + e - 4 of the second 16, so two accumulator tiles one
// below the other are an operand of the next product as they are.
#pragma once

#include <type_traits>

#include "seq_common.h"

namespace cgconv {
namespace ruledev {

using namespace seqdev;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kT = kRuleChunk;          // tokens of a chunk: four tiles of 16
constexpr int kTiles = kT / 16;
constexpr int kWalkWaves = 8;           // of a block that walks the chunks, 16 columns each
constexpr int kBlocks = kRuleTriangle;  // 16 x 16 blocks on and below the diagonal of kT x kT
__host__ __device__ constexpr int block_of(int i, int j) { return i * (i + 1) / 2 + j; }
__host__ __device__ constexpr int row_of(int block) { return block < 1 ? 0 : block < 3 ? 1 : block < 6 ? 2 : 3; }

// Parts of an operand of storage type T.
template <class T>
constexpr int kParts = sizeof(T) == 2 ? 1 : 3;

// Eight values of one lane (one part).
union Frag {
  uint4 all;
  uint32_t w[4];
  uint2 h[2];
  v8bf f;
};

__device__ __forceinline__ uint32_t top_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}
__device__ __forceinline__ float without_top(float x) {
  return x - __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
}
// The parts of two values, each pair in one word.
__device__ __forceinline__ void split2(float a, float b, uint32_t& h, uint32_t& m, uint32_t& l) {
  h = top_halves(a, b);
  a = without_top(a);
  b = without_top(b);
  m = top_halves(a, b);
  l = top_halves(without_top(a), without_top(b));
}
__device__ __forceinline__ void split8(const float (&x)[8], Frag (&f)[3]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) split2(x[2 * e], x[2 * e + 1], f[0].w[e], f[1].w[e], f[2].w[e]);
}
// The parts of products x y: what is left of the first part is that of the exact product.
__device__ __forceinline__ void split_products(const v4f& xa, const v4f& ya, const v4f& xb, const v4f& yb, Frag (&f)[3]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float rest[2];
    uint32_t top[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float x = (e < 2 ? xa : xb)[2 * (e & 1) + i], y = (e < 2 ? ya : yb)[2 * (e & 1) + i];
      top[i] = __float_as_uint(x * y);
      rest[i] = fmaf(x, y, -__uint_as_float(top[i] & 0xFFFF0000u));
    }
    f[0].w[e] = __builtin_amdgcn_perm(top[1], top[0], 0x07060302);
    f[1].w[e] = top_halves(rest[0], rest[1]);
    f[2].w[e] = top_halves(without_top(rest[0]), without_top(rest[1]));
  }
}
__device__ __forceinline__ void split_tiles(const v4f& a, const v4f& b, Frag (&f)[3]) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  split8(x, f);
}
// Values of storage type T widened to x: exact in its own parts.
template <class T>
__device__ __forceinline__ void parts8(const float (&x)[8], Frag (&f)[kParts<T>]) {
  if constexpr (kParts<T> == 3) {
    split8(x, f);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[0].w[e] = top_halves(x[2 * e], x[2 * e + 1]);
  }
}

// acc += A B, the smallest products first.
template <int NA, int NB>
__device__ __forceinline__ v4f mma(const Frag (&a)[NA], const Frag (&b)[NB], v4f acc) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int p = 0; p < NA; ++p)
      if (s - p >= 0 && s - p < NB)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p].f, b[s - p].f, acc, 0, 0, 0);
  return acc;
}

// acc[i] += A[i] B: the products of one accumulator follow each other only after all the
// others', so that none waits for the one before (each takes 16 cycles and is done after 32).
template <int NI, int NA, int NB>
__device__ __forceinline__ void mma_all(const Frag (&a)[NI][NA], const Frag (&b)[NB], v4f (&acc)[NI]) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int p = 0; p < NA; ++p)
      if (s - p >= 0 && s - p < NB) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i][p].f, b[s - p].f, acc[i], 0, 0, 0);
      }
}
// acc[j] += A B[j], in the same order.
template <int NJ, int NA, int NB>
__device__ __forceinline__ void mma_each(const Frag (&a)[NA], const Frag (&b)[NJ][NB], v4f (&acc)[NJ]) {
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int p = 0; p < NA; ++p)
      if (s - p >= 0 && s - p < NB) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p].f, b[j][s - p].f, acc[j], 0, 0, 0);
      }
}
// Rows of 64 tokens in LDS, one array a part.  Row stride in elements: an odd multiple of
// four words, so that 16 rows' words at one column lie in 16 different groups of four banks.
constexpr int row_stride(int KB) { return 32 * KB + 8; }

__device__ __forceinline__ uint2 lds2(const bf16* p) { return *reinterpret_cast<const uint2*>(p); }

// Operand with rows 16 i + m of a row-major array, inner index 32 kb + ...
template <int NP, int ST>
__device__ __forceinline__ void rows_frag(const bf16 (&buf)[NP][kT * ST], int i, int kb, int m, int q, Frag (&f)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const bf16* at = buf[p] + (16 * i + m) * ST + 32 * kb + 4 * q;
    f[p].h[0] = lds2(at);
    f[p].h[1] = lds2(at + 16);
  }
}

// Operand with rows (columns of the array) 16 i + m, whose inner index is the
// array's row 32 kb + ...: transposed reads, the 16 lanes of a group fetch four
// rows of 16 elements and get a column of them each.
template <int NP, int ST>
__device__ __forceinline__ void columns_frag(const bf16 (&buf)[NP][kT * ST], int i, int kb, int m, int q,
                                             Frag (&f)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const bf16* at = buf[p] + (32 * kb + 16 * half + 4 * q + (m >> 2)) * ST + 16 * i + 4 * (m & 3);
      const v4s t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)at);
      __builtin_memcpy(&f[p].h[half], &t, 8);
    }
}

// Triangle blocks in LDS, a lane's four values of a block in 8 bytes a part; block
// (i, j) holds rows i, or of the transposed triangle rows j.
typedef uint2 TriangleParts[3][kBlocks][64];
__device__ __forceinline__ void put_block(TriangleParts& t, int block, int lane, float x, float y, float z, float w) {
  uint2 h, m, l;
  split2(x, y, h.x, m.x, l.x);
  split2(z, w, h.y, m.y, l.y);
  t[0][block][lane] = h;
  t[1][block][lane] = m;
  t[2][block][lane] = l;
}
// Rows 16 i + m, inner index 32 kb + ... of the lower triangle; UPPER: of its transpose.
template <bool UPPER>
__device__ __forceinline__ void triangle_frag(const TriangleParts& t, int i, int kb, int lane, Frag (&f)[3]) {
#pragma unroll
  for (int p = 0; p < 3; ++p)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int j = 2 * kb + half;
      if (UPPER ? j >= i : j <= i)
        f[p].h[half] = t[p][UPPER ? block_of(j, i) : block_of(i, j)][lane];
      else
        f[p].h[half] = make_uint2(0, 0);
    }
}
template <bool UPPER>
__device__ __forceinline__ constexpr bool triangle_has(int i, int kb) {
  return UPPER ? 2 * kb + 1 >= i : 2 * kb <= i;
}

// mma_all of a triangle's rows: those without a block in this half are left out.
template <bool UPPER, int NB>
__device__ __forceinline__ void mma_triangle(const uint2 (&t)[3][kBlocks][64], int kb, int lane, const Frag (&b)[NB],
                                             v4f (&acc)[kTiles]) {
  Frag f[kTiles][3];
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
    if (triangle_has<UPPER>(i, kb)) triangle_frag<UPPER>(t, i, kb, lane, f[i]);
#pragma unroll
  for (int s = 2; s >= 0; --s)
#pragma unroll
    for (int p = 0; p < 3; ++p)
      if (s - p >= 0 && s - p < NB) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (triangle_has<UPPER>(i, kb))
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i][p].f, b[s - p].f, acc[i], 0, 0, 0);
      }
}

// A triangle's zeros let nothing through but what is not finite: 0 x NaN is NaN.  So where
// there is such a value, before a product with a triangle a column's values from the first one
// on (of a transposed triangle: up to the last one) give way to zeros, and afterwards the
// results from there on are NaN, as the formula has them; the others are those of finite values
// bit by bit.  An infinity counts as a NaN: split into parts it is one.  What is not finite
// never leaves a column of the state, so the walks look at the last one of a segment, and
// repeat the segment in this way if there is any: looking at every chunk's values instead took
// prompts of heads of 128 x 128 from 622 to 686 us.
template <int TILES>
__device__ __forceinline__ bool any_odd(const v4f (&x)[TILES]) {  // in any lane of the wave
  float z = 0.f;
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) z = fmaf(x[i][r], 0.f, z);
  return __builtin_amdgcn_ballot_w64(z != 0.f) != 0;
}
// A place in the order of a triangle's products: tokens, or from the last one back.
template <bool UPPER>
__device__ __forceinline__ int place_of(int i, int r, int q) {
  return UPPER ? kT - 1 - (16 * i + 4 * q + r) : 16 * i + 4 * q + r;
}
// The first place whose value in the lane's column is not finite, kT if there is none.
template <bool UPPER>
__device__ __forceinline__ int first_odd(const v4f (&x)[kTiles], int q) {
  int at = kT;
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!(__builtin_fabsf(x[i][r]) < __builtin_inff())) at = min(at, place_of<UPPER>(i, r, q));
  at = min(at, __shfl_xor(at, 16));
  return min(at, __shfl_xor(at, 32));
}
// x from a place on.
template <bool UPPER>
__device__ __forceinline__ void put_from(v4f (&x)[kTiles], int at, int q, float value) {
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) x[i][r] = place_of<UPPER>(i, r, q) >= at ? value : x[i][r];
}

// The only argument of a kernel, read once more: what a second part of the kernel needs of it is
// then not held in registers through the first.
template <class A>
__device__ __forceinline__ A argument_anew() {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  A a;
  __builtin_memcpy(&a, (const void*)p, sizeof a);
  return a;
}

// The numbers of a token that its chunk's kernels need, made by rule_prepare_kernel:
// x = beta, y = rk e^G, z = rk e^(G_end - G), w = scale rq e^G with G the sum of the
// decays of the chunk up to the token, rk and rq the factors that norm key and query.
// Second: x = rk, y = rq, z + w = G log2(e), so that a decay is one exponential of base 2 of
// a difference rounded once.
struct Token {
  float4 a, b;
};
__device__ __forceinline__ float decay_between(const float4& i, const float4& j) {
  return __builtin_amdgcn_exp2f((i.z - j.z) + (i.w - j.w));
}

// A head's column (component, channel) in a token's row; columns past V: none.
struct Column {
  int at;
  bool there;
  Column() = default;
  __device__ __forceinline__ Column(int col, int V, int P, int C, int h) {
    there = col < V;
    const int k = there ? col / P : 0;
    at = k * C + h * P + (there ? col - k * P : 0);
  }
};

// Loads on the way from global memory to LDS or to the products, a chunk ahead of their
// use.  They are not masked, which would take a branch and a wait each: what is not there
// is read from a place that is, and left out where the values are used.

// A place in bytes from a uniform base: 32 bits a lane.  The largest is in a chunk of the widest
// rows, 64 tokens of 16384 key heads of 128 in fp32, and below 2^29; a row has at most 2^23
// bytes, so that a token's number times it is a product of 24 bits each.
template <class T>
__device__ __forceinline__ T& place(T* base, uint32_t bytes) {
  typedef typename std::conditional<std::is_const<T>::value, const char, char>::type Byte;
  return *reinterpret_cast<T*>(reinterpret_cast<Byte*>(base) + bytes);
}
// A chunk's key or query rows, tokens >= 1 of them.
template <class T, int KB, int THREADS>
struct RowStage {
  static constexpr int kAll = 256 * KB, kEach = (kAll + THREADS - 1) / THREADS;  // pieces of eight
  Raw<T, 8> raw[kEach];
  __device__ __forceinline__ void load(const T* base, int stride, int tokens, int D, int tid) {
#pragma unroll
    for (int p = 0; p < kEach; ++p) {
      const int at = p * THREADS + tid, row = at / (4 * KB), c = at % (4 * KB) * 8;
      const uint32_t o = __umul24(min(row, tokens - 1), stride * (int)sizeof(T));
      if (D % 8 == 0) {
        raw[p].load(&place(base, o + (c < D ? c : 0) * (int)sizeof(T)));
      } else {
        T t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = place(base, o + min(c + e, D - 1) * (int)sizeof(T));
        __builtin_memcpy(raw[p].w, t, sizeof t);
      }
    }
  }
  template <int NP, int N>
  __device__ __forceinline__ void store(bf16 (&buf)[NP][N], int tokens, int D, int tid) const {
    constexpr int ST = row_stride(KB);
#pragma unroll
    for (int p = 0; p < kEach; ++p) {
      const int at = p * THREADS + tid, row = at / (4 * KB), c = at % (4 * KB) * 8;
      if (kAll % THREADS && at >= kAll) break;
      const int n = row < tokens ? D - c : 0;
      Frag f[NP];
      if constexpr (NP == 1) {
        __builtin_memcpy(&f[0], raw[p].w, 16);
        if (D % 8 == 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) f[0].w[e] = n > 0 ? f[0].w[e] : 0u;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            f[0].w[e] = n >= 2 * e + 2 ? f[0].w[e] : n > 2 * e ? f[0].w[e] & 0xFFFFu : 0u;
        }
      } else {
        float x[8];
        raw[p].widen_to(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? x[e] : 0.f;
        split8(x, f);
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        *reinterpret_cast<Frag*>(buf[i] + row * ST + c) = f[i];
      }
    }
  }
};

// Blocks of a triangle, 640 quadruples.
template <int THREADS>
struct BlockStage {
  static constexpr int kEach = (kBlocks * 64 + THREADS - 1) / THREADS;
  float4 v[kEach];
  __device__ __forceinline__ void load(const float4* base, int tid) {
#pragma unroll
    for (int p = 0; p < kEach; ++p) v[p] = base[min(p * THREADS + tid, kBlocks * 64 - 1)];
  }
  __device__ __forceinline__ void store(TriangleParts& t, int tid) const {
#pragma unroll
    for (int p = 0; p < kEach; ++p) {
      const int at = p * THREADS + tid;
      if (at < kBlocks * 64) put_block(t, at >> 6, at & 63, v[p].x, v[p].y, v[p].z, v[p].w);
    }
  }
};

// A chunk in LDS: its keys, queries, triangles and tokens.  Two of them where they fit: the
// next one is filled while the waves work on this one, and they meet once a chunk.
template <class T, int KB, bool QUERIES, bool INSIDE>
struct Stage {
  static constexpr int NP = kParts<T>, ST = row_stride(KB);
  alignas(16) bf16 k[NP][kT * ST];
  alignas(16) bf16 q[QUERIES ? NP : 1][QUERIES ? kT * ST : 8];
  TriangleParts inv;
  uint2 inside[INSIDE ? 3 : 1][INSIDE ? kBlocks : 1][INSIDE ? 64 : 1];
  float4 token[kT];
  static constexpr int kBytes = 2 * NP * kT * ST * (QUERIES ? 2 : 1) + (int)sizeof(TriangleParts) * (INSIDE ? 2 : 1) + 16 * kT + 64;
  static constexpr int kCount = 2 * kBytes <= 160 * 1024 ? 2 : 1;
};

// The 16 values of a lane's column in a chunk: tokens 16 i + 4 q + r.  In place of a token
// that is not there comes the last one, whose products with the zero key, query and beta of
// that row are as harmless as they are in its own row.
template <class T>
struct ColumnStage {
  T v[kTiles][4];
  __device__ __forceinline__ void load(const T* base, int stride, int tokens, const Column& c, int q) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[i][r] = place(base, __umul24(min(16 * i + 4 * q + r, tokens - 1), stride * (int)sizeof(T)) +
                                  c.at * (int)sizeof(T));
  }
  __device__ __forceinline__ float get(int i, int r, const Column& c) const { return c.there ? widen(v[i][r]) : 0.f; }
};

// The same 16 values to a tensor of which `left` tokens are left from the chunk's first on;
// zeros from `tokens` on.
template <class T>
__device__ __forceinline__ void store_column(T* base, int stride, int left, int tokens, const Column& c, int q,
                                             const v4f (&x)[kTiles]) {
  if (!c.there) return;
  const int row = afresh(stride) * (int)sizeof(T);
  const uint32_t at = __umul24(4 * q, row) + c.at * (int)sizeof(T);
  if (tokens >= kT) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) place(base, at + (16 * i + r) * row) = (T)x[i][r];
    return;
  }
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = 16 * i + 4 * q + r;
      if (t < left) place(base, at + (16 * i + r) * row) = t < tokens ? (T)x[i][r] : (T)0.f;
    }
}

// Accumulator tiles one below the other to columns `col` of rows of a workspace array.
template <int TILES>
__device__ __forceinline__ void store_tiles(float* base, int stride, int col, int q, const v4f (&x)[TILES]) {
  const int row = afresh(stride) * 4;
  const uint32_t at = __umul24(4 * q, row) + col * 4;
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) place(base, at + (16 * i + r) * row) = x[i][r];
}

}  // namespace ruledev
}  // namespace cgconv
