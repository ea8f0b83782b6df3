// Layer norm by degree, forward and backward, for gfx950.  For a token's
// features x[(l,m),c] (K = (L+1)^2 components of C channels, the degrees'
// (2l+1) C values contiguous):
//
//   d = x - [l = 0] mean_c x                      only invariants may be shifted
//   r_l = 1 / sqrt(mean_{m,c} d^2 + eps)
//   y = w[l,c] d r_l + [l = 0] bias[c]
//
// L = 0 is the ordinary layer norm over C.  Backward, with h = d r (the
// normalised values) and g = w gy:
//
//   gx = r_l (g - [l = 0] mean g - h mean(g h)),   gw[l,c] = sum_{t,m} gy h,   gb[c] = sum_t gy_0
//
// Two forms.  Rows (one component's C channels) of at most 64 vectors are
// shared by 1..64 lanes, and a block takes whole tokens of several rows per
// pass, all of them in registers: the sum of a row is a lane reduction, the sum
// of a degree adds the sums of its rows through LDS.  Longer rows: a block per
// degree of a token.  Either way every input is read once and every output
// written once, but for an 8-bit checkpoint of rows of the second form with L > 0
// whose channels are no multiple of 32: a pass of its own reads x again.  In the
// backward the threads keep their columns from token to token, so gw and gb grow in
// registers over all tokens of a block; the blocks' sums are added by a second
// kernel in a fixed order.  Registers: where no vector of four elements divides a
// row of the second form with L > 0, a thread of the longest rows holds 8 or 16
// vectors and spills (16 in the forward up to 464 bytes of scratch a thread, in the
// backward 36 to 524; the other backward kernels of that form at most 40).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "norm_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

// Dynamic LDS: a row's sums, then a degree's.
template <class T, int V, int R, bool CODES, bool TAIL>
__global__ void norm_rows_kernel(NormArgs a, RowShape sh) {
  extern __shared__ float lds[];
  const int tid = threadIdx.x, per = sh.threads / sh.lanes;  // rows per pass
  const int j = tid & (sh.lanes - 1), rg = tid / sh.lanes;
  const int c = j * V;
  const int left = a.C - c;  // channels from c on
  const bool col = left > 0;
  const long long t0 = (long long)blockIdx.x * sh.tokens;
  const int toks = (int)min((long long)sh.tokens, a.tokens - t0);
  const int rows = toks * a.K;
  float* rowsum = lds;
  float* rs = lds + sh.tokens * a.K;
  const T* x = static_cast<const T*>(a.x) + t0 * a.K * a.C;
  float v[R][V];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = 0.f;
    if (col && r < rows) load_part<TAIL>(x + (long long)r * a.C + c, left, v[i]);
  }
  const int nb = (a.C + kPackBlock - 1) / kPackBlock;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
    if (CODES) {
      constexpr int kLanes = kPackBlock / V;
      const uint32_t scale = pack_scale(group_max_bits(max_bits(v[i]), min(kLanes, sh.lanes)));
      if (col && r < rows) {
        const long long row = t0 * a.K + r;
        store_codes<TAIL>(a.codes + row * a.C + c, left, v[i], scale);
        if (j % kLanes == 0) a.scales[row * nb + c / kPackBlock] = (uint8_t)scale;
      }
    }
    const int tok = divide(r, sh.magic);
    if (r - tok * a.K == 0) {  // the invariants' row
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) s += v[i][e];
      const float mean = group_sum(s, sh.lanes) / (float)a.C;
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = e < left ? v[i][e] - mean : 0.f;
      if (a.mean && j == 0 && r < rows) a.mean[t0 + tok] = mean;
    }
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) q = fmaf(v[i][e], v[i][e], q);
    q = group_sum(q, sh.lanes);
    if (j == 0 && r < rows) rowsum[r] = q;
  }
  __syncthreads();
  const int degs = a.L + 1;
  degree_sums(rowsum, rs, toks, degs, a.K, sh.threads, [&](float s, int i, int l) {
    const float r = 1.f / __builtin_sqrtf(s / (float)((2 * l + 1) * a.C) + a.eps);
    if (a.rstd) a.rstd[t0 * degs + i] = r;
    return r;
  });
  __syncthreads();
  T* y = static_cast<T*>(a.y) + t0 * a.K * a.C;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
    if (!col || r >= rows) continue;
    const int tok = divide(r, sh.magic), comp = r - tok * a.K, l = degree_of(comp);
    const float m = rs[tok * degs + l];
    float w[V];
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = m;
    if (a.weight) {
      load_part<TAIL>(a.weight + l * a.C + c, left, w);
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] *= m;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] *= w[e];
    if (comp == 0 && a.bias) {
      float b[V];
      load_part<TAIL>(a.bias + c, left, b);
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] += b[e];
    }
    store_part<TAIL>(y + (long long)r * a.C + c, left, v[i]);
  }
}

// Wide rows: block (token, degree), the degree's (2l+1) C values in registers.
// CODES only where a scale's lanes are neighbours: C a multiple of 32, or L = 0.
// TAIL: L = 0 and C no multiple of V.
template <class T, int V, int R, bool CODES, int MAXT, bool TAIL>
__global__ __launch_bounds__(MAXT) void norm_wide_kernel(NormArgs a, uint32_t magic) {
  __shared__ float lds[16];
  const int tid = threadIdx.x, threads = blockDim.x, l = blockIdx.y;
  const int n = (2 * l + 1) * a.C;
  const long long t = blockIdx.x;
  const long long base = (t * a.K + l * l) * a.C;
  const T* x = static_cast<const T*>(a.x) + base;
  float v[R][V];
  const int nb = (a.C + kPackBlock - 1) / kPackBlock;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = 0.f;
    if (e0 < n) load_part<TAIL>(x + e0, n - e0, v[i]);
    if (CODES) {
      constexpr int kLanes = kPackBlock / V;
      const uint32_t scale = pack_scale(group_max_bits(max_bits(v[i]), kLanes));
      if (e0 < n) {
        store_codes<TAIL>(a.codes + base + e0, n - e0, v[i], scale);
        const int m = l == 0 ? 0 : divide(e0, magic);
        if (tid % kLanes == 0) a.scales[(t * a.K + l * l + m) * nb + (e0 - m * a.C) / kPackBlock] = (uint8_t)scale;
      }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) s += v[i][e];
  }
  if (l == 0) {
    const float mean = block_sum(s, lds, threads) / (float)a.C;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int left = n - (i * threads + tid) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) v[i][e] = (TAIL ? e < left : left > 0) ? v[i][e] - mean : 0.f;
    }
    if (a.mean && tid == 0) a.mean[t] = mean;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) q = fmaf(v[i][e], v[i][e], q);
  const float r = 1.f / __builtin_sqrtf(block_sum(q, lds, threads) / (float)n + a.eps);
  if (a.rstd && tid == 0) a.rstd[t * (a.L + 1) + l] = r;
  T* y = static_cast<T*>(a.y) + base;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
    if (e0 >= n) continue;
    const int c = l == 0 ? e0 : e0 - divide(e0, magic) * a.C;
    float w[V], b[V];
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = 1.f, b[e] = 0.f;
    if (a.weight) load_part<TAIL>(a.weight + (long long)l * a.C + c, n - e0, w);
    if (l == 0 && a.bias) load_part<TAIL>(a.bias + c, n - e0, b);
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = fmaf(v[i][e] * r, w[e], b[e]);
    store_part<TAIL>(y + e0, n - e0, v[i]);
  }
}

// ---- backward --------------------------------------------------------------------

// Input values of a row vector: x itself, or its 8-bit checkpoint.
template <class T, int V, bool CODES, bool TAIL>
__device__ __forceinline__ void load_input(const NormBwdArgs& a, long long row, int c, int nb, float (&v)[V]) {
  if (CODES)
    load_codes<TAIL>(a.codes + row * a.C + c, a.C - c, a.scales[row * nb + c / kPackBlock], v);
  else
    load_part<TAIL>(static_cast<const T*>(a.x) + row * a.C + c, a.C - c, v);
}

// Block b takes tiles b, b + gridDim.x, ... of sh.tokens tokens.  Dynamic LDS:
// sums of rows and of degrees while the tiles run, then the staging of gw.
// Partial sums of block b: part[b][L+1 degrees, then gb][C].
constexpr int kBwdRowThreads = 512;

template <class T, int V, int R, bool CODES, bool TAIL>
__global__ __launch_bounds__(kBwdRowThreads) void norm_rows_bwd_kernel(NormBwdArgs a, RowShape sh, long long tiles) {
  extern __shared__ float lds[];
  const int tid = threadIdx.x, per = sh.threads / sh.lanes;
  const int j = tid & (sh.lanes - 1), rg = tid / sh.lanes;
  const int c = j * V;
  const int left = a.C - c;  // channels from c on
  const bool col = left > 0;
  const int nb = (a.C + kPackBlock - 1) / kPackBlock, degs = a.L + 1;
  float* rowsum = lds;
  float* ds = lds + sh.tokens * a.K;  // mean(g h) of every degree
  float gw[R][V], gb[V];
  int tok[R], comp[R], deg[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
    tok[i] = divide(r, sh.magic);
    comp[i] = r - tok[i] * a.K;
    deg[i] = degree_of(comp[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) gw[i][e] = 0.f;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) gb[e] = 0.f;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const long long t0 = tile * sh.tokens;
    const int toks = (int)min((long long)sh.tokens, a.tokens - t0);
    const T* gy = static_cast<const T*>(a.gy) + t0 * a.K * a.C;
    float h[R][V], g[R][V], m0[R], r0[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = g[i][e] = 0.f;
      m0[i] = r0[i] = 0.f;
      if (col && tok[i] < toks) {
        const int r = i * per + rg;
        load_input<T, V, CODES, TAIL>(a, t0 * a.K + r, c, nb, h[i]);
        load_part<TAIL>(gy + (long long)r * a.C + c, left, g[i]);
        r0[i] = a.rstd[(t0 + tok[i]) * degs + deg[i]];
        if (comp[i] == 0) m0[i] = a.mean[t0 + tok[i]];
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float w[V];
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = 1.f;
      if (a.weight && col) load_part<TAIL>(a.weight + deg[i] * a.C + c, left, w);
      float q = 0.f, s = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        h[i][e] = (h[i][e] - m0[i]) * r0[i];
        gw[i][e] = fmaf(g[i][e], h[i][e], gw[i][e]);
        if (comp[i] == 0) gb[e] += g[i][e];
        g[i][e] *= w[e];
        q = fmaf(g[i][e], h[i][e], q);
        s += g[i][e];
      }
      q = group_sum(q, sh.lanes);
      if (comp[i] == 0) {
        s = group_sum(s, sh.lanes) / (float)a.C;
#pragma unroll
        for (int e = 0; e < V; ++e) g[i][e] -= s;
      }
      if (j == 0 && tok[i] < toks) rowsum[i * per + rg] = q;
    }
    __syncthreads();
    degree_sums(rowsum, ds, toks, degs, a.K, sh.threads,
                [&](float s, int, int l) { return s / (float)((2 * l + 1) * a.C); });
    __syncthreads();
    if (a.gx) {
      T* gx = static_cast<T*>(a.gx) + t0 * a.K * a.C;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (!col || tok[i] >= toks) continue;
        const float d = ds[tok[i] * degs + deg[i]];
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = r0[i] * fmaf(-h[i][e], d, g[i][e]);
        store_part<TAIL>(gx + (long long)(i * per + rg) * a.C + c, left, o);
      }
    }
    // the next tile writes rowsum only, which every thread has read before the
    // second barrier, and ds after its own first barrier
  }
  if (!a.part) return;
  // gw of the block: all rows through LDS, each output adds its degree's rows
  float* part = a.part + (long long)blockIdx.x * (degs + 1) * a.C;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (col) {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (!TAIL || e < left) lds[(i * per + rg) * a.C + c + e] = gw[i][e];
    }
  __syncthreads();
  for (int o = tid; o < degs * a.C; o += sh.threads) {
    const int l = o / a.C, ch = o - l * a.C;
    float s = 0.f;
    for (int t = 0; t < sh.tokens; ++t)
      for (int m = 0; m < 2 * l + 1; ++m) s += lds[(t * a.K + l * l + m) * a.C + ch];
    part[o] = s;
  }
  __syncthreads();
  if (col) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (!TAIL || e < left) lds[rg * a.C + c + e] = gb[e];
  }
  __syncthreads();
  for (int ch = tid; ch < a.C; ch += sh.threads) {
    float s = 0.f;
    for (int r = 0; r < per; ++r) s += lds[r * a.C + ch];
    part[degs * a.C + ch] = s;
  }
}

// Wide rows: block (slot, degree) takes tokens slot, slot + gridDim.x, ..., each
// loaded as it is stored while the one before is computed for bf16 rows of whole
// vectors, where that takes 16 registers and four waves per SIMD still fit (8 x
// 2048 tokens of 4096 channels, forward and backward: 185 -> 164 us, at three waves
// 190; with 8-bit inputs three waves, the backward of 32768 of 1024 73 -> 54; fp32, 4 x 4096
// tokens of L=2 C=512 with 32 registers ahead: 320 -> 392).
// Partial sums: part[slot][K components, then gb][C].
template <class T, int V, int R, bool CODES, int MAXT, bool TAIL>
__global__ __launch_bounds__(MAXT, MAXT > 256 || V == 4 ? 4 : V == 8 ? (CODES ? 3 : 4) : 2) void norm_wide_bwd_kernel(
    NormBwdArgs a, uint32_t magic) {
  constexpr bool kAhead = MAXT <= 256 && V == 8;
  __shared__ float lds[32];
  const int tid = threadIdx.x, threads = blockDim.x, l = blockIdx.y;
  const int n = (2 * l + 1) * a.C, nb = (a.C + kPackBlock - 1) / kPackBlock;
  float gw[R][V], gb[R][V];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) gw[i][e] = gb[i][e] = 0.f;
  constexpr int kHeld = kAhead ? R : 1;
  Raw<T, V> xr[kHeld], gr[kHeld];
  Raw<int8_t, V> cr[kHeld];
  uint32_t sc[kHeld];
  float r0n = 0.f, m0n = 0.f;
  auto fetch = [&](long long t) {
    const long long row0 = t * a.K + l * l;
    r0n = a.rstd[t * (a.L + 1) + l];
    m0n = l == 0 ? a.mean[t] : 0.f;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int e0 = (i * threads + tid) * V;
      if (e0 < n) {
        if (CODES) {
          const int m = l == 0 ? 0 : divide(e0, magic);
          cr[i].template load_part<TAIL>(a.codes + row0 * a.C + e0, n - e0);
          sc[i] = a.scales[(row0 + m) * nb + (e0 - m * a.C) / kPackBlock];
        } else {
          xr[i].template load_part<TAIL>(static_cast<const T*>(a.x) + row0 * a.C + e0, n - e0);
        }
        gr[i].template load_part<TAIL>(static_cast<const T*>(a.gy) + row0 * a.C + e0, n - e0);
      }
    }
  };
  if (kAhead && blockIdx.x < a.tokens) fetch(blockIdx.x);
  for (long long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const float r0 = kAhead ? r0n : a.rstd[t * (a.L + 1) + l];
    const float m0 = kAhead ? m0n : l == 0 ? a.mean[t] : 0.f;
    float h[R][V], g[R][V];
    float q = 0.f, s = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = m0, g[i][e] = 0.f;
      if (e0 >= n) continue;
      if constexpr (kAhead) {
        if (CODES)
          unpack_codes(cr[i], sc[i], h[i]);
        else
          xr[i].widen_to(h[i]);
        gr[i].widen_to(g[i]);
      } else {
        const long long row0 = t * a.K + l * l;
        const int m = l == 0 ? 0 : divide(e0, magic);
        load_input<T, V, CODES, TAIL>(a, row0 + m, e0 - m * a.C, nb, h[i]);
        load_part<TAIL>(static_cast<const T*>(a.gy) + row0 * a.C + e0, n - e0, g[i]);
      }
    }
    if (kAhead && t + gridDim.x < a.tokens) fetch(t + gridDim.x);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
      float w[V];
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = 1.f;
      const int c = l == 0 ? e0 : e0 - divide(e0, magic) * a.C;
      if (a.weight && e0 < n) load_part<TAIL>(a.weight + (long long)l * a.C + c, n - e0, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        h[i][e] = (h[i][e] - m0) * r0;
        gw[i][e] = fmaf(g[i][e], h[i][e], gw[i][e]);
        gb[i][e] += g[i][e];
        g[i][e] *= w[e];
        q = fmaf(g[i][e], h[i][e], q);
        s += g[i][e];
      }
    }
    if (!a.gx) continue;
    block_sum2(q, s, lds, threads);
    const float d = q / (float)n, m1 = l == 0 ? s / (float)n : 0.f;
    T* gx = static_cast<T*>(a.gx) + (t * a.K + l * l) * a.C;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
      if (e0 >= n) continue;
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = r0 * fmaf(-h[i][e], d, g[i][e] - m1);
      store_part<TAIL>(gx + e0, n - e0, o);
    }
  }
  if (!a.part) return;
  float* part = a.part + (long long)blockIdx.x * (a.K + 1) * a.C;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
    if (e0 >= n) continue;
    store_part<TAIL>(part + (long long)l * l * a.C + e0, n - e0, gw[i]);
    if (l == 0) store_part<TAIL>(part + (long long)a.K * a.C + e0, n - e0, gb[i]);
  }
}

// Adds the blocks' partial sums: block of 16 slices x 64 outputs, a slice adds
// every 16th block's sum, in a fixed order.  per_degree: rows of part are the
// degrees (row form), else the K components.
constexpr int kSumSlices = 16;
__global__ __launch_bounds__(64 * kSumSlices) void norm_sum_kernel(const float* __restrict__ part, int blocks, int L,
                                                                   int K, int C, int per_degree, float* gw, float* gb) {
  __shared__ float lds[kSumSlices][64];
  const int o = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
  const int l = o / C, c = o - l * C;  // l = L + 1: gb
  const int rows = (per_degree ? L + 1 : K) + 1;
  float s = 0.f;
  if (l <= L + 1) {
    const bool bias = l == L + 1;
    const int first = bias ? rows - 1 : (per_degree ? l : l * l), n = bias || per_degree ? 1 : 2 * l + 1;
    for (int m = 0; m < n; ++m) {
      const float* p = part + (long long)(first + m) * C + c;
#pragma unroll 4
      for (int b = slice; b < blocks; b += kSumSlices) s += p[(long long)b * rows * C];
    }
  }
  lds[slice][threadIdx.x & 63] = s;
  __syncthreads();
  if (slice == 0 && l <= L + 1) {
    float t = 0.f;
    for (int i = 0; i < kSumSlices; ++i) t += lds[i][threadIdx.x];
    if (l == L + 1) {
      if (gb) gb[c] = t;
    } else if (gw) {
      gw[o] = t;
    }
  }
}

// ---- launch shapes -----------------------------------------------------------------

constexpr int kBwdBlocks = 1024;
int row_bwd_blocks(long long tokens, const RowShape& sh) {
  const long long tiles = (tokens + sh.tokens - 1) / sh.tokens;
  return (int)std::min<long long>(tiles, kBwdBlocks * 256 / sh.threads);
}
// A thread's share of the chip per degree, at most 2048 blocks in all: each writes
// sums that are read again (16384 tokens of 4096 bf16 channels in blocks of 256: 512
// blocks 178 us, 1024 164, 2048 179; 32768 of 1024 in blocks of 64: 1024 173, 2048
// 139).
int wide_bwd_blocks(long long tokens, int L, int threads) {
  return (int)std::min<long long>(tokens, std::max(64, std::min(2048, (1 << 18) / threads) / (L + 1)));
}

size_t row_lds_floats(const RowShape& sh, int K, int L) { return (size_t)sh.tokens * (K + L + 1); }

template <class T, int V, bool TAIL, int R>
hipError_t norm_rows(const NormArgs& a, const RowShape& sh, hipStream_t s) {
  const long long blocks = (a.tokens + sh.tokens - 1) / sh.tokens;
  if (!launch_fits(blocks, sh.threads)) return hipErrorInvalidConfiguration;
  const size_t lds = row_lds_floats(sh, a.K, a.L) * sizeof(float);
  if (lds > 64 * 1024) return hipErrorInvalidValue;
  if (a.codes)
    hipLaunchKernelGGL((norm_rows_kernel<T, V, R, true, TAIL>), dim3((unsigned)blocks), dim3(sh.threads), lds, s, a, sh);
  else
    hipLaunchKernelGGL((norm_rows_kernel<T, V, R, false, TAIL>), dim3((unsigned)blocks), dim3(sh.threads), lds, s, a, sh);
  return hipGetLastError();
}

// Vectors that a thread of the wide form holds, and at most in a row that is longer
// than 1024 threads of them (vectors of one or two elements).
constexpr int usual_vecs(int V, bool backward) { return backward && V == 8 ? 2 : 4; }
constexpr int max_vecs(int V, bool backward) { return std::max(usual_vecs(V, backward), 16 / V); }

// f of the most threads a block of R vectors a thread has: fewer vectors than usual
// are blocks of 64 threads, more blocks of 1024.  BYTES of a vector: of two, a row that
// takes the wide form has more than 256 threads' worth.
template <int R, int USUAL, int BYTES, class F>
hipError_t by_threads(int threads, F f) {
  if constexpr (R <= USUAL && BYTES > 2) {
    if (threads <= 256) return f(std::integral_constant<int, 256>());
  }
  if constexpr (R >= USUAL) {
    if (threads > 256) return f(std::integral_constant<int, 1024>());
  }
  return hipErrorInvalidValue;
}

template <class T, int V, bool TAIL, int R>
hipError_t norm_wide(const NormArgs& a, int threads, hipStream_t s) {
  if (!launch_fits(a.tokens, threads)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)a.tokens, a.L + 1);
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a, magic_of(a.C));
    return hipGetLastError();
  };
  return by_threads<R, usual_vecs(V, false), V * (int)sizeof(T)>(threads, [&](auto most) {
    constexpr int kMost = decltype(most)::value;
    if constexpr (V >= 4) {  // narrower vectors: C no multiple of four, L > 0
      if (a.codes && (a.C % kPackBlock == 0 || a.L == 0)) return run(norm_wide_kernel<T, V, R, true, kMost, TAIL>);
    }
    if (a.codes) {  // a scale's channels would straddle the lanes: a pass of its own
      const hipError_t e = launch_pack(a.type, a.x, a.codes, a.scales, a.tokens * a.K, a.C, s);
      if (e != hipSuccess) return e;
    }
    return run(norm_wide_kernel<T, V, R, false, kMost, TAIL>);
  });
}

template <class T, int V, bool TAIL, int R>
hipError_t norm_rows_bwd(const NormBwdArgs& a, const RowShape& sh, hipStream_t s) {
  const long long tiles = (a.tokens + sh.tokens - 1) / sh.tokens;
  const int blocks = row_bwd_blocks(a.tokens, sh);
  const int per = sh.threads / sh.lanes;
  const size_t lds = std::max(row_lds_floats(sh, a.K, a.L), a.part ? (size_t)per * R * a.C : 0) * sizeof(float);
  if (lds > 64 * 1024) return hipErrorInvalidValue;
  if (a.codes)
    hipLaunchKernelGGL((norm_rows_bwd_kernel<T, V, R, true, TAIL>), dim3(blocks), dim3(sh.threads), lds, s, a, sh, tiles);
  else
    hipLaunchKernelGGL((norm_rows_bwd_kernel<T, V, R, false, TAIL>), dim3(blocks), dim3(sh.threads), lds, s, a, sh, tiles);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(norm_sum_kernel, dim3(((a.L + 2) * a.C + 63) / 64), dim3(64 * kSumSlices), 0, s, a.part, blocks,
                     a.L, a.K, a.C, 1, a.gw, a.gb);
  return hipGetLastError();
}

template <class T, int V, bool TAIL, int R>
hipError_t norm_wide_bwd(const NormBwdArgs& a, int threads, hipStream_t s) {
  const int blocks = wide_bwd_blocks(a.tokens, a.L, threads);
  const dim3 grid(blocks, a.L + 1);
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a, magic_of(a.C));
    return hipGetLastError();
  };
  const hipError_t e = by_threads<R, usual_vecs(V, true), V * (int)sizeof(T)>(threads, [&](auto most) {
    constexpr int kMost = decltype(most)::value;
    return a.codes ? run(norm_wide_bwd_kernel<T, V, R, true, kMost, TAIL>)
                   : run(norm_wide_bwd_kernel<T, V, R, false, kMost, TAIL>);
  });
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(norm_sum_kernel, dim3(((a.L + 2) * a.C + 63) / 64), dim3(64 * kSumSlices), 0, s, a.part, blocks,
                     a.L, a.K, a.C, 0, a.gw, a.gb);
  return hipGetLastError();
}

// Rows per thread of the row form, whose vectors have at least four elements: up to
// 32 values of one array in the forward, 16 in the backward (which holds four arrays).
constexpr int kFwdPasses = 4;
constexpr int bwd_passes(int V) { return 16 / V; }

// f of the number of vectors per thread, a power of two from R up to MAX.  A row of
// the wide form has more than 64 vectors, and more than 128 where they are narrower
// than four elements, so that its 64 threads hold two and four of them at least.
template <int R, int MAX, class F>
hipError_t by_vecs(int vecs, F f) {
  if (vecs == R) return f(std::integral_constant<int, R>());
  if constexpr (R < MAX) return by_vecs<2 * R, MAX>(vecs, f);
  return hipErrorInvalidValue;
}

// The kernels of a call.  Vectors of at least four elements that divide a row where
// there are such; else (two channels in three are odd or twice odd) full ones, the
// last of a row in part, from rows that start anywhere: element by element 13 x 2018
// rows of 3377 bf16 channels took 805 us with the 8-bit input, 396 this way.  The
// wide form's degrees above 0 wrap from row to row, where only dividing vectors do.
struct Form {
  int v = 0;
  bool tail = false;
  RowShape row{};
  WideShape wide{};  // where row.tokens == 0
};
Form norm_form(int type, int C, int L, bool backward) {
  const int K = (L + 1) * (L + 1), exact = seq_vec(type, C), full = type == SEQ_BF16 ? 8 : 4;
  Form f;
  f.tail = exact < 4;
  f.v = f.tail ? full : exact;
  f.row = backward ? row_shape(C, K, f.v, bwd_passes(f.v), kBwdRowThreads, 16384, 1.0)  // 64 KiB of gw in LDS
                   : row_shape(C, K, f.v, kFwdPasses, 1024, 1024 * 32, 0.1);
  if (f.row.tokens) return f;
  if (f.tail && L > 0) {
    f.tail = false;
    f.v = exact;
  }
  f.wide = wide_shape((2 * L + 1) * C, f.v, usual_vecs(f.v, backward));
  return f;
}

template <class T, int V, bool TAIL>
hipError_t norm_any(const NormArgs& a, const Form& f, hipStream_t s) {
  if constexpr (V >= 4) {
    if (f.row.tokens) return f.row.passes == 2 ? norm_rows<T, V, TAIL, 2>(a, f.row, s) : norm_rows<T, V, TAIL, 4>(a, f.row, s);
  }
  return by_vecs<(V >= 4 ? 2 : 4), max_vecs(V, false)>(
      f.wide.vecs, [&](auto r) { return norm_wide<T, V, TAIL, decltype(r)::value>(a, f.wide.threads, s); });
}

template <class T, int V, bool TAIL>
hipError_t norm_any(const NormBwdArgs& a, const Form& f, hipStream_t s) {
  if constexpr (V >= 4) {
    if (f.row.tokens)
      return f.row.passes == 2 ? norm_rows_bwd<T, V, TAIL, 2>(a, f.row, s)
                               : norm_rows_bwd<T, V, TAIL, bwd_passes(V)>(a, f.row, s);
  }
  return by_vecs<(V >= 4 ? 2 : 4), max_vecs(V, true)>(
      f.wide.vecs, [&](auto r) { return norm_wide_bwd<T, V, TAIL, decltype(r)::value>(a, f.wide.threads, s); });
}

template <class T, class Args>
hipError_t norm_typed(const Args& a, const Form& f, hipStream_t s) {
  constexpr int kFull = 16 / (int)sizeof(T);
  if (f.tail) return norm_any<T, kFull, true>(a, f, s);
  if constexpr (kFull == 8) {
    if (f.v == 8) return norm_any<T, 8, false>(a, f, s);
  }
  switch (f.v) {
    case 4: return norm_any<T, 4, false>(a, f, s);
    case 2: return norm_any<T, 2, false>(a, f, s);
    default: return norm_any<T, 1, false>(a, f, s);
  }
}

}  // namespace

size_t norm_bwd_part_bytes(long long tokens, int L, int C) {
  const int K = (L + 1) * (L + 1);
  size_t rows = 0;
  for (int type : {SEQ_F32, SEQ_BF16}) {
    const Form f = norm_form(type, C, L, true);
    rows = std::max(rows, f.row.tokens ? (size_t)row_bwd_blocks(tokens, f.row) * (L + 2)
                                       : (size_t)wide_bwd_blocks(tokens, L, f.wide.threads) * (K + 1));
  }
  return rows * C * sizeof(float);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  const Form f = norm_form(a.type, a.C, a.L, false);
  return a.type == SEQ_BF16 ? norm_typed<bf16>(a, f, s) : norm_typed<float>(a, f, s);
}

hipError_t launch_norm_backward(const NormBwdArgs& a, hipStream_t s) {
  const Form f = norm_form(a.type, a.C, a.L, true);
  return a.type == SEQ_BF16 ? norm_typed<bf16>(a, f, s) : norm_typed<float>(a, f, s);
}

}  // namespace cgconv
