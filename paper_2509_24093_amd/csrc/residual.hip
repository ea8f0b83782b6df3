// The norms on both sides of a residual connection in one pass, forward and backward, for
// gfx950.  For a token with the stream x, a block's output u and a gate (K = (L+1)^2
// components of C channels; norms by degree as in norm.hip):
//
//   h = (u - [l = 0] mean_c u) ru_l            ru_l = 1 / sqrt(mean_{m,c} (.)^2 + eps)
//   r = x + scale[c] silu(gate[c]) wp[l,c] h   the stream behind the block
//   k = (r - [l = 0] mean_c r) rr_l            y = w[l,c] k + [l = 0] bias[c]
//
// Backward, from the gradients gr of r and gy of y, with s = silu(gate):
//
//   g = w gy            G = gr + rr_l (g - [l = 0] mean g - k mean(g k))       gx = G
//   p = G scale s wp    gu = ru_l (p - [l = 0] mean p - h mean(p h))
//   ggate[c] = silu'(gate) sum_{l,m} G scale wp h
//   gw[l,c] = sum_{t,m} gy k,  gb[c] = sum_t gy_0,  Q[l,c] = sum_{t,m} G s h,
//   gwp = scale Q,  gscale[c] = sum_l wp Q
//
// r is formed again from x, u and the gate: the stored r has been rounded, and gw, a sum in
// 32 bits, would see it.  Both directions are bound by memory: every input is read once and
// every output written once, but in the third form.
//
// Three forms.  Rows (one component's C channels): as in norm.hip a block takes whole tokens of
// several rows a pass, each row on a power of two of lanes with one vector each (four fp32 or
// eight bf16 channels; in the backward four of either where two rows a thread hold a token).  It
// takes rows of at most 64 vectors whose (L+1)^2 rows a block holds: its threads times the rows of
// each over a row's lanes, 4096 / lanes in the forward, in the backward 2048 (fp32) and 1024 (bf16)
// / lanes.  Longer rows of scalars (L = 0): a block per token, in registers.  What is left, a block
// per token whose threads keep to a channel each and read the inputs again from the caches for
// every sum: rows of vectors of more than 256 fp32 or 512 bf16 channels; at L = 8 more than 128 or
// 256 in the forward; in the backward more than 128 from L = 5 on and 64 at L = 8, in bf16 also more
// than 256 at L = 4.  It runs at 1.2 to 2.2 TB/s forward and 0.35 to 1.9 backward, the rows at 2.2 to
// 5.4 and 0.9 to 4.6 (2.4e8 values of bf16, half as many of fp32; slowest where C is just above a
// power of two, fastest where lanes and rows are full).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "norm_common.h"

namespace cgconv {

namespace {

// 1 / (1 + e^-z) within two units of the last place down to z = -87 (3.83 half units with silu's own
// product over 2.9e5 gates, tests/test_residual_rows_gpu.py), zero or below 2^-125 under it: a
// power of 2 whose argument is reduced with log2(e) in two parts, as Cody and Waite do it, so that
// its rounding is made up for, and a reciprocal with one step of Newton's method.  With expf and a division, which are twice
// the instructions, the wide rows' backward is bound by them (16384 tokens of 4096: 331 us, so
// 271), and the rows' forward waits for its tokens' gates (131072 of L=6 C=32: 712 us, so 627).
__device__ __forceinline__ float sigmoid(float z) {
  const float c = __builtin_amdgcn_fmed3f(z, -1e4f, 1e4f), t = -c * 1.44269502f;       // log2(e) = the one
  const float rest = fmaf(-c, 1.92596299e-8f, fmaf(-c, 1.44269502f, -t));              // constant + the other
  const float e = __builtin_amdgcn_exp2f(t) * fmaf(rest, 0.693147181f, 1.f);
  const float d = fminf(1.f + e, 3e38f), r = __builtin_amdgcn_rcpf(d);
  return fmaf(fmaf(-d, r, 1.f), r, r);
}
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }
__device__ __forceinline__ float silu_slope(float z) {
  const float s = sigmoid(z);
  return s * fmaf(z, 1.f - s, 1.f);
}

// Statistics of a token: mean of u, ru of every degree, mean of r, rr of every degree.
__host__ __device__ inline int stats_of(int L) { return 2 * (L + 2); }

// V values of a per-channel array from c on, or `none` where there is no array.
template <bool TAIL, class T, int V>
__device__ __forceinline__ void load_or(const T* p, int n, float none, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = none;
  if (p) load_part<TAIL>(p, n, v);
}

// V elements at an offset in a tile, zeros where `there` is false (then the tile's first).
template <bool TAIL, class T, int V>
__device__ __forceinline__ void load_there(const T* tile, int at, int n, bool there, float (&v)[V]) {
  if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    if (there) load_part<true>(tile + at, n, v);
  } else {
    load_vec(tile + (there ? at : 0), v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = there ? v[e] : 0.f;
  }
}

// silu(gate) of a block's tokens, one value a thread at a time, where several rows share it.
template <class T>
__device__ __forceinline__ void stage_gates(const T* gate, float* to, int n, int threads) {
  for (int i = threadIdx.x; i < n; i += threads) to[i] = silu(widen(gate[i]));
}
// V of them at channel c of a token of the block (gate: the block's first token); ones without a gate.
template <bool TAIL, class T, int V>
__device__ __forceinline__ void gates_of(const T* gate, const float* staged, int K, int tok, int C, int c, float (&s)[V]) {
  if (K > 1 || !gate) {
    load_or<TAIL>(gate ? staged + tok * C + c : nullptr, C - c, 1.f, s);
    return;
  }
  load_or<TAIL>(gate + (long long)tok * C + c, C - c, 0.f, s);
#pragma unroll
  for (int e = 0; e < V; ++e) s[e] = silu(s[e]);
}

// ---- rows ------------------------------------------------------------------------------

// Dynamic LDS: a row's sums (twice), a degree's (twice), silu(gate) of the tokens.
template <class T, int V, int R, bool TAIL>
__global__ void residual_rows_kernel(ResidualArgs a, RowShape sh) {
  extern __shared__ float lds[];
  const int tid = threadIdx.x, per = sh.threads / sh.lanes;
  const int j = tid & (sh.lanes - 1), rg = tid / sh.lanes;
  const int c = j * V, left = a.C - c, degs = a.L + 1;
  const bool col = left > 0;
  const long long t0 = (long long)blockIdx.x * sh.tokens;
  const int toks = (int)min((long long)sh.tokens, a.tokens - t0);
  const int rows = toks * a.K;
  float* sums = lds;
  float* sums2 = sums + sh.tokens * a.K;
  float* ru = sums2 + sh.tokens * a.K;
  float* rr = ru + sh.tokens * degs;
  float* gates = rr + sh.tokens * degs;
  const long long base = t0 * a.K * a.C;
  const T* u = static_cast<const T*>(a.u) + base;
  const T* x = static_cast<const T*>(a.x) + base;
  float* stats = a.stats ? a.stats + t0 * stats_of(a.L) : nullptr;
  float v[R][V], w[R][V];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = w[i][e] = 0.f;
    if (col && r < rows) {
      load_part<TAIL>(u + (long long)r * a.C + c, left, v[i]);
      load_part<TAIL>(x + (long long)r * a.C + c, left, w[i]);
    }
  }
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + t0 * a.C : nullptr;
  if (gate && a.K > 1) stage_gates(gate, gates, toks * a.C, sh.threads);
  // deviations from the mean of the invariants' row, sums of squares
  const auto center = [&](float (&d)[R][V], float* to, int at) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = i * per + rg, tok = divide(r, sh.magic);
      if (r - tok * a.K == 0) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) s += d[i][e];
        const float mean = group_sum(s, sh.lanes) / (float)a.C;
#pragma unroll
        for (int e = 0; e < V; ++e) d[i][e] = e < left ? d[i][e] - mean : 0.f;
        if (stats && j == 0 && r < rows) stats[(long long)tok * stats_of(a.L) + at] = mean;
      }
      float q = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) q = fmaf(d[i][e], d[i][e], q);
      q = group_sum(q, sh.lanes);
      if (j == 0 && r < rows) to[r] = q;
    }
  };
  const auto factors = [&](const float* from, float* to, int at) {
    __syncthreads();
    degree_sums(from, to, toks, degs, a.K, sh.threads, [&](float s, int i, int l) {
      const float r = 1.f / __builtin_sqrtf(s / (float)((2 * l + 1) * a.C) + a.eps);
      if (stats) stats[(long long)(i / degs) * stats_of(a.L) + at + l] = r;
      return r;
    });
    __syncthreads();
  };
  center(v, sums, 0);
  factors(sums, ru, 1);
  float sc[V];
  load_or<TAIL>(col ? a.scale ? a.scale + c : nullptr : nullptr, left, 1.f, sc);
  T* ro = static_cast<T*>(a.r) + base;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
    if (!col || r >= rows) continue;
    const int tok = divide(r, sh.magic), comp = r - tok * a.K, l = degree_of(comp);
    const float m = ru[tok * degs + l];
    float p[V], s[V];
    load_or<TAIL>(a.post_weight ? a.post_weight + l * a.C + c : nullptr, left, 1.f, p);
    gates_of<TAIL>(gate, gates, a.K, tok, a.C, c, s);
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = e < left ? fmaf(v[i][e] * m, p[e] * (s[e] * sc[e]), w[i][e]) : 0.f;
    store_part<TAIL>(ro + (long long)r * a.C + c, left, v[i]);
  }
  center(v, sums2, a.L + 2);
  factors(sums2, rr, a.L + 3);
  T* y = static_cast<T*>(a.y) + base;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
    if (!col || r >= rows) continue;
    const int tok = divide(r, sh.magic), comp = r - tok * a.K, l = degree_of(comp);
    const float m = rr[tok * degs + l];
    float p[V], b[V];
    load_or<TAIL>(a.weight ? a.weight + l * a.C + c : nullptr, left, 1.f, p);
    load_or<TAIL>(comp == 0 && a.bias ? a.bias + c : nullptr, left, 0.f, b);
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = fmaf(v[i][e] * m, p[e], b[e]);
    store_part<TAIL>(y + (long long)r * a.C + c, left, v[i]);
  }
}

// Block b takes tiles b, b + gridDim.x, ... of sh.tokens tokens; the next tile's gates are
// staged, and its statistics, behind this one's first sums, so that the threads meet twice a
// tile.  Dynamic LDS: sums of rows (twice), silu(gate) (of two tiles) and the rows' products for
// the gate's gradient while the tiles run; then the staging of the parameters' sums.  Partial
// sums of block b: part[b][gw of L + 1 degrees, Q of L + 1 degrees, gb][C].  131072 tokens of
// L=6 C=32 in fp32, 4.9 GB: 1.21 ms, 4.1 TB/s; 1.80 with five meetings a tile; with the next
// tile asked for ahead it needs more registers, so that a block less fits a CU, and is slower.
constexpr int kResidualRowThreads = 512;

template <class T, int V, int R, int MAXT, bool TAIL>
__global__ __launch_bounds__(MAXT, R * V <= 8 ? 3 : 2) void residual_rows_bwd_kernel(ResidualBwdArgs g, RowShape sh,
                                                                                      long long tiles) {
  extern __shared__ float lds[];
  const ResidualArgs& a = g.a;
  const int tid = threadIdx.x, per = sh.threads / sh.lanes;
  const int j = tid & (sh.lanes - 1), rg = tid / sh.lanes;
  const int c = j * V, left = a.C - c, degs = a.L + 1, ns = stats_of(a.L);
  const bool col = left > 0, shared = a.gate && a.K > 1;
  const int rowsum = sh.tokens * a.K, gated = sh.tokens * a.C;
  float* sums = lds;
  float* gates = sums + 2 * rowsum;
  float* stats = gates + (a.K > 1 ? 2 * gated : 0);  // of two tiles
  float* prod = stats + 2 * sh.tokens * ns;          // [rows][C]; the gates too only where K > 1
  float* slices = prod + rowsum * a.C;               // of prod's sums over a token's rows, [slice][gated]
  const int count = max(1, min(8, sh.threads / gated));
  float gw[R][V], gq[R][V], gb[V], f[R][V], w[R][V];  // f: scale post_weight
  int tok[R], comp[R], deg[R];
  float share[R];  // of an element in its degree's mean
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = i * per + rg;
    tok[i] = divide(r, sh.magic);
    comp[i] = r - tok[i] * a.K;
    deg[i] = degree_of(comp[i]);
    share[i] = 1.f / (float)((2 * deg[i] + 1) * a.C);
#pragma unroll
    for (int e = 0; e < V; ++e) gw[i][e] = gq[i][e] = 0.f;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) gb[e] = 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    float sc[V];
    const int at = deg[i] * a.C + c;
    const bool on = col && tok[i] < sh.tokens;
    load_or<TAIL>(on && a.scale ? a.scale + c : nullptr, left, 1.f, sc);
    load_or<TAIL>(on && a.post_weight ? a.post_weight + at : nullptr, left, 1.f, f[i]);
    load_or<TAIL>(on && a.weight ? a.weight + at : nullptr, left, 1.f, w[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) f[i][e] *= sc[e];
  }
  const auto stage = [&](long long tile, int half) {
    const long long t0 = tile * sh.tokens;
    const int toks = (int)min((long long)sh.tokens, a.tokens - t0);
    for (int i = tid; i < toks * ns; i += sh.threads) stats[half * sh.tokens * ns + i] = a.stats[t0 * ns + i];
    if (shared) stage_gates(static_cast<const T*>(a.gate) + t0 * a.C, gates + half * gated, toks * a.C, sh.threads);
  };
  if (blockIdx.x < tiles) stage(blockIdx.x, 0);
  __syncthreads();
  int half = 0;
  // the gate's gradient of a tile, a slice of the rows a thread: the slices are added one
  // barrier later, in the next tile
  const auto gate_out = [&](long long tile) {
    const long long t0 = tile * sh.tokens;
    const int n = (int)min((long long)sh.tokens, a.tokens - t0) * a.C;
    for (int o = tid; o < n; o += sh.threads) {
      float s = 0.f;
      for (int i = 0; i < count; ++i) s += slices[i * gated + o];
      const long long at = t0 * a.C + o;
      static_cast<T*>(g.ggate)[at] = (T)(s * silu_slope(widen(static_cast<const T*>(a.gate)[at])));
    }
  };
  const bool gates_wanted = g.ggate && a.K > 1;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x, half ^= 1) {
    const long long t0 = tile * sh.tokens, base = t0 * a.K * a.C;
    const int toks = (int)min((long long)sh.tokens, a.tokens - t0);
    const T* gate = a.gate ? static_cast<const T*>(a.gate) + t0 * a.C : nullptr;
    bool there[R];
#pragma unroll
    for (int i = 0; i < R; ++i) there[i] = col && tok[i] < toks;
    const auto gate_of = [&](int i, float (&s)[V]) {
      if (TAIL || !shared) {
        gates_of<TAIL>(there[i] ? gate : nullptr, gates + half * gated, a.K, tok[i], a.C, c, s);
      } else {
        load_vec(gates + half * gated + (there[i] ? tok[i] * a.C + c : 0), s);
      }
    };
    float h[R][V], k[R][V], gy[R][V], G[R][V], fu[R], fr[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = (i * per + rg) * a.C + c;
      load_there<TAIL>(static_cast<const T*>(a.u) + base, at, left, there[i], h[i]);
      load_there<TAIL>(static_cast<const T*>(a.x) + base, at, left, there[i], k[i]);
      load_there<TAIL>(static_cast<const T*>(g.gy) + base, at, left, there[i], gy[i]);
      load_there<TAIL>(static_cast<const T*>(g.gr ? g.gr : g.gy) + base, at, left, there[i] && g.gr, G[i]);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float* st = stats + half * sh.tokens * ns + (there[i] ? tok[i] * ns : 0);
      const float m = comp[i] == 0 ? st[0] : 0.f, m2 = comp[i] == 0 ? st[a.L + 2] : 0.f;
      fu[i] = there[i] ? st[1 + deg[i]] : 0.f;  // zero: nothing of a lane without a vector remains
      fr[i] = there[i] ? st[a.L + 3 + deg[i]] : 0.f;
      float s[V];
      gate_of(i, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float x = (h[i][e] - m) * fu[i], y = (fmaf(x, s[e] * f[i][e], k[i][e]) - m2) * fr[i];
        h[i][e] = there[i] ? x : 0.f;
        k[i][e] = there[i] ? y : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float q = 0.f, sum = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        gw[i][e] = fmaf(gy[i][e], k[i][e], gw[i][e]);
        if (comp[i] == 0) gb[e] += gy[i][e];
        gy[i][e] *= w[i][e];
        q = fmaf(gy[i][e], k[i][e], q);
        sum += gy[i][e];
      }
      q = group_sum(q, sh.lanes);
      if (comp[i] == 0) {
        sum = group_sum(sum, sh.lanes) * share[i];
#pragma unroll
        for (int e = 0; e < V; ++e) gy[i][e] -= sum;
      }
      if (j == 0 && tok[i] < toks) sums[i * per + rg] = q;
    }
    // the mean over a row's degree, added by the row's lanes
    const auto mean_of = [&](int i, const float* from) {
      float s = 0.f;
      if (tok[i] < toks)
        for (int m = j; m < 2 * deg[i] + 1; m += sh.lanes) s += from[tok[i] * a.K + deg[i] * deg[i] + m];
      return group_sum(s, sh.lanes) * share[i];
    };
    __syncthreads();
    if (gates_wanted && tile != blockIdx.x) gate_out(tile - gridDim.x);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const bool on = there[i];
      const float d = mean_of(i, sums);
      float s[V], o[V];
      gate_of(i, s);
#pragma unroll
      for (int e = 0; e < V; ++e) G[i][e] = fmaf(fr[i], fmaf(-k[i][e], d, gy[i][e]), G[i][e]);
      if (on && g.gx)
        store_part<TAIL>(static_cast<T*>(g.gx) + base + (long long)(i * per + rg) * a.C + c, left, G[i]);
      float q = 0.f, sum = 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float gh = TAIL && e >= left ? 0.f : G[i][e] * h[i][e];
        gq[i][e] = fmaf(gh, s[e], gq[i][e]);
        o[e] = gh * f[i][e];
        k[i][e] = TAIL && e >= left ? 0.f : G[i][e] * (s[e] * f[i][e]);  // p of the header
        q = fmaf(k[i][e], h[i][e], q);
        sum += k[i][e];
      }
      if (on && g.ggate) {
        if (a.K > 1) {
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (!TAIL || e < left) prod[(i * per + rg) * a.C + c + e] = o[e];
        } else {
          const long long at = (t0 + tok[i]) * a.C + c;
          float z[V];
          load_part<TAIL>(static_cast<const T*>(a.gate) + at, left, z);
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] *= silu_slope(z[e]);
          store_part<TAIL>(static_cast<T*>(g.ggate) + at, left, o);
        }
      }
      q = group_sum(q, sh.lanes);
      if (comp[i] == 0) {
        sum = group_sum(sum, sh.lanes) * share[i];
#pragma unroll
        for (int e = 0; e < V; ++e) k[i][e] -= sum;
      }
      if (j == 0 && tok[i] < toks) sums[rowsum + i * per + rg] = q;
    }
    if (tile + gridDim.x < tiles) stage(tile + gridDim.x, half ^ 1);
    __syncthreads();
    if (g.gu) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float d = mean_of(i, sums + rowsum);
        if (!there[i]) continue;
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fu[i] * fmaf(-h[i][e], d, k[i][e]);
        store_part<TAIL>(static_cast<T*>(g.gu) + base + (long long)(i * per + rg) * a.C + c, left, o);
      }
    }
    if (gates_wanted) {
      for (int i = tid; i < count * gated; i += sh.threads) {
        const int slice = i / gated, o = i - slice * gated, t = o / a.C;
        float s = 0.f;
        for (int m = slice; m < a.K; m += count) s += prod[(t * a.K + m) * a.C + o - t * a.C];
        slices[i] = s;
      }
    }
    // The next tile writes the first sums, which nobody has read since the last barrier, then
    // everything else behind its own first.
  }
  if (gates_wanted && blockIdx.x < tiles) {
    __syncthreads();
    gate_out(blockIdx.x + (tiles - 1 - blockIdx.x) / gridDim.x * gridDim.x);
  }
  if (!g.part) return;
  float* part = g.part + (long long)blockIdx.x * (2 * degs + 1) * a.C;
  const auto reduce = [&](const float (&v)[R][V], float* to) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (col) {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (!TAIL || e < left) lds[(i * per + rg) * a.C + c + e] = v[i][e];
      }
    __syncthreads();
    for (int o = tid; o < degs * a.C; o += sh.threads) {
      const int l = o / a.C, ch = o - l * a.C;
      float s = 0.f;
      for (int t = 0; t < sh.tokens; ++t)
        for (int m = 0; m < 2 * l + 1; ++m) s += lds[(t * a.K + l * l + m) * a.C + ch];
      to[o] = s;
    }
  };
  reduce(gw, part);
  reduce(gq, part + degs * a.C);
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
    part[2 * degs * a.C + ch] = s;
  }
}

// ---- wide rows of scalars ------------------------------------------------------------------

// Block per token, its C channels in registers.  16384 tokens of 4096 in bf16, 0.67 GB: 143 us,
// 4.7 TB/s.
template <class T, int V, int R, int MAXT, bool TAIL>
__global__ __launch_bounds__(MAXT) void residual_wide_kernel(ResidualArgs a) {
  __shared__ float lds[16];
  const int tid = threadIdx.x, threads = blockDim.x, n = a.C;
  const long long t = blockIdx.x, base = t * n;
  float v[R][V], w[R][V], s[R][V];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = w[i][e] = 0.f, s[i][e] = 1.f;
    if (e0 >= n) continue;
    load_part<TAIL>(static_cast<const T*>(a.u) + base + e0, n - e0, v[i]);
    load_part<TAIL>(static_cast<const T*>(a.x) + base + e0, n - e0, w[i]);
    if (a.gate) load_part<TAIL>(static_cast<const T*>(a.gate) + base + e0, n - e0, s[i]);
  }
  // the mean goes, the factor of the norm comes back
  const auto center = [&](int at) {
    float sum = 0.f, q = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) sum += v[i][e];
    const float mean = block_sum(sum, lds, threads) / (float)n;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int left = n - (i * threads + tid) * V;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[i][e] = (TAIL ? e < left : left > 0) ? v[i][e] - mean : 0.f;
        q = fmaf(v[i][e], v[i][e], q);
      }
    }
    const float r = 1.f / __builtin_sqrtf(block_sum(q, lds, threads) / (float)n + a.eps);
    if (a.stats && tid == 0) {
      a.stats[t * 4 + at] = mean;
      a.stats[t * 4 + at + 1] = r;
    }
    return r;
  };
  const float ru = center(0);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
    if (e0 >= n) continue;
    float p[V], sc[V];
    load_or<TAIL>(a.post_weight ? a.post_weight + e0 : nullptr, n - e0, 1.f, p);
    load_or<TAIL>(a.scale ? a.scale + e0 : nullptr, n - e0, 1.f, sc);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float f = a.gate ? silu(s[i][e]) : 1.f;
      v[i][e] = !TAIL || e < n - e0 ? fmaf(v[i][e] * ru, p[e] * (f * sc[e]), w[i][e]) : 0.f;
    }
    store_part<TAIL>(static_cast<T*>(a.r) + base + e0, n - e0, v[i]);
  }
  const float rr = center(2);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
    if (e0 >= n) continue;
    float p[V], b[V];
    load_or<TAIL>(a.weight ? a.weight + e0 : nullptr, n - e0, 1.f, p);
    load_or<TAIL>(a.bias ? a.bias + e0 : nullptr, n - e0, 0.f, b);
#pragma unroll
    for (int e = 0; e < V; ++e) v[i][e] = fmaf(v[i][e] * rr, p[e], b[e]);
    store_part<TAIL>(static_cast<T*>(a.y) + base + e0, n - e0, v[i]);
  }
}

// Block `slot` takes tokens slot, slot + gridDim.x, ..., each asked for while the one before is
// computed; partial sums part[slot][gw, Q, gb][C].  16384 tokens of 4096 in bf16, 1.07 GB:
// 271 us, 4.0 TB/s.
template <class T, int V, int R, int MAXT, bool TAIL>
__global__ __launch_bounds__(MAXT, MAXT == 1024 ? 4 : 2) void residual_wide_bwd_kernel(ResidualBwdArgs g) {
  __shared__ float lds[32];
  const ResidualArgs& a = g.a;
  const int tid = threadIdx.x, threads = blockDim.x, n = a.C;
  float gw[R][V], gq[R][V], gb[R][V];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) gw[i][e] = gq[i][e] = gb[i][e] = 0.f;
  Raw<T, V> hr[R], kr[R], yr[R], Gr[R], zr[R];
  float4 st;
  const auto fetch = [&](long long t) {
    const long long base = t * n;
    st = reinterpret_cast<const float4*>(a.stats)[t];  // mean of u, ru, mean of r, rr
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
      if (e0 >= n) continue;
      hr[i].template load_part<TAIL>(static_cast<const T*>(a.u) + base + e0, n - e0);
      kr[i].template load_part<TAIL>(static_cast<const T*>(a.x) + base + e0, n - e0);
      yr[i].template load_part<TAIL>(static_cast<const T*>(g.gy) + base + e0, n - e0);
      if (g.gr) Gr[i].template load_part<TAIL>(static_cast<const T*>(g.gr) + base + e0, n - e0);
      if (a.gate) zr[i].template load_part<TAIL>(static_cast<const T*>(a.gate) + base + e0, n - e0);
    }
  };
  if (blockIdx.x < a.tokens) fetch(blockIdx.x);
  for (long long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const long long base = t * n;
    const float mu = st.x, ru = st.y, mr = st.z, rr = st.w;
    float h[R][V], k[R][V], y[R][V], G[R][V], z[R][V];
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = k[i][e] = y[i][e] = G[i][e] = z[i][e] = 0.f;
      if ((i * threads + tid) * V >= n) continue;
      hr[i].widen_to(h[i]);
      kr[i].widen_to(k[i]);
      yr[i].widen_to(y[i]);
      if (g.gr) Gr[i].widen_to(G[i]);
      if (a.gate) zr[i].widen_to(z[i]);
    }
    if (t + gridDim.x < a.tokens) fetch(t + gridDim.x);
    float q = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
      if (e0 >= n) continue;
      float p[V], sc[V], w[V];
      load_or<TAIL>(a.post_weight ? a.post_weight + e0 : nullptr, n - e0, 1.f, p);
      load_or<TAIL>(a.scale ? a.scale + e0 : nullptr, n - e0, 1.f, sc);
      load_or<TAIL>(a.weight ? a.weight + e0 : nullptr, n - e0, 1.f, w);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float f = a.gate ? silu(z[i][e]) : 1.f;
        h[i][e] = (h[i][e] - mu) * ru;
        k[i][e] = (fmaf(h[i][e], p[e] * (f * sc[e]), k[i][e]) - mr) * rr;
        gw[i][e] = fmaf(y[i][e], k[i][e], gw[i][e]);
        gb[i][e] += y[i][e];
        y[i][e] *= w[e];
        q = fmaf(y[i][e], k[i][e], q);
        sum += y[i][e];
      }
    }
    block_sum2(q, sum, lds, threads);
    const float d = q / (float)n, mean = sum / (float)n;
    q = sum = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
      if (e0 >= n) continue;
      float p[V], sc[V], o[V];
      load_or<TAIL>(a.post_weight ? a.post_weight + e0 : nullptr, n - e0, 1.f, p);
      load_or<TAIL>(a.scale ? a.scale + e0 : nullptr, n - e0, 1.f, sc);
#pragma unroll
      for (int e = 0; e < V; ++e) G[i][e] = fmaf(rr, fmaf(-k[i][e], d, y[i][e] - mean), G[i][e]);
      if (g.gx) store_part<TAIL>(static_cast<T*>(g.gx) + base + e0, n - e0, G[i]);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float f = a.gate ? silu(z[i][e]) : 1.f;
        const float gh = G[i][e] * h[i][e];
        gq[i][e] = fmaf(gh, f, gq[i][e]);
        o[e] = gh * (sc[e] * p[e]) * silu_slope(z[i][e]);
        k[i][e] = TAIL && e >= n - e0 ? 0.f : G[i][e] * (p[e] * (f * sc[e]));  // p of the header
        q = fmaf(k[i][e], h[i][e], q);
        sum += k[i][e];
      }
      if (g.ggate) store_part<TAIL>(static_cast<T*>(g.ggate) + base + e0, n - e0, o);
    }
    if (!g.gu) continue;
    block_sum2(q, sum, lds, threads);
    const float d2 = q / (float)n, mean2 = sum / (float)n;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int e0 = (i * threads + tid) * V;
      if (e0 >= n) continue;
      float o[V];
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = ru * fmaf(-h[i][e], d2, k[i][e] - mean2);
      store_part<TAIL>(static_cast<T*>(g.gu) + base + e0, n - e0, o);
    }
  }
  if (!g.part) return;
  float* part = g.part + (long long)blockIdx.x * 3 * n;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int e0 = (i * threads + tid) * V;
    if (e0 >= n) continue;
    store_part<TAIL>(part + e0, n - e0, gw[i]);
    store_part<TAIL>(part + n + e0, n - e0, gq[i]);
    store_part<TAIL>(part + 2 * n + e0, n - e0, gb[i]);
  }
}

// ---- wide rows of vectors --------------------------------------------------------------------

constexpr int kChannelThreads = 512;

// Block per token; f(element, degree, channel) of all elements of a degree, a thread keeping to
// its channels, summed.
template <class F>
__device__ __forceinline__ float over_degree(int l, int C, F f) {
  float s = 0.f;
  for (int c = threadIdx.x; c < C; c += kChannelThreads)
    for (int m = l * l; m < (l + 1) * (l + 1); ++m) s += f(m * C + c, c);
  return s;
}

template <class T>
__global__ __launch_bounds__(kChannelThreads) void residual_channels_kernel(ResidualArgs a) {
  __shared__ float lds[16];
  const long long t = blockIdx.x, base = t * a.K * a.C;
  const T* u = static_cast<const T*>(a.u) + base;
  const T* x = static_cast<const T*>(a.x) + base;
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + t * a.C : nullptr;
  float* stats = a.stats ? a.stats + t * stats_of(a.L) : nullptr;
  for (int l = 0; l <= a.L; ++l) {
    const float n = (float)((2 * l + 1) * a.C);
    const float* p = a.post_weight ? a.post_weight + l * a.C : nullptr;
    // mean (of the invariants only) and factor of the norm of f
    const auto norm = [&](auto f, float& mean, float& r) {
      mean = l == 0 ? block_sum(over_degree(l, a.C, f), lds, kChannelThreads) / n : 0.f;
      const float q = over_degree(l, a.C, [&](int at, int c) {
        const float d = f(at, c) - mean;
        return d * d;
      });
      r = 1.f / __builtin_sqrtf(block_sum(q, lds, kChannelThreads) / n + a.eps);
    };
    float mu, ru, mr, rr;
    norm([&](int at, int) { return widen(u[at]); }, mu, ru);
    const auto stream = [&](int at, int c) {
      const float s = gate ? silu(widen(gate[c])) : 1.f;
      return fmaf((widen(u[at]) - mu) * ru, (p ? p[c] : 1.f) * (s * (a.scale ? a.scale[c] : 1.f)), widen(x[at]));
    };
    norm(stream, mr, rr);
    over_degree(l, a.C, [&](int at, int c) {
      const float r = stream(at, c);
      static_cast<T*>(a.r)[base + at] = (T)r;
      static_cast<T*>(a.y)[base + at] = (T)fmaf((r - mr) * rr, a.weight ? a.weight[l * a.C + c] : 1.f,
                                                l == 0 && a.bias ? a.bias[c] : 0.f);
      return 0.f;
    });
    if (stats && threadIdx.x == 0) {
      if (l == 0) {
        stats[0] = mu;
        stats[a.L + 2] = mr;
      }
      stats[1 + l] = ru;
      stats[a.L + 3 + l] = rr;
    }
  }
}

// Partial sums as in the row form, which their threads hold in memory.  Dynamic LDS: the
// gate's gradient of the token.
template <class T>
__global__ __launch_bounds__(kChannelThreads) void residual_channels_bwd_kernel(ResidualBwdArgs g) {
  extern __shared__ float products[];
  __shared__ float lds[32];
  const ResidualArgs& a = g.a;
  const int tid = threadIdx.x, C = a.C, degs = a.L + 1;
  float* part = g.part ? g.part + (long long)blockIdx.x * (2 * degs + 1) * C : nullptr;
  if (part)
    for (int i = 0; i < 2 * degs + 1; ++i)
      for (int c = tid; c < C; c += kChannelThreads) part[i * C + c] = 0.f;
  for (long long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
    const long long base = t * a.K * C;
    const T* u = static_cast<const T*>(a.u) + base;
    const T* x = static_cast<const T*>(a.x) + base;
    const T* gy = static_cast<const T*>(g.gy) + base;
    const T* gr = g.gr ? static_cast<const T*>(g.gr) + base : nullptr;
    const T* gate = a.gate ? static_cast<const T*>(a.gate) + t * C : nullptr;
    const float* stats = a.stats + t * stats_of(a.L);
    for (int c = tid; c < C; c += kChannelThreads) products[c] = 0.f;
    for (int l = 0; l < degs; ++l) {
      const float n = (float)((2 * l + 1) * C), ru = stats[1 + l], rr = stats[a.L + 3 + l];
      const float mu = l == 0 ? stats[0] : 0.f, mr = l == 0 ? stats[a.L + 2] : 0.f;
      float q = 0.f, sum = 0.f;
      for (int c = tid; c < C; c += kChannelThreads) {
        const float f = (a.post_weight ? a.post_weight[l * C + c] : 1.f) *
                        ((gate ? silu(widen(gate[c])) : 1.f) * (a.scale ? a.scale[c] : 1.f));
        const float w = a.weight ? a.weight[l * C + c] : 1.f;
        float gw = 0.f, gb = 0.f;
        for (int m = l * l; m < (l + 1) * (l + 1); ++m) {
          const int at = m * C + c;
          const float k = (fmaf((widen(u[at]) - mu) * ru, f, widen(x[at])) - mr) * rr, y = widen(gy[at]);
          gw = fmaf(y, k, gw);
          gb += y;
          q = fmaf(y * w, k, q);
          sum = fmaf(y, w, sum);
        }
        if (part) {
          part[l * C + c] += gw;
          if (l == 0) part[2 * degs * C + c] += gb;
        }
      }
      block_sum2(q, sum, lds, kChannelThreads);
      const float d = q / n, mean = l == 0 ? sum / n : 0.f;
      // G, and p of the header, of a channel's components
      const auto each = [&](auto f) {
        for (int c = tid; c < C; c += kChannelThreads) {
          const float po = a.post_weight ? a.post_weight[l * C + c] : 1.f, sc = a.scale ? a.scale[c] : 1.f;
          const float s = gate ? silu(widen(gate[c])) : 1.f, w = a.weight ? a.weight[l * C + c] : 1.f;
          float total = 0.f;
          for (int m = l * l; m < (l + 1) * (l + 1); ++m) {
            const int at = m * C + c;
            const float h = (widen(u[at]) - mu) * ru;
            const float k = (fmaf(h, po * (s * sc), widen(x[at])) - mr) * rr;
            const float G = (gr ? widen(gr[at]) : 0.f) + rr * fmaf(-k, d, fmaf(widen(gy[at]), w, -mean));
            f(at, h, G, G * (po * (s * sc)));
            total = fmaf(G, h, total);
          }
          f.end(c, total, s, sc * po);
        }
      };
      struct Sums {
        const ResidualBwdArgs& g;
        float* part;
        float* products;
        T* gx;
        float &q, &sum;
        __device__ void operator()(int at, float h, float G, float p) {
          if (gx) gx[at] = (T)G;
          q = fmaf(p, h, q);
          sum += p;
        }
        __device__ void end(int c, float total, float s, float f) {
          if (part) part[c] += total * s;
          products[c] = fmaf(total, f, products[c]);
        }
      };
      q = sum = 0.f;
      each(Sums{g, part ? part + (degs + l) * C : nullptr, products,
                g.gx ? static_cast<T*>(g.gx) + base : nullptr, q, sum});
      if (!g.gu) continue;
      block_sum2(q, sum, lds, kChannelThreads);
      struct Out {
        T* gu;
        float ru, d, mean;
        __device__ void operator()(int at, float h, float, float p) { gu[at] = (T)(ru * fmaf(-h, d, p - mean)); }
        __device__ void end(int, float, float, float) {}
      };
      each(Out{static_cast<T*>(g.gu) + base, ru, q / n, l == 0 ? sum / n : 0.f});
    }
    if (g.ggate)
      for (int c = tid; c < C; c += kChannelThreads)
        static_cast<T*>(g.ggate)[t * C + c] = (T)(products[c] * silu_slope(widen(gate[c])));
  }
}

// Adds the blocks' partial sums [blocks][gw of L + 1 degrees, Q of L + 1, gb][C] in a fixed
// order: block of 16 slices x 64 outputs.  gscale needs all degrees of a channel: its thread
// adds them one after the other.
constexpr int kResidualSlices = 16;
__global__ __launch_bounds__(64 * kResidualSlices) void residual_sum_kernel(ResidualBwdArgs g, int blocks) {
  __shared__ float lds[kResidualSlices][64];
  const ResidualArgs& a = g.a;
  const int degs = a.L + 1, rows = 2 * degs + 1;
  const int o = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
  const int what = o / a.C, c = o - what * a.C;  // rows of part; behind them gscale
  const auto total = [&](int row) {
    float s = 0.f;
    if (row < rows) {
      const float* p = g.part + (long long)row * a.C + c;
#pragma unroll 4
      for (int b = slice; b < blocks; b += kResidualSlices) s += p[(long long)b * rows * a.C];
    }
    __syncthreads();
    lds[slice][threadIdx.x & 63] = s;
    __syncthreads();
    float t = 0.f;
    for (int i = 0; i < kResidualSlices; ++i) t += lds[i][threadIdx.x & 63];
    return t;
  };
  const float t = total(what);
  const bool first = slice == 0;
  if (first && what < degs && g.gw) g.gw[o] = t;
  if (first && what >= degs && what < 2 * degs && g.gpost) g.gpost[o - degs * a.C] = t * (a.scale ? a.scale[c] : 1.f);
  if (first && what == 2 * degs && g.gb) g.gb[c] = t;
  if (!g.gscale) return;
  float s = 0.f;
  for (int l = 0; l < degs; ++l) {  // every thread: the block's barriers are in it
    const float q = total(what == rows ? degs + l : rows);
    if (what == rows) s = fmaf(a.post_weight ? a.post_weight[l * a.C + c] : 1.f, q, s);
  }
  if (first && what == rows) g.gscale[c] = s;
}

// ---- launch shapes -----------------------------------------------------------------------------

constexpr int kFwdPasses = 4;
constexpr int bwd_passes(int V) { return 16 / V; }
constexpr int kRowValues = 8192;    // of one array in the backward's tiles: 32 KiB of products
constexpr int kRowBlocks = 768, kChannelBlocks = 512;  // of 256 threads: three a CU are resident

enum class Kind { kRows, kWide, kChannels };
struct Form {
  Kind kind;
  int v;
  bool tail;
  RowShape row{};
  WideShape wide{};
};

constexpr int usual_vecs(int V, bool backward) { return backward ? 16 / V : 2; }

Form residual_form(int type, int C, int L, bool backward) {
  const int K = (L + 1) * (L + 1);
  Form f{Kind::kRows, type == SEQ_BF16 ? 8 : 4, false};
  f.tail = C % f.v != 0;
  if (backward) {
    // Two rows of four channels a thread where a token of them fits a block of 256, so that three
    // waves share a SIMD: 65536 tokens of L=2 C=64 in fp32 238 us, 444 with four rows; in bf16
    // 202, 242 with eight channels; 32768 of L=6 C=32 in bf16 289, 341.  In blocks of 512, of
    // which a CU holds one, they are slower (32768 of L=4 C=128 in bf16 981, 603 with eight
    // channels in 256).
    f.row = row_shape(C, K, 4, 2, 256, kRowValues, 1.0);
    if (f.row.tokens) {
      f.v = 4;
      f.tail = C % 4 != 0;
      return f;
    }
  }
  f.row = backward ? row_shape(C, K, f.v, bwd_passes(f.v), kResidualRowThreads, kRowValues, 1.0)
                   : row_shape(C, K, f.v, kFwdPasses, 1024, 1024 * 32, 0.1);
  if (f.row.tokens) return f;
  f.kind = L == 0 ? Kind::kWide : Kind::kChannels;
  if (L == 0) f.wide = wide_shape(C, f.v, usual_vecs(f.v, backward));
  return f;
}

size_t rows_lds(const RowShape& sh, int K, int L, int C, bool gate) {
  return ((size_t)sh.tokens * 2 * (K + L + 1) + (gate && K > 1 ? (size_t)sh.tokens * C : 0)) * sizeof(float);
}
size_t rows_bwd_lds(const RowShape& sh, int K, int L, int C) {
  const size_t rows = (size_t)(sh.threads / sh.lanes) * sh.passes;
  const int slices = std::max(1, std::min(8, sh.threads / (sh.tokens * C)));
  const size_t shared = K > 1 ? sh.tokens * (size_t)(K + 2 + slices) * C : 0;
  return std::max(sh.tokens * (size_t)(2 * (K + stats_of(L))) + shared, rows * C) * sizeof(float);
}
int residual_blocks(const Form& f, long long tokens) {
  if (f.kind == Kind::kRows) {
    const long long tiles = (tokens + f.row.tokens - 1) / f.row.tokens;
    return (int)std::min<long long>(tiles, kRowBlocks * 256 / f.row.threads);
  }
  if (f.kind == Kind::kWide) return (int)std::min<long long>(tokens, std::max(64, std::min(2048, (1 << 18) / f.wide.threads)));
  return (int)std::min<long long>(tokens, kChannelBlocks);
}

// f of the vectors a thread holds and of the most threads a block of them has (the forms of
// wide_shape for more than 64 vectors).
template <int R, int MAXT>
struct Shape {
  static constexpr int kVecs = R, kThreads = MAXT;
};
template <class T, class F>
hipError_t wide_forward(const WideShape& w, F f) {
  if (w.vecs == 2) return w.threads <= 256 ? f(Shape<2, 256>()) : f(Shape<2, 1024>());
  if constexpr (sizeof(T) == 4) {
    if (w.vecs == 4) return f(Shape<4, 1024>());
  }
  return hipErrorInvalidValue;
}
template <class T, class F>
hipError_t wide_backward(const WideShape& w, F f) {
  constexpr int R = sizeof(T) == 4 ? 4 : 2;
  if constexpr (R == 4) {
    if (w.vecs == 2) return f(Shape<2, 64>());
  }
  if (w.vecs != R) return hipErrorInvalidValue;
  return w.threads <= 256 ? f(Shape<R, 256>()) : w.threads <= 512 ? f(Shape<R, 512>()) : f(Shape<R, 1024>());
}

template <class T, int V, bool TAIL>
hipError_t residual_any(const ResidualArgs& a, const Form& f, hipStream_t s) {
  if (f.kind == Kind::kRows) {
    // few tokens: a CU each, rather than blocks filled to the last lane (64 tokens of L=2 C=4:
    // 12 us in two blocks, 5.7 in 64)
    RowShape row = f.row;
    row.tokens = (int)std::min<long long>(row.tokens, (a.tokens + 255) / 256);
    const long long blocks = (a.tokens + row.tokens - 1) / row.tokens;
    const size_t lds = rows_lds(row, a.K, a.L, a.C, a.gate != nullptr);
    if (!launch_fits(blocks, row.threads) || lds > 160 * 1024) return hipErrorInvalidConfiguration;
    const auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(row.threads), lds, s, a, row);
      return hipGetLastError();
    };
    return f.row.passes == 2 ? run(residual_rows_kernel<T, V, 2, TAIL>) : run(residual_rows_kernel<T, V, 4, TAIL>);
  }
  if (!launch_fits(a.tokens, f.wide.threads)) return hipErrorInvalidConfiguration;
  return wide_forward<T>(f.wide, [&](auto shape) {
    constexpr int R = decltype(shape)::kVecs, MAXT = decltype(shape)::kThreads;
    hipLaunchKernelGGL((residual_wide_kernel<T, V, R, MAXT, TAIL>), dim3((unsigned)a.tokens), dim3(f.wide.threads), 0,
                       s, a);
    return hipGetLastError();
  });
}

template <class T, int V, bool TAIL>
hipError_t residual_any(const ResidualBwdArgs& g, const Form& f, hipStream_t s) {
  const int blocks = residual_blocks(f, g.a.tokens);
  if (f.kind == Kind::kRows) {
    const size_t lds = rows_bwd_lds(f.row, g.a.K, g.a.L, g.a.C);
    if (lds > 160 * 1024) return hipErrorInvalidConfiguration;
    const long long tiles = (g.a.tokens + f.row.tokens - 1) / f.row.tokens;
    const auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(blocks), dim3(f.row.threads), lds, s, g, f.row, tiles);
      return hipGetLastError();
    };
    if constexpr (V == 4) {
      if (f.row.passes == 2) return run(residual_rows_bwd_kernel<T, V, 2, 256, TAIL>);
    }
    if constexpr (V * sizeof(T) == 16) {
      constexpr int R = bwd_passes(V);
      return f.row.threads <= 256 ? run(residual_rows_bwd_kernel<T, V, R, 256, TAIL>)
                                  : run(residual_rows_bwd_kernel<T, V, R, 512, TAIL>);
    }
  }
  if constexpr (V * sizeof(T) == 16) {
    return wide_backward<T>(f.wide, [&](auto shape) {
      constexpr int R = decltype(shape)::kVecs, MAXT = decltype(shape)::kThreads;
      hipLaunchKernelGGL((residual_wide_bwd_kernel<T, V, R, MAXT, TAIL>), dim3(blocks), dim3(f.wide.threads), 0, s, g);
      return hipGetLastError();
    });
  }
  return hipErrorInvalidValue;
}

template <class T, class Args>
hipError_t residual_typed(const Args& a, const Form& f, hipStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  if constexpr (V > 4 && std::is_same<Args, ResidualBwdArgs>::value) {
    if (f.v == 4) return f.tail ? residual_any<T, 4, true>(a, f, s) : residual_any<T, 4, false>(a, f, s);
  }
  return f.tail ? residual_any<T, V, true>(a, f, s) : residual_any<T, V, false>(a, f, s);
}

}  // namespace

size_t residual_part_bytes(long long tokens, int L, int C) {
  size_t blocks = 0;
  for (int type : {SEQ_F32, SEQ_BF16})
    blocks = std::max(blocks, (size_t)residual_blocks(residual_form(type, C, L, true), tokens));
  return blocks * (2 * (L + 1) + 1) * C * sizeof(float);
}

hipError_t launch_residual(const ResidualArgs& a, hipStream_t s) {
  const Form f = residual_form(a.type, a.C, a.L, false);
  if (f.kind == Kind::kChannels) {
    if (!launch_fits(a.tokens, kChannelThreads)) return hipErrorInvalidConfiguration;
    if (a.type == SEQ_BF16)
      hipLaunchKernelGGL(residual_channels_kernel<bf16>, dim3((unsigned)a.tokens), dim3(kChannelThreads), 0, s, a);
    else
      hipLaunchKernelGGL(residual_channels_kernel<float>, dim3((unsigned)a.tokens), dim3(kChannelThreads), 0, s, a);
    return hipGetLastError();
  }
  return a.type == SEQ_BF16 ? residual_typed<bf16>(a, f, s) : residual_typed<float>(a, f, s);
}

hipError_t launch_residual_backward(const ResidualBwdArgs& g, hipStream_t s) {
  const Form f = residual_form(g.a.type, g.a.C, g.a.L, true);
  const int blocks = residual_blocks(f, g.a.tokens);
  hipError_t e;
  if (f.kind == Kind::kChannels) {
    const size_t lds = g.a.C * sizeof(float);
    if (g.a.type == SEQ_BF16)
      hipLaunchKernelGGL(residual_channels_bwd_kernel<bf16>, dim3(blocks), dim3(kChannelThreads), lds, s, g);
    else
      hipLaunchKernelGGL(residual_channels_bwd_kernel<float>, dim3(blocks), dim3(kChannelThreads), lds, s, g);
    e = hipGetLastError();
  } else {
    e = g.a.type == SEQ_BF16 ? residual_typed<bf16>(g, f, s) : residual_typed<float>(g, f, s);
  }
  if (e != hipSuccess || !g.part) return e;
  const int outputs = (2 * (g.a.L + 1) + 2) * g.a.C;
  hipLaunchKernelGGL(residual_sum_kernel, dim3((outputs + 63) / 64), dim3(64 * kResidualSlices), 0, s, g, blocks);
  return hipGetLastError();
}

}  // namespace cgconv
