// Shared by the kernels that normalise by degree (norm.hip, residual.hip): the launch
// shapes of their two forms, the sums over rows, degrees and blocks.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

// n / d of n d < 2^32 by one multiply-high (magic = floor((2^32 - 1) / d) + 1; d >= 2;
// d = 1 has no such magic and is n itself).
__device__ __forceinline__ int divide(int n, uint32_t magic) {
  return magic ? (int)__umulhi((uint32_t)n, magic) : n;
}
uint32_t magic_of(int d) { return d > 1 ? 0xFFFFFFFFu / (uint32_t)d + 1 : 0; }

// Launch shape of the row form.
struct RowShape {
  int lanes;    // per row (a power of two)
  int threads;  // per block
  int passes;   // rows per thread: a multiple of kPassStep
  int tokens;   // per block
  uint32_t magic = 0;  // of K
};

__device__ __forceinline__ int degree_of(int comp) { return (int)__builtin_sqrtf((float)comp + 0.5f); }

// out[i] = f(sum of the rows of degree i % (L+1) of token i / (L+1)), 16 lanes per
// sum: a lane reads one row's sum (the first also the 17th row's of degree 8), so
// the block waits for one LDS access and four lane steps rather than for a loop
// over the rows.
template <class F>
__device__ __forceinline__ void degree_sums(const float* rowsum, float* out, int toks, int degs, int K, int threads,
                                            F f) {
  const int lane = threadIdx.x & 15;
  for (int i = threadIdx.x >> 4; i < toks * degs; i += threads >> 4) {
    const int tok = i / degs, l = i - tok * degs;
    const float* p = rowsum + tok * K + l * l;
    float s = lane < 2 * l + 1 ? p[lane] : 0.f;
    if (lane == 0 && l == 8) s += p[16];
    s = group_sum(s, 16);
    if (lane == 0) out[i] = f(s, i, l);
  }
}

// Sum over the block (up to 16 waves), the same in every thread.
__device__ __forceinline__ float block_sum(float v, float* lds, int threads) {
  v = group_sum(v, 64);
  if (threads == 64) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < threads / 64; ++w) s += lds[w];
  return s;
}

// Sums of two values over the block in one exchange.
__device__ __forceinline__ void block_sum2(float& u, float& v, float* lds, int threads) {
  u = group_sum(u, 64);
  v = group_sum(v, 64);
  if (threads == 64) return;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    lds[threadIdx.x >> 6] = u;
    lds[16 + (threadIdx.x >> 6)] = v;
  }
  __syncthreads();
  u = v = 0.f;
  for (int w = 0; w < threads / 64; ++w) {
    u += lds[w];
    v += lds[16 + w];
  }
}

// ---- launch shapes -----------------------------------------------------------------

constexpr int kPassStep = 2;

// Row form: the block and pass count that leave the fewest lanes without a row,
// at most max_passes rows per thread, max_threads threads and max_values values
// per block; a block larger than 256 threads has to gain `gain` of its lanes for
// it; 0 tokens if a token does not fit.  At B=8 N=16384 L=6 C=32 (49 rows of 8
// lanes): forward, 512 threads x 4 rows (96% of the lanes) against 256 x 8 and 256
// x 4 (77%), whole step 753, 773, 772 us; backward, whose blocks wait for each
// other at two barriers a tile, 256 x 4 against 512 x 4: 773, 784, with the 8-bit
// input 778, 899.
RowShape row_shape(int C, int K, int V, int max_passes, int max_threads, int max_values, double gain) {
  RowShape best{1, 0, 0, 0, magic_of(K)};
  const int vecs = (C + V - 1) / V;
  if (vecs > 64) return best;
  while (best.lanes < vecs) best.lanes *= 2;
  double score = 0;
  for (int threads = 256; threads <= max_threads; threads *= 2) {
    const int per = threads / best.lanes;
    for (int passes = kPassStep; passes <= max_passes; passes += kPassStep) {
      const int tokens = per * passes / K;
      if (tokens < 1 || threads * passes * V > max_values) continue;
      const double use = (double)(tokens * K) / (per * passes);
      if (use > score + (threads > best.threads && best.threads ? gain : 0.02)) {
        score = use;
        best.threads = threads;
        best.passes = passes;
        best.tokens = tokens;
      }
    }
  }
  return best;
}

struct WideShape {
  int threads = 0, vecs = 0;  // vecs: per thread, a power of two
};
// Wide form: the usual number of vectors a thread, more where 1024 threads would not do.
WideShape wide_shape(int n, int V, int usual) {
  WideShape w;
  const int total = (n + V - 1) / V;
  for (w.threads = 64; w.threads < 1024; w.threads *= 2)
    if (total <= w.threads * usual) break;
  w.vecs = 1;
  while (w.vecs * w.threads < total) w.vecs *= 2;
  return w;
}

}  // namespace

}  // namespace cgconv
