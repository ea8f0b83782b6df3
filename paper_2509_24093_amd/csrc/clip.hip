// Clipping of many tensors by their global norm, for gfx950: norm = sqrt(sum g^2) over all
// values of all tensors, out = g min(1, max_norm / (norm + eps)).  The squares are added in
// 64 bits: neither the square of a large value nor the sum of very many overflows or loses
// a small one, and at memory speed the two fp64 instructions a value are free.
//
// Two launches of up to kClipTensors tensors each, whose addresses and sizes are the kernel's
// arguments: nothing is copied to the device.  A block of the first adds a piece of one
// tensor; every block of the second adds the blocks' sums again, in the same order, rather
// than waiting for a launch between (2048 sums are 16 KiB from L2).  More sums than that are
// brought to one by a launch of their own.  Bound by memory: two reads (the factor is not
// known before the norm) and one write of every value; in place with a factor of 1 nothing is
// written.  290 tensors of 7e8 values, most bf16 (1.7 GB, 0.98 ms at the rate of a large copy):
// 1.03 ms in up to 16384 pieces, 1.09 in 8192, 1.15 in 4096, 1.28 in 2048 without the launch
// between: pieces of one length leave CUs without work at a launch's end.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

constexpr int kClipTensors = 112;  // of a launch: 3.6 KB of arguments
constexpr int kClipThreads = 256;
constexpr int kClipBlocks = 16384;  // sums of one call, and one more for every tensor
constexpr long long kClipPiece = 8192;
constexpr int kClipDirect = 2048;   // sums that every block adds itself

struct Batch {
  const void* g[kClipTensors];
  void* out[kClipTensors];
  long long count[kClipTensors];
  int first[kClipTensors + 1];  // block
  uint8_t half[kClipTensors];   // bf16
  int n;
  long long piece;  // values of a block, a multiple of 8
};

// The tensor of a block and its piece [from, to).
__device__ __forceinline__ int find(const Batch& b, int block, long long& from, long long& to) {
  int lo = 0, hi = b.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (b.first[mid] <= block)
      lo = mid;
    else
      hi = mid;
  }
  from = (block - b.first[lo]) * b.piece;
  to = min(from + b.piece, b.count[lo]);
  return lo;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ double block_total(double v, double* lds) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// f(values, place, how many of them) over a piece, kAhead vectors of a thread in flight.
template <class T, class F>
__device__ __forceinline__ void over_piece(const T* g, long long from, long long to, F f) {
  constexpr int V = 16 / (int)sizeof(T), kAhead = 4, kStep = kClipThreads * V;
  long long at = from + threadIdx.x * V;
  for (; at + (kAhead - 1) * kStep + V <= to; at += kAhead * kStep) {
    Raw<T, V> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) raw[i].load(g + at + i * kStep);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      float v[V];
      raw[i].widen_to(v);
      f(v, at + i * kStep, V);
    }
  }
  for (; at < to; at += kStep) {
    float v[V];
    const int n = (int)min((long long)V, to - at);
    load_part<true>(g + at, n, v);
    f(v, at, n);
  }
}

__global__ __launch_bounds__(kClipThreads) void clip_sum_kernel(Batch b, double* part) {
  __shared__ double lds[4];
  long long from, to;
  const int t = find(b, blockIdx.x, from, to);
  double s = 0.0;
  const auto add = [&](const auto& v, long long, int) {
    for (float x : v) s = fma((double)x, (double)x, s);
  };
  if (b.half[t])
    over_piece(static_cast<const bf16*>(b.g[t]), from, to, add);
  else
    over_piece(static_cast<const float*>(b.g[t]), from, to, add);
  s = block_total(s, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double add_sums(const double* part, int n, double* lds) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kClipThreads) s += part[i];
  return block_total(s, lds);
}

constexpr int kTotalThreads = 1024;
__global__ __launch_bounds__(kTotalThreads) void clip_total_kernel(const double* part, int n, double* total) {
  __shared__ double lds[kTotalThreads / 64];
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kTotalThreads) s += part[i];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = 0.0;
  for (int i = 0; i < kTotalThreads / 64; ++i) s += lds[i];
  *total = s;
}

// The first block of the first launch writes the norm.
__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(Batch b, const double* part, int n, float max_norm,
                                                                  float eps, float* norm) {
  __shared__ double lds[4];
  const double total = sqrt(add_sums(part, n, lds));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
  if (b.n == 0) return;
  // without a limit, or with nothing but zeros and no eps, the values stay
  const double under = total + (double)eps;
  const double ratio = max_norm == __builtin_inff() || under == 0.0 ? 1.0 : (double)max_norm / under;
  const float factor = ratio >= 1.0 ? 1.f : (float)ratio;  // a NaN stays one
  long long from, to;
  const int t = find(b, blockIdx.x, from, to);
  if (factor == 1.f && b.out[t] == b.g[t]) return;
  const auto scale = [&](auto* out) {
    return [=](auto& v, long long at, int m) {
      for (float& x : v) x *= factor;
      store_part<true>(out + at, m, v);
    };
  };
  if (b.half[t])
    over_piece(static_cast<const bf16*>(b.g[t]), from, to, scale(static_cast<bf16*>(b.out[t])));
  else
    over_piece(static_cast<const float*>(b.g[t]), from, to, scale(static_cast<float*>(b.out[t])));
}

long long piece_of(long long n, const int64_t* counts) {
  long long total = 0;
  for (long long i = 0; i < n; ++i) total += counts[i];
  return std::max(kClipPiece, (total / kClipBlocks + 8) / 8 * 8);
}

}  // namespace

size_t clip_workspace_bytes(long long n, const int64_t* counts) {
  const long long piece = piece_of(n, counts);
  long long blocks = 0;
  for (long long i = 0; i < n; ++i) blocks += (counts[i] + piece - 1) / piece;
  return (size_t)(blocks + 1) * sizeof(double);
}

hipError_t launch_clip(const ClipArgs& a, hipStream_t s) {
  const long long piece = piece_of(a.n, a.counts);
  double* part = a.ws + 1;
  int blocks = 0;
  // f of every batch of tensors that have a value, and of its number of blocks
  const auto batches = [&](auto f) {
    Batch b;
    b.n = 0;
    b.piece = piece;
    int used = 0;
    for (long long i = 0; i <= a.n; ++i) {
      if (b.n && (i == a.n || b.n == kClipTensors)) {
        b.first[b.n] = used;
        const hipError_t e = f(b, used);
        if (e != hipSuccess) return e;
        b.n = used = 0;
      }
      if (i == a.n || a.counts[i] == 0) continue;
      b.g[b.n] = a.grads[i];
      b.out[b.n] = a.out[i];
      b.count[b.n] = a.counts[i];
      b.half[b.n] = a.types[i] == SEQ_BF16;
      b.first[b.n++] = used;
      used += (int)((a.counts[i] + piece - 1) / piece);
    }
    return hipSuccess;
  };
  hipError_t e = batches([&](const Batch& b, int used) {
    hipLaunchKernelGGL(clip_sum_kernel, dim3(used), dim3(kClipThreads), 0, s, b, part + blocks);
    blocks += used;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  if (blocks > kClipDirect) {
    hipLaunchKernelGGL(clip_total_kernel, dim3(1), dim3(kTotalThreads), 0, s, part, blocks, a.ws);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    part = a.ws;
    blocks = 1;
  }
  float* norm = a.norm;
  e = batches([&](const Batch& b, int used) {
    hipLaunchKernelGGL(clip_scale_kernel, dim3(used), dim3(kClipThreads), 0, s, b, part, blocks, a.max_norm, a.eps, norm);
    norm = nullptr;
    return hipGetLastError();
  });
  if (e != hipSuccess || !norm) return e;
  Batch none;
  none.n = 0;
  hipLaunchKernelGGL(clip_scale_kernel, dim3(1), dim3(kClipThreads), 0, s, none, part, 0, a.max_norm, a.eps, norm);
  return hipGetLastError();
}

}  // namespace cgconv
