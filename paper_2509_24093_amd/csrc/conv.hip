// Short causal convolution of every column (component k, channel c) over the
// tokens, width W = 2..8, for gfx950:
//
//   z[t,k,c] = sum_{j<W} w[j,l(k),c] x[t-j,k,c] + [k = 0] bias[c]
//   y_0 = z_0 sigmoid(z_0) (or z_0),  y_k = z_k
//
// A thread takes V neighbouring columns over a chunk of tokens and keeps the
// last inputs in registers, so x is read once but for the W - 1 tokens before
// a chunk; the next four tokens are asked for, as stored, while four are computed
// (bf16, 4 x 8192 tokens of 2048 channels: forward 71 -> 51 us, backward 157 ->
// 104).  The backward walks a chunk in the same direction: it forms z again,
// gz = gy y'(z), adds gz[t] x[t-j] to gw in registers and emits
// gx[t] = sum_j w[j] gz[t+j] W - 1 tokens later; the tokens behind a chunk are
// formed twice.  Both are streams, in fp32 bound by HBM (8 x 16384 tokens of 49 x 32:
// 4.9 and 4.5 TB/s of what must move), in bf16 the backward by its vector
// operations (4.0 TB/s).  A block's chunks add their
// gw through LDS, the blocks' sums are added by a second kernel in a fixed
// order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

constexpr int kThreads = 256;
constexpr int kAhead = 4;  // tokens loaded ahead of their use

struct ConvShape {
  int cols;    // columns groups of V: K C / V
  int width;   // column groups per block, a power of two <= 64; kThreads / width chunks
  int colblocks;  // blocks over the columns, the fastest part of the block index
  int chunk;   // tokens per chunk
  int chunks;  // per batch element
  long long units;  // B * chunks
};

__device__ __forceinline__ int length_of(const ConvArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.N) : a.N;
}

// (the reciprocal to one unit in the last place; a division would be ten instructions)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// Weights of the thread's columns (j < a.W only) and the bias (component 0).
template <int V, int WM>
__device__ __forceinline__ void load_weights(const ConvArgs& a, int k, int c, float (&w)[WM][V], float (&b)[V]) {
  const int l = (int)__builtin_sqrtf((float)k + 0.5f);
#pragma unroll
  for (int j = 0; j < WM; ++j) {
#pragma unroll
    for (int e = 0; e < V; ++e) w[j][e] = 0.f;
    if (j < a.W) load_vec(a.weight + ((long long)j * (a.L + 1) + l) * a.C + c, w[j]);
  }
#pragma unroll
  for (int e = 0; e < V; ++e) b[e] = 0.f;
  if (k == 0 && a.bias) load_vec(a.bias + c, b);
}

// Input of token t of the batch element (t < len): x, the state before the
// first token, or zero.
template <class T, int V>
__device__ __forceinline__ void load_token(const T* x, const T* state, int t, int W, long long KC, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = 0.f;
  if (t >= 0)
    load_vec(x + t * KC, v);
  else if (state && t >= 1 - W)
    load_vec(state + (t + W - 1) * KC, v);
}

template <class T, int V, int WM>
__global__ __launch_bounds__(kThreads) void conv_kernel(ConvArgs a, ConvShape sh) {
  const int rowblock = blockIdx.x / sh.colblocks;
  const int col = (blockIdx.x - rowblock * sh.colblocks) * sh.width + (threadIdx.x & (sh.width - 1));
  const long long unit = (long long)rowblock * (kThreads / sh.width) + threadIdx.x / sh.width;
  if (col >= sh.cols || unit >= sh.units) return;
  const int b = (int)(unit / sh.chunks), ch = (int)(unit - (long long)b * sh.chunks);
  const long long KC = (long long)a.K * a.C;
  const int e0 = col * V, k = e0 / a.C, c = e0 - k * a.C;
  const int len = length_of(a, b);
  const T* x = static_cast<const T*>(a.x) + (long long)b * a.N * KC + e0;
  const T* state = a.state_in ? static_cast<const T*>(a.state_in) + (long long)b * (a.W - 1) * KC + e0 : nullptr;
  T* y = static_cast<T*>(a.y) + (long long)b * a.N * KC + e0;
  float w[WM][V], bias[V];
  load_weights<V, WM>(a, k, c, w, bias);
  const bool act = a.activation && k == 0;
  const int t0 = ch * sh.chunk, t1 = min(a.N, t0 + sh.chunk), t2 = min(t1, len);
  float row[WM - 1 + kAhead][V];  // row[WM - 1 + i]: token t + i
  if (t0 < t2) {
#pragma unroll
    for (int j = 1; j < WM; ++j) {
      if (j < a.W)
        load_token(x, state, t0 - j, a.W, KC, row[WM - 1 - j]);
      else {
#pragma unroll
        for (int e = 0; e < V; ++e) row[WM - 1 - j][e] = 0.f;
      }
    }
  }
  Raw<T, V> ahead[kAhead];  // the next tokens as stored, asked for while these are computed
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i].load(x + (long long)min(t + i, t2 - 1) * KC);
  };
  if (t0 < t2) fetch(t0);
  for (int t = t0; t < t2; t += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead[i].widen_to(row[WM - 1 + i]);
    fetch(t + kAhead);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t + i >= t2) break;
      float z[V];
#pragma unroll
      for (int e = 0; e < V; ++e) z[e] = bias[e];
#pragma unroll
      for (int j = 0; j < WM; ++j)
        if (j < a.W) {
#pragma unroll
          for (int e = 0; e < V; ++e) z[e] = fmaf(w[j][e], row[WM - 1 + i - j][e], z[e]);
        }
      if (act) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] *= sigmoid(z[e]);
      }
      store_vec(y + (t + i) * KC, z);
    }
#pragma unroll
    for (int j = 0; j < WM - 1; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) row[j][e] = row[j + kAhead][e];
  }
  const float zero[V] = {};
  for (int t = max(t0, t2); t < t1; ++t) store_vec(y + t * KC, zero);
  if (a.state_out && ch == 0) {
    T* out = static_cast<T*>(a.state_out) + (long long)b * (a.W - 1) * KC + e0;
    for (int j = 0; j < a.W - 1; ++j) {
      float v[V];
      load_token(x, state, len - (a.W - 1) + j, a.W, KC, v);
      store_vec(out + j * KC, v);
    }
  }
}

// One token: y and the state, moved on by one row, in place.
template <class T, int V, int WM>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(ConvArgs a, int cols, long long threads) {
  const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (id >= threads) return;
  const long long b = id / cols;
  const int e0 = (int)(id - b * cols) * V, k = e0 / a.C, c = e0 - k * a.C;
  const long long KC = (long long)a.K * a.C;
  T* state = static_cast<T*>(a.state_out) + b * (a.W - 1) * KC + e0;
  float w[WM][V], z[V], row[WM][V];  // row[j]: the input j tokens ago
  load_vec(static_cast<const T*>(a.x) + b * KC + e0, row[0]);
#pragma unroll
  for (int j = 1; j < WM; ++j)
    if (j < a.W) load_vec(state + (a.W - 1 - j) * KC, row[j]);
  load_weights<V, WM>(a, k, c, w, z);
#pragma unroll
  for (int j = 0; j < WM; ++j)
    if (j < a.W) {
#pragma unroll
      for (int e = 0; e < V; ++e) z[e] = fmaf(w[j][e], row[j][e], z[e]);
    }
  if (a.activation && k == 0) {
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] *= sigmoid(z[e]);
  }
  store_vec(static_cast<T*>(a.y) + b * KC + e0, z);
#pragma unroll
  for (int j = 0; j < WM - 1; ++j)
    if (j < a.W - 1) store_vec(state + (a.W - 2 - j) * KC, row[j]);
}

// Backward from the zero state.  part: [row blocks][W, then gb][K C].
template <class T, int V, int WM>
__global__ __launch_bounds__(kThreads) void conv_bwd_kernel(ConvBwdArgs g, ConvShape sh) {
  __shared__ float lds[kThreads * V];
  const ConvArgs& a = g.a;
  const int lane = threadIdx.x & (sh.width - 1), slot = threadIdx.x / sh.width, slots = kThreads / sh.width;
  const int rowblock = blockIdx.x / sh.colblocks;
  const int col = (blockIdx.x - rowblock * sh.colblocks) * sh.width + lane;
  const long long unit = (long long)rowblock * slots + slot;
  const bool here = col < sh.cols && unit < sh.units;
  const long long KC = (long long)a.K * a.C;
  const int e0 = col * V;
  float gw[WM][V], gb[V];
#pragma unroll
  for (int e = 0; e < V; ++e) gb[e] = 0.f;
#pragma unroll
  for (int j = 0; j < WM; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) gw[j][e] = 0.f;
  if (here) {
    const int b = (int)(unit / sh.chunks), ch = (int)(unit - (long long)b * sh.chunks);
    const int k = e0 / a.C, c = e0 - k * a.C;
    const int len = length_of(a, b);
    const T* x = static_cast<const T*>(a.x) + (long long)b * a.N * KC + e0;
    const T* gy = static_cast<const T*>(g.gy) + (long long)b * a.N * KC + e0;
    T* gx = g.gx ? static_cast<T*>(g.gx) + (long long)b * a.N * KC + e0 : nullptr;
    float w[WM][V], bias[V];
    load_weights<V, WM>(a, k, c, w, bias);
    const bool act = a.activation && k == 0;
    const int t0 = ch * sh.chunk, t1 = min(a.N, t0 + sh.chunk);
    float row[WM][V], gz[WM][V];  // [j]: j tokens ago
#pragma unroll
    for (int j = 0; j < WM; ++j) {
#pragma unroll
      for (int e = 0; e < V; ++e) row[j][e] = gz[j][e] = 0.f;
      // row[j] becomes row[j + 1] at the first token
      if (j + 1 < a.W && t0 < len) load_token<T, V>(x, nullptr, t0 - 1 - j, a.W, KC, row[j]);
    }
    const int end = t1 + WM - 1, there = min(end, len);
    Raw<T, V> xr[kAhead], gr[kAhead];  // the next tokens as stored, asked for while these are computed
    auto fetch = [&](int t) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const long long at = (long long)max(min(t + i, there - 1), 0) * KC;
        xr[i].load(x + at);
        gr[i].load(gy + at);
      }
    };
    fetch(t0);
    for (int tb = t0; tb < end; tb += kAhead) {
      float xn[kAhead][V], gn[kAhead][V];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        xr[i].widen_to(xn[i]);
        gr[i].widen_to(gn[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          xn[i][e] = tb + i < there ? xn[i][e] : 0.f;
          gn[i][e] = tb + i < there ? gn[i][e] : 0.f;
        }
      }
      fetch(tb + kAhead);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int t = tb + i;
        if (t >= end) break;
#pragma unroll
        for (int j = WM - 1; j > 0; --j)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            row[j][e] = row[j - 1][e];
            gz[j][e] = gz[j - 1][e];
          }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          row[0][e] = xn[i][e];
          gz[0][e] = gn[i][e];
        }
        if (act && t < len) {
          float z[V];
#pragma unroll
          for (int e = 0; e < V; ++e) z[e] = bias[e];
#pragma unroll
          for (int j = 0; j < WM; ++j)
            if (j < a.W) {
#pragma unroll
              for (int e = 0; e < V; ++e) z[e] = fmaf(w[j][e], row[j][e], z[e]);
            }
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float s = sigmoid(z[e]);
            gz[0][e] *= s * fmaf(z[e], 1.f - s, 1.f);
          }
        }
        if (t < t1) {
#pragma unroll
          for (int j = 0; j < WM; ++j)
            if (j < a.W) {
#pragma unroll
              for (int e = 0; e < V; ++e) gw[j][e] = fmaf(gz[0][e], row[j][e], gw[j][e]);
            }
#pragma unroll
          for (int e = 0; e < V; ++e) gb[e] += gz[0][e];
        }
        const int to = t - (WM - 1);
        if (gx && to >= t0) {
          float o[V];
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = 0.f;
#pragma unroll
          for (int j = 0; j < WM; ++j)
            if (j < a.W) {
#pragma unroll
              for (int e = 0; e < V; ++e) o[e] = fmaf(w[j][e], gz[WM - 1 - j][e], o[e]);
            }
          store_vec(gx + to * KC, o);
        }
      }
    }
  }
  if (!g.part) return;
  float* part = g.part + (long long)rowblock * (a.W + 1) * KC + e0;
#pragma unroll
  for (int j = 0; j <= WM; ++j) {
    if (j < WM && j >= a.W) continue;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) lds[threadIdx.x * V + e] = j < WM ? gw[j < WM ? j : 0][e] : gb[e];
    __syncthreads();
    if (slot == 0 && col < sh.cols) {
      float s[V];
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] = 0.f;
      for (int i = 0; i < slots; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] += lds[(i * sh.width + lane) * V + e];
      store_vec(part + (j < WM ? j : a.W) * KC, s);
    }
  }
}

// gw[j][l][c] and gb[c] from the blocks' sums: 64 slices x 16 outputs per block
// (16 x 64 left most of the chip idle: 23 us for 500 outputs of 313 blocks).
constexpr int kSumSlices = 64, kSumLanes = 16;
__global__ __launch_bounds__(kSumSlices * kSumLanes) void conv_sum_kernel(const float* __restrict__ part, int blocks,
                                                                          int W, int L, int K, int C, float* gw,
                                                                          float* gb) {
  __shared__ float lds[kSumSlices][kSumLanes];
  const int lane = threadIdx.x & (kSumLanes - 1), slice = threadIdx.x / kSumLanes;
  const int o = blockIdx.x * kSumLanes + lane;
  const int row = o / C, c = o - row * C;  // row = j (L + 1) + l, or W (L + 1): gb
  const int j = row / (L + 1), l = j < W ? row - j * (L + 1) : 0;
  const bool here = row <= W * (L + 1);
  float s = 0.f;
  if (here) {
    const int n = j < W ? 2 * l + 1 : 1;
    const float* p = part + ((long long)j * K + l * l) * C + c;
    const long long stride = (long long)(W + 1) * K * C;
    if (n == 1) {
#pragma unroll 8
      for (int b = slice; b < blocks; b += kSumSlices) s += p[b * stride];
    } else {
      for (int b = slice; b < blocks; b += kSumSlices) {
#pragma unroll 8
        for (int m = 0; m < n; ++m) s += p[b * stride + (long long)m * C];
      }
    }
  }
  lds[slice][lane] = s;
  __syncthreads();
  for (int n = kSumSlices / 2; n > 0; n /= 2) {
    if (slice < n) lds[slice][lane] += lds[slice + n][lane];
    __syncthreads();
  }
  if (slice == 0 && here) {
    if (j < W) {
      if (gw) gw[o] = lds[0][lane];
    } else if (gb) {
      gb[c] = lds[0][lane];
    }
  }
}

// Chunks as long as leaves this many columns in flight over all threads: short
// ones read the tokens between them twice and write more partial sums, long ones
// leave the chip idle (4 x 5000 tokens of 36 x 20 in vectors of four: 2^18 columns
// forward 21 us, backward 44, 2^19 22 and 54; 4 x 2048 of 16 x 33 one by one: 2^18 10
// and 22, 2^16 13 and 28).
constexpr long long kWantedColumns = 1 << 18;

ConvShape conv_shape(int64_t B, int64_t N, int K, int64_t C, int V) {
  ConvShape s;
  s.cols = (int)(K * C / V);
  s.width = 1;
  while (s.width < 64 && s.width < s.cols) s.width *= 2;
  s.colblocks = (s.cols + s.width - 1) / s.width;
  s.chunk = 64;
  while (s.chunk > 8 && B * ((N + s.chunk - 1) / s.chunk) * s.cols * V < kWantedColumns) s.chunk /= 2;
  s.chunks = (int)((N + s.chunk - 1) / s.chunk);
  s.units = B * s.chunks;
  return s;
}

long long row_blocks(const ConvShape& s) {
  const int slots = kThreads / s.width;
  return (s.units + slots - 1) / slots;
}

template <class T, int V, int WM>
hipError_t conv_fwd(const ConvArgs& a, hipStream_t s) {
  const ConvShape sh = conv_shape(a.B, a.N, a.K, a.C, V);
  const long long blocks = row_blocks(sh) * sh.colblocks;
  if (!launch_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((conv_kernel<T, V, WM>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, sh);
  return hipGetLastError();
}

template <class T, int V, int WM>
hipError_t conv_step(const ConvArgs& a, hipStream_t s) {
  const int cols = a.K * a.C / V;
  const long long threads = (long long)a.B * cols;
  const long long blocks = (threads + kThreads - 1) / kThreads;
  if (!launch_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((conv_step_kernel<T, V, WM>), dim3((unsigned)blocks), dim3(kThreads), 0, s, a, cols, threads);
  return hipGetLastError();
}

template <class T, int V, int WM>
hipError_t conv_bwd(const ConvBwdArgs& g, hipStream_t s) {
  const ConvArgs& a = g.a;
  const ConvShape sh = conv_shape(a.B, a.N, a.K, a.C, V);
  const long long rows = row_blocks(sh);
  if (!launch_fits(rows * sh.colblocks, kThreads)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((conv_bwd_kernel<T, V, WM>), dim3((unsigned)(rows * sh.colblocks)), dim3(kThreads), 0, s, g, sh);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !g.part) return e;
  const int outputs = (a.W * (a.L + 1) + 1) * a.C;
  hipLaunchKernelGGL(conv_sum_kernel, dim3((outputs + kSumLanes - 1) / kSumLanes), dim3(kSumSlices * kSumLanes), 0, s,
                     g.part, (int)rows, a.W, a.L, a.K, a.C, g.gw, g.gb);
  return hipGetLastError();
}

enum Pass { kForward, kStep, kBackward };

template <class T, int V, Pass P>
hipError_t by_width(const ConvBwdArgs& g, hipStream_t s) {
  if constexpr (P == kForward) return g.a.W <= 4 ? conv_fwd<T, V, 4>(g.a, s) : conv_fwd<T, V, 8>(g.a, s);
  if constexpr (P == kStep) return g.a.W <= 4 ? conv_step<T, V, 4>(g.a, s) : conv_step<T, V, 8>(g.a, s);
  if constexpr (P == kBackward) return g.a.W <= 4 ? conv_bwd<T, V, 4>(g, s) : conv_bwd<T, V, 8>(g, s);
}

// Four columns a thread at most: the registers of eight taps.
// Only vectors that divide a row: full ones with a row's last in part were slower where
// none divides it (forward and backward of 4 x 2048 tokens, bf16: 1001 channels 18 and 34
// us against 18 and 38, 16 x 33 10 and 23 against 14 and 39).
int conv_vec(int type, int64_t C) { return std::min(4, seq_vec(type, C)); }

template <Pass P>
hipError_t dispatch(const ConvBwdArgs& g, hipStream_t s) {
  const int v = conv_vec(g.a.type, g.a.C);
  if (g.a.W < 2 || g.a.W > kConvMaxWidth) return hipErrorInvalidValue;
  if (g.a.type == SEQ_BF16) {
    switch (v) {
      case 4: return by_width<bf16, 4, P>(g, s);
      case 2: return by_width<bf16, 2, P>(g, s);
      default: return by_width<bf16, 1, P>(g, s);
    }
  }
  switch (v) {
    case 4: return by_width<float, 4, P>(g, s);
    case 2: return by_width<float, 2, P>(g, s);
    default: return by_width<float, 1, P>(g, s);
  }
}

}  // namespace

size_t conv_bwd_part_bytes(int64_t B, int64_t N, int K, int64_t C) {
  const ConvShape s = conv_shape(B, N, K, C, conv_vec(SEQ_F32, C));  // bf16 takes the same vectors
  return (size_t)row_blocks(s) * (kConvMaxWidth + 1) * K * C * sizeof(float);
}

hipError_t launch_conv(const ConvArgs& a, hipStream_t s) {
  ConvBwdArgs g{};
  g.a = a;
  return dispatch<kForward>(g, s);
}

hipError_t launch_conv_step(const ConvArgs& a, hipStream_t s) {
  ConvBwdArgs g{};
  g.a = a;
  return dispatch<kStep>(g, s);
}

hipError_t launch_conv_backward(const ConvBwdArgs& g, hipStream_t s) { return dispatch<kBackward>(g, s); }

}  // namespace cgconv
