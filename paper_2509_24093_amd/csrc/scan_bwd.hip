// Backward of the selective scan for gfx950, from the zero state (formulas of
// the forward: scan_common.h).  With g_t = dL/dh_t (everything behind t):
//
//   g_t = r_t + C_t gy_t,   r_{t-1} = exp(delta_t A) g_t   (r behind the last token: 0)
//   gC_t[s] = sum_{k,c} gy_t h_t[s],    gB_t[s] = sum_{k,c} g_t[s] delta_t x_t
//   gx_t = delta_t sum_s B_t[s] g_t[s] + D gy_t
//   q_t[s,c] = sum_k r_{t-1}[s] h_{t-1}[s],   gA = sum_{b,t} delta_t q_t
//   gdelta_t = sum_s A q_t[s] + sum_k x_t sum_s B_t[s] g_t[s],   graw = gdelta sigmoid(raw + bias)
//
// The states are formed again rather than kept (S times the input) or run
// backwards (a division by decays that may vanish): chunks of kChunk tokens from
// their start states (the forward's passes 1 and 2), inside a chunk the states
// before every kSub tokens in LDS, the kSub states of a piece in registers.
// Like the states, r enters a chunk from a pass over the chunks in reverse.  gB
// and gC add over the lanes: the 2 SP values of a token are halved from step to
// step, each lane keeping the half of its bit, so 64 lanes x 32 values take 31
// exchanges instead of 192; waves add through LDS, column blocks in a last
// kernel.  No atomics: every sum has a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "scan_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

constexpr float kLn2 = 0.69314718055994530942f;

// Tokens per chunk and per piece, threads per block, by states: the piece's
// states take kSub SP registers, the pieces' starts (chunk / sub - 1) SP threads
// 4 bytes of LDS (48 KiB).
template <int SP>
struct BwdShape {
  static constexpr int kSub = SP == 32 ? 4 : 8;
  static constexpr int kChunk = SP == 32 ? 16 : 32;
  static constexpr int kThreads = SP == 32 ? 128 : 256;
};
int bwd_chunk(int S) { return scan_padded(S) == 32 ? BwdShape<32>::kChunk : BwdShape<16>::kChunk; }
int bwd_threads(int S) { return scan_padded(S) == 32 ? BwdShape<32>::kThreads : BwdShape<16>::kThreads; }

// Pass over the chunks behind the first: the gradient that a chunk's own
// outputs send to the state before it, and its sum of delta.
template <class T, int SP>
__global__ __launch_bounds__(256) void reverse_kernel(ScanBwdArgs g, ScanChunks sh, ScanSpace ws, int colblocks) {
  const ScanArgs& a = g.a;
  const int ch = blockIdx.x / colblocks + 1, b = blockIdx.y;
  const int KC = a.K * a.C;
  const int id = (blockIdx.x - (ch - 1) * colblocks) * blockDim.x + threadIdx.x;
  const bool here = id < KC;
  const int j = here ? id : 0, c = j % a.C;
  const int len = scan_length(a.lengths, b, a.N);
  const int t0 = ch * sh.chunk, t2 = min(min(a.N, t0 + sh.chunk), len);
  float A2[SP], r[SP];
#pragma unroll
  for (int s = 0; s < SP; ++s) {
    A2[s] = s < a.S ? a.A[(long long)c * a.S + s] * kLog2e : 0.f;
    r[s] = 0.f;
  }
  const float bias = a.bias ? a.bias[c] : 0.f;
  const long long row0 = (long long)b * a.N;
  const T* gyp = static_cast<const T*>(g.gy) + row0 * KC + j;
  const T* dp = static_cast<const T*>(a.delta) + row0 * a.C + c;
  const ConstFloats bc = (ConstFloats)(ws.bc + row0 * 2 * SP);
  float total = 0.f;
#pragma unroll 2
  for (int t = t2 - 1; t >= t0; --t) {
    const float d = softplus(widen(dp[(long long)t * a.C]) + bias), gy = widen(gyp[(long long)t * KC]);
    total += d;
    const ConstFloats p = bc + (long long)t * 2 * SP + SP;
#pragma unroll
    for (int s = 0; s < SP; ++s) r[s] = exp2_fast(d * A2[s]) * fmaf(p[s], gy, r[s]);
  }
  if (!here) return;
  float* out = ws.rs + ((long long)b * sh.chunks + ch) * a.S * KC + j;
#pragma unroll
  for (int s = 0; s < SP; ++s)
    if (s < a.S) out[(long long)s * KC] = r[s];
  if (j < a.C) ws.ds[((long long)b * sh.chunks + ch) * a.C + c] = total;
}

__device__ __forceinline__ void swap32(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap16(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}

// One halving over the lanes that differ in `bit` (partners by CTRL, which also
// flips lower bits only): lane keeps v[i], or v[i + N/2] where the bit is set.
template <int CTRL, int N>
__device__ __forceinline__ void halve(float* v, bool bit) {
  if constexpr (N > 1) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float keep = bit ? v[i + N / 2] : v[i], send = bit ? v[i] : v[i + N / 2];
      v[i] = keep + dpp<CTRL>(send);
    }
  } else {
    v[0] += dpp<CTRL>(v[0]);
  }
}

// Sums v[0..N) over the wave: returns the sum of v[index_of(lane)].
template <int N>
__device__ __forceinline__ float wave_scatter_sum(float (&v)[N], int lane) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    swap32(v[i], v[i + N / 2]);
    v[i] += v[i + N / 2];
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    swap16(v[i], v[i + N / 4]);
    v[i] += v[i + N / 4];
  }
  halve<0x140, N / 4>(v, lane & 8);                      // row mirror
  halve<0x141, N / 8>(v, lane & 4);                      // half-row mirror
  halve<0x4E, N / 16>(v, lane & 2);                      // quad_perm 2, 3, 0, 1
  halve<0xB1, (N / 32 > 0 ? N / 32 : 1)>(v, lane & 1);   // quad_perm 1, 0, 3, 2
  return v[0];
}
// Lane bits 5, 4, 3, ... choose the halves from the largest on; the lowest bits
// of fewer than 64 values hold copies.
template <int N>
__device__ __forceinline__ int scatter_index(int lane) { return lane / (64 / N); }

// Block (chunk, column block) of a batch element; thread = column k C + c.
template <class T, int SP>
__global__ __launch_bounds__(BwdShape<SP>::kThreads) void scan_bwd_kernel(ScanBwdArgs g, ScanChunks sh, ScanSpace ws,
                                                                          int colblocks) {
  constexpr int kSub = BwdShape<SP>::kSub, kThreads = BwdShape<SP>::kThreads;
  constexpr int kPieces = BwdShape<SP>::kChunk / kSub, kWaves = kThreads / 64;
  __shared__ float starts[kPieces - 1][SP][kThreads];
  __shared__ float red[kWaves][kSub][2 * SP];
  const ScanArgs& a = g.a;
  const int ch = blockIdx.x / colblocks, cb = blockIdx.x - ch * colblocks, b = blockIdx.y;
  const int KC = a.K * a.C, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int id = cb * kThreads + tid;
  const bool here = id < KC;
  const int j = here ? id : 0, c = j % a.C;
  const int len = scan_length(a.lengths, b, a.N);
  const int t0 = ch * sh.chunk, t1 = min(a.N, t0 + sh.chunk), t2 = min(t1, len);
  const long long row0 = (long long)b * a.N;
  const T* xp = static_cast<const T*>(a.x) + row0 * KC + j;
  const T* gyp = static_cast<const T*>(g.gy) + row0 * KC + j;
  const T* dp = static_cast<const T*>(a.delta) + row0 * a.C + c;
  T* gxp = static_cast<T*>(g.gx) + row0 * KC + j;
  float* gdp = ws.gd + row0 * KC + j;
  const ConstFloats bc = (ConstFloats)(ws.bc + row0 * 2 * SP);
  const long long at = ((long long)b * sh.chunks + ch) * a.S * KC + j;
  float A2[SP], h[SP], r[SP], gA[SP];
#pragma unroll
  for (int s = 0; s < SP; ++s) {
    const bool there = s < a.S && here;
    A2[s] = s < a.S ? a.A[(long long)c * a.S + s] * kLog2e : 0.f;
    h[s] = there && sh.chunks > 1 ? ws.hs[at + (long long)s * KC] : 0.f;
    r[s] = there && sh.chunks > 1 ? ws.rs[at + (long long)s * KC] : 0.f;
    gA[s] = 0.f;
  }
  const float bias = a.bias ? a.bias[c] : 0.f, D = a.D ? a.D[c] : 0.f;
  float gD = 0.f;
  // the states before every piece but the first
#pragma unroll 1
  for (int t = t0; t < t2; ++t) {
    const int n = t - t0;
    if (n > 0 && n % kSub == 0) {
#pragma unroll
      for (int s = 0; s < SP; ++s) starts[n / kSub - 1][s][tid] = h[s];
    }
    if (t - t0 >= (t2 - t0 - 1) / kSub * kSub) break;  // the last piece forms its own
    const float d = softplus(widen(dp[(long long)t * a.C]) + bias);
    const float dx = d * widen(xp[(long long)t * KC]);
    const ConstFloats p = bc + (long long)t * 2 * SP;
#pragma unroll
    for (int s = 0; s < SP; ++s) h[s] = fmaf(exp2_fast(d * A2[s]), h[s], p[s] * dx);
  }
  for (int piece = t2 > t0 ? (t2 - t0 - 1) / kSub : -1; piece >= 0; --piece) {
    const int ts = t0 + piece * kSub, n = min(kSub, t2 - ts);
    float hist[kSub + 1][SP], d[kSub], x[kSub], gy[kSub];
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      const int t = ts + min(i, n - 1);
      const bool on = here && i < n;
      d[i] = widen(dp[(long long)t * a.C]);
      x[i] = on ? widen(xp[(long long)t * KC]) : 0.f;
      gy[i] = on ? widen(gyp[(long long)t * KC]) : 0.f;
    }
#pragma unroll
    for (int s = 0; s < SP; ++s)
      hist[0][s] = piece ? starts[piece - 1][s][tid]
                         : (s < a.S && here && sh.chunks > 1 ? ws.hs[at + (long long)s * KC] : 0.f);
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      if (i < n) {  // uniform
        d[i] = softplus(d[i] + bias);
        const float dx = d[i] * x[i];
        const ConstFloats p = bc + (long long)(ts + i) * 2 * SP;
#pragma unroll
        for (int s = 0; s < SP; ++s) hist[i + 1][s] = fmaf(exp2_fast(d[i] * A2[s]), hist[i][s], p[s] * dx);
      }
    }
#pragma unroll
    for (int i = kSub - 1; i >= 0; --i) {
      if (i < n) {
        const int t = ts + i;
        const ConstFloats p = bc + (long long)t * 2 * SP;
        const float dx = d[i] * x[i];
        float v[2 * SP], into = 0.f, gd = 0.f;
#pragma unroll
        for (int s = 0; s < SP; ++s) {
          const float gs = fmaf(p[SP + s], gy[i], r[s]);
          v[s] = gs * dx;
          v[SP + s] = hist[i + 1][s] * gy[i];
          into = fmaf(p[s], gs, into);
          r[s] = exp2_fast(d[i] * A2[s]) * gs;
          const float q = r[s] * hist[i][s];
          gA[s] = fmaf(d[i], q, gA[s]);
          gd = fmaf(A2[s], q, gd);
        }
        gD = fmaf(gy[i], x[i], gD);
        if (here) {
          if (g.gx) gxp[(long long)t * KC] = (T)fmaf(d[i], into, D * gy[i]);
          gdp[(long long)t * KC] = fmaf(gd, kLn2, into * x[i]);
        }
        const float sum = wave_scatter_sum(v, lane);
        const int o = scatter_index<2 * SP>(lane);
        red[wave][i][o] = sum;
      }
    }
    __syncthreads();
    float* out = ws.gbc + (((long long)cb * a.B + b) * a.N + ts) * 2 * SP;
    for (int o = tid; o < n * 2 * SP; o += kThreads) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s += (&red[w][0][0])[o];
      out[o] = s;
    }
    __syncthreads();
  }
  if (!here) return;
  if (g.gx)
    for (int t = max(t0, t2); t < t1; ++t) gxp[(long long)t * KC] = (T)0.f;
  float* ga = ws.ga + ((long long)b * sh.chunks + ch) * (a.S + 1) * KC + j;
#pragma unroll
  for (int s = 0; s < SP; ++s)
    if (s < a.S) ga[(long long)s * KC] = gA[s];
  ga[(long long)a.S * KC] = gD;
}

// gB_t, gC_t from the column blocks' sums.
template <class T>
__global__ __launch_bounds__(256) void sum_bc_kernel(ScanBwdArgs g, const float* __restrict__ gbc, int colblocks,
                                                     int SP) {
  const ScanArgs& a = g.a;
  const long long n = (long long)a.B * a.N * 2 * SP;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const long long row = i / (2 * SP);
  const int j = (int)(i - row * 2 * SP), s = j < SP ? j : j - SP;
  if (s >= a.S) return;
  T* out = static_cast<T*>(j < SP ? g.gB : g.gC);
  if (!out) return;
  const int b = (int)(row / a.N), t = (int)(row - (long long)b * a.N);
  float v = 0.f;
  if (t < scan_length(a.lengths, b, a.N))
    for (int cb = 0; cb < colblocks; ++cb) v += gbc[cb * n + i];
  out[row * a.S + s] = (T)v;
}

// graw from the components' parts of gdelta, and its sums over kBiasTokens
// tokens: block of 64 channels x 4 token slots.
constexpr int kBiasTokens = 64;
template <class T>
__global__ __launch_bounds__(256) void delta_kernel(ScanBwdArgs g, ScanSpace ws, int colblocks) {
  __shared__ float lds[4][64];
  const ScanArgs& a = g.a;
  const int tb = blockIdx.x / colblocks, c = (blockIdx.x - tb * colblocks) * 64 + (threadIdx.x & 63);
  const int slot = threadIdx.x >> 6;
  const long long rows = (long long)a.B * a.N, r0 = (long long)tb * kBiasTokens;
  const long long r1 = min(rows, r0 + kBiasTokens);
  float sum = 0.f;
  if (c < a.C) {
    const float bias = a.bias ? a.bias[c] : 0.f;
    for (long long row = r0 + slot; row < r1; row += 4) {
      const int b = (int)(row / a.N), t = (int)(row - (long long)b * a.N);
      float v = 0.f;
      if (t < scan_length(a.lengths, b, a.N)) {
        const float* p = ws.gd + row * a.K * a.C + c;
        for (int k = 0; k < a.K; ++k) v += p[(long long)k * a.C];
        v /= 1.f + exp2_fast(-kLog2e * (load1<T>(a.delta, row * a.C + c) + bias));
      }
      if (g.gdelta) static_cast<T*>(g.gdelta)[row * a.C + c] = (T)v;
      sum += v;
    }
  }
  lds[slot][threadIdx.x & 63] = sum;
  __syncthreads();
  if (slot == 0 && c < a.C)
    ws.gbp[(long long)tb * a.C + c] = lds[0][threadIdx.x] + lds[1][threadIdx.x] + lds[2][threadIdx.x] + lds[3][threadIdx.x];
}

// out[row, c] = sum over units and components of part[unit][row][k C + c]:
// 16 slices x 64 outputs per block.  The first `rowsA` rows go to outA[c rowsA +
// row], one behind them to outD[c].
constexpr int kSumSlices = 16;
__global__ __launch_bounds__(64 * kSumSlices) void sum_units_kernel(const float* __restrict__ part, long long units,
                                                                    int rows, int rowsA, int K, int C, float* outA,
                                                                    float* outD) {
  __shared__ float lds[kSumSlices][64];
  const int o = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
  const int row = o / C, c = o - row * C;
  float s = 0.f;
  if (row < rows) {
    for (int k = 0; k < K; ++k) {
      const float* p = part + ((long long)row * K + k) * C + c;
      const long long stride = (long long)rows * K * C;
#pragma unroll 8
      for (long long u = slice; u < units; u += kSumSlices) s += p[u * stride];
    }
  }
  lds[slice][threadIdx.x & 63] = s;
  __syncthreads();
  if (slice == 0 && row < rows) {
    float v = 0.f;
    for (int i = 0; i < kSumSlices; ++i) v += lds[i][threadIdx.x];
    if (row < rowsA) {
      if (outA) outA[(long long)c * rowsA + row] = v;
    } else if (outD) {
      outD[c] = v;
    }
  }
}

ScanChunks backward_chunks(int64_t N, int S) {
  ScanChunks s;
  s.chunk = bwd_chunk(S);
  s.chunks = (int)((N + s.chunk - 1) / s.chunk);
  return s;
}

long long bias_blocks(int64_t B, int64_t N) { return (B * N + kBiasTokens - 1) / kBiasTokens; }

ScanSpace backward_space(void* base, int64_t B, int64_t N, int K, int64_t C, int S) {
  ScanSpace w;
  const ScanChunks ch = backward_chunks(N, S);
  const size_t KC = (size_t)K * C, units = (size_t)B * ch.chunks;
  const size_t colblocks = (KC + bwd_threads(S) - 1) / bwd_threads(S);
  w.place(base, &w.bc, (size_t)B * N * 2 * scan_padded(S));
  if (ch.chunks > 1) {
    w.place(base, &w.hs, units * S * KC);
    w.place(base, &w.rs, units * S * KC);
    w.place(base, &w.ds, units * C);
  }
  w.place(base, &w.gbc, colblocks * B * N * 2 * scan_padded(S));
  w.place(base, &w.gd, (size_t)B * N * KC);
  w.place(base, &w.ga, units * (S + 1) * KC);
  w.place(base, &w.gbp, (size_t)bias_blocks(B, N) * C);
  return w;
}

template <class T, int SP>
hipError_t run_backward(const ScanBwdArgs& g, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  const ScanArgs& a = g.a;
  const int KC = a.K * a.C;
  constexpr int kThreads = BwdShape<SP>::kThreads;
  const int colblocks = (KC + kThreads - 1) / kThreads;
  const long long blocks = (long long)colblocks * ch.chunks;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  hipError_t e;
  if (ch.chunks > 1) {
    if ((e = launch_scan_local(a, ch, w, s)) != hipSuccess) return e;
    if ((e = launch_scan_carry(a, ch, nullptr, w.hs, w.ds, false, s)) != hipSuccess) return e;
    hipLaunchKernelGGL((reverse_kernel<T, SP>), dim3((unsigned)(blocks - colblocks), a.B), dim3(kThreads), 0, s, g, ch,
                       w, colblocks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if ((e = launch_scan_carry(a, ch, nullptr, w.rs, w.ds, true, s)) != hipSuccess) return e;
  }
  hipLaunchKernelGGL((scan_bwd_kernel<T, SP>), dim3((unsigned)blocks, a.B), dim3(kThreads), 0, s, g, ch, w, colblocks);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (g.gB || g.gC) {
    const long long n = ((long long)a.B * a.N * 2 * SP + 255) / 256;
    if (n > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(sum_bc_kernel<T>, dim3((unsigned)n), dim3(256), 0, s, g, w.gbc, colblocks, SP);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (g.gdelta || g.gbias) {
    const int cbs = (a.C + 63) / 64;
    const long long tbs = bias_blocks(a.B, a.N);
    if (tbs * cbs > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(delta_kernel<T>, dim3((unsigned)(tbs * cbs)), dim3(256), 0, s, g, w, cbs);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (g.gbias) {
      hipLaunchKernelGGL(sum_units_kernel, dim3(cbs), dim3(64 * kSumSlices), 0, s, w.gbp, tbs, 1, 0, 1, a.C, nullptr,
                         g.gbias);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (g.gA || g.gD) {
    const int outputs = (a.S + 1) * a.C;
    hipLaunchKernelGGL(sum_units_kernel, dim3((outputs + 63) / 64), dim3(64 * kSumSlices), 0, s, w.ga,
                       (long long)a.B * ch.chunks, a.S + 1, a.S, a.K, a.C, g.gA, g.gD);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t by_states(const ScanBwdArgs& g, hipStream_t s) {
  const ScanArgs& a = g.a;
  const ScanChunks ch = backward_chunks(a.N, a.S);
  const ScanSpace w = backward_space(a.ws, a.B, a.N, a.K, a.C, a.S);
  const hipError_t e = launch_scan_prepare(a, w.bc, s);
  if (e != hipSuccess) return e;
  switch (scan_padded(a.S)) {
    case 8: return run_backward<T, 8>(g, ch, w, s);
    case 16: return run_backward<T, 16>(g, ch, w, s);
    default: return run_backward<T, 32>(g, ch, w, s);
  }
}

}  // namespace

size_t scan_backward_bytes(int64_t B, int64_t N, int K, int64_t C, int S) {
  return backward_space(nullptr, B, N, K, C, S).bytes;
}

hipError_t launch_scan_backward(const ScanBwdArgs& g, hipStream_t s) {
  return g.a.type == SEQ_BF16 ? by_states<bf16>(g, s) : by_states<float>(g, s);
}

}  // namespace cgconv
