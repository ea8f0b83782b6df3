// Selective state space scan for gfx950, forward and single tokens (formulas
// and layout: scan_common.h).
//
// A sequence is cut into chunks so that there are enough waves: (1) every chunk
// but the last from a zero state to its end, (2) the chunks' starts one after
// the other, h <- exp(A sum delta) h + end, (3) every chunk from its start,
// writing y.  Where batch and channels give waves enough there is one chunk
// and only (3).  It is bound by the vector units: per state an exponential (a
// quarter of the rate) and its product, and three operations for each of the
// KG components a thread holds.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "scan_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

// Thread of column id = kg C + c: components kg KG .. of channel c.
template <int KG>
struct Column {
  bool here;
  int c, k0, nk;
  __device__ Column(int id, int K, int C) {
    const int groups = (K + KG - 1) / KG;
    here = id < groups * C;
    if (!here) id = 0;
    const int kg = id / C;
    c = id - kg * C;
    k0 = kg * KG;
    nk = min(KG, K - k0);
  }
};

constexpr int kAhead = 4;  // tokens loaded ahead of their use

// LOCAL: pass (1), else pass (3) from `starts` (or the caller's state, or zero).
template <class T, int KG, int SP, bool LOCAL>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(ScanArgs a, ScanChunks sh, ScanSpace ws, int colblocks) {
  const int ch = blockIdx.x / colblocks, b = blockIdx.y;
  const Column<KG> q((blockIdx.x - ch * colblocks) * blockDim.x + threadIdx.x, a.K, a.C);
  const int len = scan_length(a.lengths, b, a.N);
  const int t0 = ch * sh.chunk, t1 = min(a.N, t0 + sh.chunk), t2 = min(t1, len);
  const long long KC = (long long)a.K * a.C;
  const long long col = (long long)q.k0 * a.C + q.c;
  float A2[SP], h[SP][KG];
#pragma unroll
  for (int s = 0; s < SP; ++s) {
    A2[s] = s < a.S ? a.A[(long long)q.c * a.S + s] * kLog2e : 0.f;
#pragma unroll
    for (int i = 0; i < KG; ++i) h[s][i] = 0.f;
  }
  const float* start = LOCAL ? nullptr
                       : sh.chunks > 1 ? ws.hs + ((long long)b * sh.chunks + ch) * a.S * KC
                       : a.state_in ? a.state_in + (long long)b * a.S * KC : nullptr;
  if (start) {
#pragma unroll
    for (int s = 0; s < SP; ++s)
#pragma unroll
      for (int i = 0; i < KG; ++i)
        if (s < a.S && i < q.nk) h[s][i] = start[s * KC + col + (long long)i * a.C];
  }
  const float bias = a.bias ? a.bias[q.c] : 0.f, D = !LOCAL && a.D ? a.D[q.c] : 0.f;
  const long long row0 = (long long)b * a.N;
  const T* xp = static_cast<const T*>(a.x) + row0 * KC + col;
  T* yp = static_cast<T*>(a.y) + row0 * KC + col;
  const T* dp = static_cast<const T*>(a.delta) + row0 * a.C + q.c;
  const ConstFloats bc = (ConstFloats)(ws.bc + row0 * 2 * SP);
  float total = 0.f;
  for (int tb = t0; tb < t2; tb += kAhead) {
    float dn[kAhead], xn[kAhead][KG];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = min(tb + u, t2 - 1);
      dn[u] = widen(dp[(long long)t * a.C]);
#pragma unroll
      for (int i = 0; i < KG; ++i) xn[u][i] = i < q.nk ? widen(xp[t * KC + (long long)i * a.C]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = tb + u;
      if (t >= t2) break;
      const float d = softplus(dn[u] + bias);
      if (LOCAL) total += d;
      float dx[KG], y[KG];
#pragma unroll
      for (int i = 0; i < KG; ++i) {
        dx[i] = d * xn[u][i];
        y[i] = D * xn[u][i];
      }
      const ConstFloats p = bc + (long long)t * 2 * SP;
#pragma unroll
      for (int s = 0; s < SP; ++s) {
        const float e = exp2_fast(d * A2[s]);
#pragma unroll
        for (int i = 0; i < KG; ++i) {
          h[s][i] = fmaf(e, h[s][i], p[s] * dx[i]);
          if (!LOCAL) y[i] = fmaf(p[SP + s], h[s][i], y[i]);
        }
      }
      if (!LOCAL && q.here) {
#pragma unroll
        for (int i = 0; i < KG; ++i)
          if (i < q.nk) yp[t * KC + (long long)i * a.C] = (T)y[i];
      }
    }
  }
  if (!q.here) return;
  if (!LOCAL) {
    for (int t = max(t0, t2); t < t1; ++t)
      for (int i = 0; i < q.nk; ++i) yp[t * KC + (long long)i * a.C] = (T)0.f;
  }
  // the last chunk with tokens holds the final state; chunks behind it start (and
  // end) with the same one
  float* out = LOCAL ? ws.hs + ((long long)b * sh.chunks + ch) * a.S * KC
               : a.state_out && ch == sh.chunks - 1 ? a.state_out + (long long)b * a.S * KC : nullptr;
  if (out) {
#pragma unroll
    for (int s = 0; s < SP; ++s)
#pragma unroll
      for (int i = 0; i < KG; ++i)
        if (s < a.S && i < q.nk) out[s * KC + col + (long long)i * a.C] = h[s][i];
  }
  if (LOCAL && q.k0 == 0) ws.ds[((long long)b * sh.chunks + ch) * a.C + q.c] = total;
}

// Pass (2): one thread per state, from chunk to chunk (backwards for the
// gradients).  hs: in, what a chunk adds; out, what it starts with.
template <bool REVERSE>
__global__ __launch_bounds__(kScanThreads) void carry_kernel(ScanArgs a, ScanChunks sh, const float* first, float* hs,
                                                             const float* ds) {
  const long long KC = (long long)a.K * a.C;
  const long long id = (long long)blockIdx.x * kScanThreads + threadIdx.x;
  const int b = blockIdx.y;
  if (id >= a.S * KC) return;
  const int s = (int)(id / KC), c = (int)((id - s * KC) % a.C);
  const float A2 = a.A[(long long)c * a.S + s] * kLog2e;
  float h = first ? first[(long long)b * a.S * KC + id] : 0.f;
  float* p = hs + (long long)b * sh.chunks * a.S * KC + id;
  const float* d = ds + (long long)b * sh.chunks * a.C + c;
  constexpr int kBatch = 8;
  for (int n = 0; n < sh.chunks; n += kBatch) {
    float add[kBatch], e[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int ch = REVERSE ? sh.chunks - 1 - (n + i) : n + i;
      // the chunk at the far end adds to nobody and was not formed
      const bool last = n + i >= sh.chunks - 1;
      add[i] = last ? 0.f : p[ch * a.S * KC];
      e[i] = last ? 1.f : exp2_fast(A2 * d[(long long)ch * a.C]);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (n + i >= sh.chunks) break;
      const int ch = REVERSE ? sh.chunks - 1 - (n + i) : n + i;
      p[ch * a.S * KC] = h;
      h = fmaf(e[i], h, add[i]);
    }
  }
}

// B_t and C_t as fp32 rows of 2 SP, zeros behind S.
template <class T>
__global__ __launch_bounds__(kScanThreads) void prepare_kernel(const T* __restrict__ Bt, const T* __restrict__ Ct,
                                                               float* __restrict__ bc, long long rows, int S, int SP) {
  const long long i = (long long)blockIdx.x * kScanThreads + threadIdx.x;
  if (i >= rows * 2 * SP) return;
  const long long row = i / (2 * SP);
  const int j = (int)(i - row * 2 * SP), s = j < SP ? j : j - SP;
  bc[i] = s < S ? widen((j < SP ? Bt : Ct)[row * S + s]) : 0.f;
}

// One token: thread of V neighbouring channels of one component, the states
// streamed through.
template <class T, int V>
__global__ __launch_bounds__(kScanThreads) void scan_step_kernel(ScanArgs a, int cols, long long threads) {
  const long long id = (long long)blockIdx.x * kScanThreads + threadIdx.x;
  if (id >= threads) return;
  const long long b = id / cols;
  const int e0 = (int)(id - b * cols) * V, c = e0 % a.C;
  const long long KC = (long long)a.K * a.C;
  float x[V], d[V], y[V], dx[V];
  load_vec(static_cast<const T*>(a.x) + b * KC + e0, x);
  load_vec(static_cast<const T*>(a.delta) + b * a.C + c, d);
  float D[V], bias[V];
#pragma unroll
  for (int e = 0; e < V; ++e) D[e] = bias[e] = 0.f;
  if (a.D) load_vec(a.D + c, D);
  if (a.bias) load_vec(a.bias + c, bias);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    d[e] = softplus(d[e] + bias[e]);
    dx[e] = d[e] * x[e];
    y[e] = D[e] * x[e];
    d[e] *= kLog2e;
  }
  float* h = a.state_out + b * a.S * KC + e0;
#pragma unroll 4
  for (int s = 0; s < a.S; ++s) {
    const float Bs = load1<T>(a.Bt, b * a.S + s), Cs = load1<T>(a.Ct, b * a.S + s);
    float v[V];
    load_vec(h + s * KC, v);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[e] = fmaf(exp2_fast(d[e] * a.A[(long long)(c + e) * a.S + s]), v[e], Bs * dx[e]);
      y[e] = fmaf(Cs, v[e], y[e]);
    }
    store_vec(h + s * KC, v);
  }
  store_vec(static_cast<T*>(a.y) + b * KC + e0, y);
}

// Waves that keep the vector units busy, and the shortest chunk worth its
// state (S values written and read per chunk and column).
constexpr long long kWantedWaves = 4096;
constexpr int kMinChunk = 32;

int components_per_thread(int K) { return K == 1 ? 1 : K == 9 ? 3 : 4; }

ScanChunks forward_chunks(int64_t B, int64_t N, int K, int64_t C) {
  const int kg = components_per_thread(K);
  const int64_t waves = B * (((K + kg - 1) / kg * C + 63) / 64);
  int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(kWantedWaves / waves, N / kMinChunk));
  ScanChunks s;
  s.chunk = (int)((N + chunks - 1) / chunks);
  s.chunks = (int)((N + s.chunk - 1) / s.chunk);
  return s;
}

ScanSpace forward_space(void* base, const ScanChunks& ch, int64_t B, int64_t N, int K, int64_t C, int S) {
  ScanSpace w;
  w.place(base, &w.bc, (size_t)B * N * 2 * scan_padded(S));
  if (ch.chunks > 1) {
    w.place(base, &w.hs, (size_t)B * ch.chunks * S * K * C);
    w.place(base, &w.ds, (size_t)B * ch.chunks * C);
  }
  return w;
}

template <class T, int KG, int SP, bool LOCAL>
hipError_t run_scan(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  const int ids = (a.K + KG - 1) / KG * a.C;
  const int threads = ids <= 64 ? 64 : ids <= 128 ? 128 : kScanThreads;
  const int colblocks = (ids + threads - 1) / threads;
  const long long blocks = (long long)colblocks * (LOCAL ? ch.chunks - 1 : ch.chunks);
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((scan_kernel<T, KG, SP, LOCAL>), dim3((unsigned)blocks, a.B), dim3(threads), 0, s, a, ch, w,
                     colblocks);
  return hipGetLastError();
}

template <class T, int KG, bool LOCAL>
hipError_t run_scan_states(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  switch (scan_padded(a.S)) {
    case 8: return run_scan<T, KG, 8, LOCAL>(a, ch, w, s);
    case 16: return run_scan<T, KG, 16, LOCAL>(a, ch, w, s);
    default: return run_scan<T, KG, 32, LOCAL>(a, ch, w, s);
  }
}

template <class T, bool LOCAL>
hipError_t run_scan_components(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  switch (components_per_thread(a.K)) {
    case 1: return run_scan_states<T, 1, LOCAL>(a, ch, w, s);
    case 3: return run_scan_states<T, 3, LOCAL>(a, ch, w, s);
    default: return run_scan_states<T, 4, LOCAL>(a, ch, w, s);
  }
}

template <class T>
hipError_t scan_forward(const ScanArgs& a, hipStream_t s) {
  const ScanChunks ch = forward_chunks(a.B, a.N, a.K, a.C);
  const ScanSpace w = forward_space(a.ws, ch, a.B, a.N, a.K, a.C, a.S);
  hipError_t e = launch_scan_prepare(a, w.bc, s);
  if (e != hipSuccess) return e;
  if (ch.chunks > 1) {
    if ((e = run_scan_components<T, true>(a, ch, w, s)) != hipSuccess) return e;
    if ((e = launch_scan_carry(a, ch, a.state_in, w.hs, w.ds, false, s)) != hipSuccess) return e;
  }
  return run_scan_components<T, false>(a, ch, w, s);
}

template <class T, int V>
hipError_t scan_step(const ScanArgs& a, hipStream_t s) {
  const int cols = a.K * a.C / V;
  const long long threads = (long long)a.B * cols;
  hipLaunchKernelGGL((scan_step_kernel<T, V>), dim3((unsigned)((threads + kScanThreads - 1) / kScanThreads)),
                     dim3(kScanThreads), 0, s, a, cols, threads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_prepare(const ScanArgs& a, float* bc, hipStream_t s) {
  const int SP = scan_padded(a.S);
  const long long rows = (long long)a.B * a.N, blocks = (rows * 2 * SP + kScanThreads - 1) / kScanThreads;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  if (a.type == SEQ_BF16)
    hipLaunchKernelGGL(prepare_kernel<bf16>, dim3((unsigned)blocks), dim3(kScanThreads), 0, s,
                       static_cast<const bf16*>(a.Bt), static_cast<const bf16*>(a.Ct), bc, rows, a.S, SP);
  else
    hipLaunchKernelGGL(prepare_kernel<float>, dim3((unsigned)blocks), dim3(kScanThreads), 0, s,
                       static_cast<const float*>(a.Bt), static_cast<const float*>(a.Ct), bc, rows, a.S, SP);
  return hipGetLastError();
}

hipError_t launch_scan_local(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  return a.type == SEQ_BF16 ? run_scan_components<bf16, true>(a, ch, w, s)
                            : run_scan_components<float, true>(a, ch, w, s);
}

hipError_t launch_scan_carry(const ScanArgs& a, const ScanChunks& ch, const float* first, float* hs, const float* ds,
                             bool reverse, hipStream_t s) {
  const long long n = (long long)a.S * a.K * a.C;
  const dim3 grid((unsigned)((n + kScanThreads - 1) / kScanThreads), a.B);
  if (reverse)
    hipLaunchKernelGGL(carry_kernel<true>, grid, dim3(kScanThreads), 0, s, a, ch, first, hs, ds);
  else
    hipLaunchKernelGGL(carry_kernel<false>, grid, dim3(kScanThreads), 0, s, a, ch, first, hs, ds);
  return hipGetLastError();
}

hipError_t launch_scan(const ScanArgs& a, hipStream_t s) {
  return a.type == SEQ_BF16 ? scan_forward<bf16>(a, s) : scan_forward<float>(a, s);
}

hipError_t launch_scan_step(const ScanArgs& a, hipStream_t s) {
  const int v = std::min(4, seq_vec(SEQ_F32, a.C));
  if (a.type == SEQ_BF16) {
    switch (v) {
      case 4: return scan_step<bf16, 4>(a, s);
      case 2: return scan_step<bf16, 2>(a, s);
      default: return scan_step<bf16, 1>(a, s);
    }
  }
  switch (v) {
    case 4: return scan_step<float, 4>(a, s);
    case 2: return scan_step<float, 2>(a, s);
    default: return scan_step<float, 1>(a, s);
  }
}

size_t scan_workspace_bytes(int64_t B, int64_t N, int K, int64_t C, int S) {
  return std::max(scan_forward_bytes(B, N, K, C, S), scan_backward_bytes(B, N, K, C, S));
}

size_t scan_forward_bytes(int64_t B, int64_t N, int K, int64_t C, int S) {
  return forward_space(nullptr, forward_chunks(B, N, K, C), B, N, K, C, S).bytes;
}

}  // namespace cgconv
