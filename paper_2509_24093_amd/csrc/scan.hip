// Selective state space scan for gfx950, forward and single tokens (formulas
// and layout: scan_common.h).
//
// A sequence is cut into chunks so that there are enough waves: (1) every chunk
// but the last from a zero state to its end, (2) the chunks' starts one after
// the other, h <- exp(A sum delta) h + end, (3) every chunk from its start,
// writing y.  Where batch and channels give waves enough there is one chunk
// and only (3).  It is bound by the vector units: per state an exponential (a
// quarter of the rate) and its product, and three operations for each of the
// KG components a thread holds.  Four components of 16 states and more take all 256
// registers and 13 to 206 accumulation registers beside them in the output pass: one wave
// per SIMD.
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

// LOCAL: pass (1), else pass (3) from pass (2)'s states (or the caller's, or zero).
template <class T, int KG, int SP, bool LOCAL>
__global__ __launch_bounds__(kScanThreads) void scan_kernel(ScanArgs a, ScanChunks sh, ScanSpace ws, int colblocks) {
  const int ch = blockIdx.x / colblocks, b = blockIdx.y;
  const Column<KG> q((blockIdx.x - ch * colblocks) * blockDim.x + threadIdx.x, a.K, a.C);
  const int len = scan_length(a.lengths, b, a.N);
  const int t0 = ch * sh.chunk, t1 = min(a.N, t0 + sh.chunk), t2 = min(t1, len);
  const long long KC = (long long)a.K * a.C;
  const long long col = (long long)q.k0 * a.C + q.c;
  const long long row0 = (long long)b * a.N;
  const T* xp = static_cast<const T*>(a.x) + row0 * KC + col;
  T* yp = static_cast<T*>(a.y) + row0 * KC + col;
  const T* dp = static_cast<const T*>(a.delta) + row0 * a.C + q.c;
  const ConstFloats bc = (ConstFloats)(ws.bc + row0 * 2 * SP);
  // tokens whose x and delta are loaded while the ones before are computed
  constexpr int kAhead = 4;
  const float rows_seen = colblocks <= 2 ? touch_rows<SP>(ws.bc + row0 * 2 * SP, t0, t2) : 0.f;
  T dn[kAhead], xn[kAhead][KG];  // as stored: widening them here would wait for them
  auto fetch = [&](int tb) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = min(tb + u, t2 - 1);
      dn[u] = dp[(long long)t * a.C];
      // (a component that is not there repeats the last one; it is never stored)
#pragma unroll
      for (int i = 0; i < KG; ++i) xn[u][i] = xp[t * KC + (long long)min(i, q.nk - 1) * a.C];
    }
  };
  TokenRows<SP> rows;
  if (t0 < t2) {
    fetch(t0);
    rows.begin(bc, t0);
  }
  float A2[SP], h[SP][KG];
#pragma unroll
  for (int s = 0; s < SP; ++s) {
    A2[s] = ws.A2[s * a.C + q.c];
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
  float total = 0.f;
  settle_rows(rows_seen);
  auto token = [&](int t, T draw, const T (&xraw)[KG]) {
    const float* p = rows.at(t, min(t + 1, t2 - 1));
    const float d = softplus(widen(draw) + bias);
    if (LOCAL) total += d;
    float dx[KG], y[KG];
#pragma unroll
    for (int i = 0; i < KG; ++i) {
      const float x = widen(xraw[i]);
      dx[i] = d * x;
      y[i] = D * x;
    }
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
  };
  int tb = t0;
  for (; tb + kAhead <= t2; tb += kAhead) {  // no conditions inside: the rows change registers without copies
    T dc[kAhead], xc[kAhead][KG];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      dc[u] = dn[u];
#pragma unroll
      for (int i = 0; i < KG; ++i) xc[u][i] = xn[u][i];
    }
    fetch(tb + kAhead);  // (the last token again at the end: under a condition it would move behind the loop)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) token(tb + u, dc[u], xc[u]);
  }
#pragma unroll
  for (int u = 0; u < kAhead - 1; ++u)
    if (tb + u < t2) token(tb + u, dn[u], xn[u]);
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

// Pass (2): h <- exp(A ds) h + add from chunk to chunk, for 64 states per block;
// each of its SLICES waves first composes its own run of chunks, then starts from
// the runs before it.  A run of at most RUN chunks stays in registers
// between the two, a longer one (not HELD) is read twice.  The arrays hold, in,
// what a chunk adds and, out, what it starts with; y = 1 of the grid goes through
// rs backwards.  The chunk at the far end adds to nobody and need not be formed.
template <int SLICES, int RUN, bool HELD>
__global__ __launch_bounds__(64 * SLICES) void carry_kernel(ScanArgs a, ScanChunks sh, ScanSpace ws,
                                                            const float* first) {
  __shared__ float scale[SLICES][64], shift[SLICES][64];
  const long long KC = (long long)a.K * a.C;
  const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, b = blockIdx.z;
  const bool reverse = blockIdx.y;
  const long long col = (long long)blockIdx.x * 64 + lane;
  const bool here = col < a.S * KC;
  const long long id = here ? col : 0;
  const int s = (int)(id / KC), c = (int)((id - s * KC) % a.C);
  const float A2 = ws.A2[s * a.C + c];
  float* p = (reverse ? ws.rs : ws.hs) + (long long)b * sh.chunks * a.S * KC + id;
  const float* d = ws.ds + (long long)b * sh.chunks * a.C + c;
  const int run = (sh.chunks + SLICES - 1) / SLICES;
  const int n0 = min(slice * run, sh.chunks), n1 = min(n0 + run, sh.chunks);
  float add[RUN], e[RUN];
  auto load = [&](int n) {
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      const int ch = reverse ? sh.chunks - 1 - (n + i) : n + i;
      const bool in = n + i < n1 && n + i < sh.chunks - 1;
      add[i] = in ? p[(long long)ch * a.S * KC] : 0.f;
      e[i] = in ? exp2_fast(A2 * d[(long long)ch * a.C]) : 1.f;
    }
  };
  float E = 1.f, H = 0.f;
  for (int n = n0; n < n1; n += RUN) {
    load(n);
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      H = fmaf(e[i], H, add[i]);
      E *= e[i];
    }
    if (HELD) break;
  }
  scale[slice][lane] = E;
  shift[slice][lane] = H;
  __syncthreads();
  float h = first && !reverse ? first[(long long)b * a.S * KC + id] : 0.f;
  for (int i = 0; i < slice; ++i) h = fmaf(scale[i][lane], h, shift[i][lane]);
  if (!here) return;
  for (int n = n0; n < n1; n += RUN) {
    if (!HELD) load(n);
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      if (n + i < n1) {
        const int ch = reverse ? sh.chunks - 1 - (n + i) : n + i;
        p[(long long)ch * a.S * KC] = h;
        h = fmaf(e[i], h, add[i]);
      }
    }
    if (HELD) break;
  }
}

// B_t and C_t as fp32 rows of 2 SP, then A log2 e as [SP][C]; zeros behind S.
template <class T>
__global__ __launch_bounds__(kScanThreads) void prepare_kernel(ScanArgs a, ScanSpace ws, int SP) {
  const long long i = (long long)blockIdx.x * kScanThreads + threadIdx.x, n = (long long)a.B * a.N * 2 * SP;
  if (i < n) {
    const long long row = i / (2 * SP);
    const int j = (int)(i - row * 2 * SP), s = j < SP ? j : j - SP;
    ws.bc[i] = s < a.S ? load1<T>(j < SP ? a.Bt : a.Ct, row * a.S + s) : 0.f;
  } else if (i < n + (long long)SP * a.C) {
    const int j = (int)(i - n), s = j / a.C, c = j - s * a.C;
    ws.A2[j] = s < a.S ? a.A[(long long)c * a.S + s] * kLog2e : 0.f;
  }
}

// One token: a thread takes V neighbouring channels of one component and four
// states; the 1 .. 8 groups of states of the same channels are lanes of one wave,
// 64 / groups apart, so the loads of a group are neighbours and y is a sum over
// lanes.  Bound by reading and writing the state: 16 states as one loop per thread
// with A read value by value took 12.8 us at 64 x 2048 channels, 7.5 this way.
constexpr int kStepStates = 4;
template <class T, int V>
__global__ __launch_bounds__(kScanThreads) void scan_step_kernel(ScanArgs a, int cols, long long vecs, int groups) {
  const int lanes = 64 / groups, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long id = ((long long)blockIdx.x * (kScanThreads / 64) + wave) * lanes + lane % lanes;
  const bool here = id < vecs;
  const int s0 = lane / lanes * kStepStates;
  const long long at = here ? id : 0, b = at / cols;
  const int e0 = (int)(at - b * cols) * V, c = e0 % a.C;
  const long long KC = (long long)a.K * a.C;
  float x[V], d[V], y[V], h[kStepStates][V], A[V][kStepStates], Bs[kStepStates], Cs[kStepStates];
  float* state = a.state_out + (b * a.S + s0) * KC + e0;
#pragma unroll
  for (int s = 0; s < kStepStates; ++s) {
#pragma unroll
    for (int e = 0; e < V; ++e) h[s][e] = 0.f;
    const bool there = s0 + s < a.S;
    if (there) load_vec(state + s * KC, h[s]);
    Bs[s] = there ? load1<T>(a.Bt, b * a.S + s0 + s) : 0.f;
    Cs[s] = there ? load1<T>(a.Ct, b * a.S + s0 + s) : 0.f;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float* p = a.A + (long long)(c + e) * a.S + s0;
    if (a.S % 4 == 0 && s0 < a.S) {  // whole rows of four, 16-byte aligned
      load_vec(p, A[e]);
    } else {
#pragma unroll
      for (int s = 0; s < kStepStates; ++s) A[e][s] = s0 + s < a.S ? p[s] : 0.f;
    }
  }
  load_vec(static_cast<const T*>(a.x) + b * KC + e0, x);
  load_vec(static_cast<const T*>(a.delta) + b * a.C + c, d);
  float D[V], bias[V];
#pragma unroll
  for (int e = 0; e < V; ++e) D[e] = bias[e] = 0.f;
  if (a.D) load_vec(a.D + c, D);
  if (a.bias) load_vec(a.bias + c, bias);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float step = softplus(d[e] + bias[e]), dx = step * x[e], d2 = step * kLog2e;
    y[e] = 0.f;
#pragma unroll
    for (int s = 0; s < kStepStates; ++s) {
      h[s][e] = fmaf(exp2_fast(d2 * A[e][s]), h[s][e], Bs[s] * dx);
      y[e] = fmaf(Cs[s], h[s][e], y[e]);
    }
    for (int n = lanes; n < 64; n *= 2) y[e] += __shfl_xor(y[e], n);
    y[e] = fmaf(D[e], x[e], y[e]);
  }
  if (!here) return;
#pragma unroll
  for (int s = 0; s < kStepStates; ++s)
    if (s0 + s < a.S) store_vec(state + s * KC, h[s]);
  if (s0 == 0) store_vec(static_cast<T*>(a.y) + b * KC + e0, y);
}

// Waves that keep the vector units busy (4 x 8192 tokens of 2048 channels, bf16, 16
// states: one chunk, 128 waves, 2690 us; in chunks, which form every state twice, 1024
// 779, 2048 529, 4096 473, 8192 443, 16384 442; with lengths from half on 769, 523, 467,
// 390, 358, for twice the chunks' states), and the shortest chunk worth its
// states (S values written and read per chunk and column), shorter in short
// sequences, whose time is that of one chunk (300 tokens of 9 x 16, whole call: 46 -> 31 us).
constexpr long long kWantedWaves = 8192;
int64_t min_chunk(int64_t N) { return std::max<int64_t>(8, std::min<int64_t>(32, N / 16)); }

// Components that share a decay: as few groups as hold four each, and those of one size
// (9 components, three threads of 3 against 4, 4 and 1, forward: 4 x 1999 tokens of 9 x
// 32, fp32, S 16: 54 us against 59; 4 x 8192 of 9 x 128, bf16, S 8, 16, 32: 146, 248 and
// 598 us against 184, 358 and 853).
int components_per_thread(int K) {
  const int groups = (K + 3) / 4;
  return (K + groups - 1) / groups;
}

ScanChunks forward_chunks(int64_t B, int64_t N, int K, int64_t C) {
  const int kg = components_per_thread(K);
  const int64_t waves = B * (((K + kg - 1) / kg * C + 63) / 64);
  int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(kWantedWaves / waves, N / min_chunk(N)));
  ScanChunks s;
  s.chunk = (int)((N + chunks - 1) / chunks);
  s.chunks = (int)((N + s.chunk - 1) / s.chunk);
  return s;
}

// States of the forward's rows and registers, S rounded up (to 4, 8, 12, 16, 24, 32
// against 8, 16, 32: 9 x 4877 tokens of 25 x 29, S 4: 138 -> 96 us; 4 x 8192 of 2048,
// S 12: 437 -> 360; 2 x 4096 of 2048, S 24: 234 -> 194).
int forward_padded(int S) { return S <= 16 ? (S + 3) / 4 * 4 : (S + 7) / 8 * 8; }

ScanSpace forward_space(void* base, const ScanChunks& ch, int64_t B, int64_t N, int K, int64_t C, int S) {
  ScanSpace w;
  w.place(base, &w.bc, (size_t)B * N * 2 * forward_padded(S));
  w.place(base, &w.A2, (size_t)forward_padded(S) * C);
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
  if (!launch_fits(blocks, threads)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((scan_kernel<T, KG, SP, LOCAL>), dim3((unsigned)blocks, a.B), dim3(threads), 0, s, a, ch, w,
                     colblocks);
  return hipGetLastError();
}

template <class T, int KG, bool LOCAL>
hipError_t run_scan_states(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  switch (forward_padded(a.S)) {
    case 4: return run_scan<T, KG, 4, LOCAL>(a, ch, w, s);
    case 8: return run_scan<T, KG, 8, LOCAL>(a, ch, w, s);
    case 12: return run_scan<T, KG, 12, LOCAL>(a, ch, w, s);
    case 16: return run_scan<T, KG, 16, LOCAL>(a, ch, w, s);
    case 24: return run_scan<T, KG, 24, LOCAL>(a, ch, w, s);
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
  hipError_t e = launch_scan_prepare(a, w, forward_padded(a.S), s);
  if (e != hipSuccess) return e;
  if (ch.chunks > 1) {
    if ((e = run_scan_components<T, true>(a, ch, w, s)) != hipSuccess) return e;
    if ((e = launch_scan_carry(a, ch, w, a.state_in, false, s)) != hipSuccess) return e;
  }
  return run_scan_components<T, false>(a, ch, w, s);
}

template <class T, int V>
hipError_t scan_step(const ScanArgs& a, hipStream_t s) {
  const int cols = a.K * a.C / V;
  const long long vecs = (long long)a.B * cols;
  int groups = 1;
  while (groups * kStepStates < a.S) groups *= 2;
  const int per = kScanThreads / groups;  // vectors per block
  const long long blocks = (vecs + per - 1) / per;
  if (!launch_fits(blocks, kScanThreads)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((scan_step_kernel<T, V>), dim3((unsigned)blocks), dim3(kScanThreads), 0, s, a, cols, vecs, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_prepare(const ScanArgs& a, const ScanSpace& w, int SP, hipStream_t s) {
  const long long n = (long long)a.B * a.N * 2 * SP + (long long)SP * a.C;
  const long long blocks = (n + kScanThreads - 1) / kScanThreads;
  if (!launch_fits(blocks, kScanThreads)) return hipErrorInvalidConfiguration;
  if (a.type == SEQ_BF16)
    hipLaunchKernelGGL(prepare_kernel<bf16>, dim3((unsigned)blocks), dim3(kScanThreads), 0, s, a, w, SP);
  else
    hipLaunchKernelGGL(prepare_kernel<float>, dim3((unsigned)blocks), dim3(kScanThreads), 0, s, a, w, SP);
  return hipGetLastError();
}

hipError_t launch_scan_carry(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, const float* first, bool reverse,
                             hipStream_t s) {
  const long long n = (long long)a.S * a.K * a.C;
  const dim3 grid((unsigned)((n + 63) / 64), reverse ? 2 : 1, a.B);
  const auto go = [&](auto kernel, int slices) {
    hipLaunchKernelGGL(kernel, grid, dim3(64 * slices), 0, s, a, ch, w, first);
  };
  // as many slices as leave four chunks to each, or sixteen (16 x 1024 tokens of 2048
  // in 16 chunks, whole scan: sixteen slices 273 us, four 253; two chunks of 24 tokens
  // of 49 x 57, both ways: the carry with sixteen 37 us, with one 7)
  if (ch.chunks <= 4)
    go(carry_kernel<1, 4, true>, 1);
  else if (ch.chunks <= 16)
    go(carry_kernel<4, 4, true>, 4);
  else if (ch.chunks <= 64)
    go(carry_kernel<16, 4, true>, 16);
  else if (ch.chunks <= 256)
    go(carry_kernel<16, 16, true>, 16);
  else
    go(carry_kernel<16, 16, false>, 16);
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
