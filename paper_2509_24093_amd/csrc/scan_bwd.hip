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
// their start states, inside a chunk the states before every kSub tokens in LDS,
// the kSub states of a piece in registers.  What the chunks add to the states
// behind them and to r before them comes from one pass over the tokens: with the
// running product P_t of the decays, sum_t P_t C_t gy_t is the chunk's own r, so
// both take one exponential per state.  gB and gC add over the lanes: the
// eight values of a token that a wave has are halved from step to step, each lane
// keeping the half of its bit, so they take 7 exchanges and 3 more instead of 48; waves add
// through LDS, column blocks in a last kernel.  No atomics: every sum has a fixed
// order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "scan_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

constexpr float kLn2 = 0.69314718055994530942f;

// A thread of the main kernel holds kGroup states of a column; the SP / kGroup
// groups of a column are waves of one block, so B_t and C_t stay scalar and the
// sums over all states go through LDS.  Tokens per chunk and per piece, columns per
// block: the states of a piece take kSub kGroup registers, the pieces' starts
// (chunk / sub - 1) kGroup columns groups 4 bytes of LDS (48 KiB), the sums kSub
// columns groups 8 bytes (16 KiB): two blocks per CU, four waves per SIMD (whose 128
// registers are 2 to 14 too few, spilled).  2 x 4096
// x 1024 bf16, 16 states, forward and backward: all 16 states in a thread, pieces of
// 8, two waves per SIMD 366 us; groups of 8, pieces of 8 413, of 6 360, of 5 357, of 4
// 351, of 3 374; the next piece's inputs asked for a piece ahead, with the other
// loads ahead of their use: 302.
constexpr int kGroup = 8;
template <int SP>
struct BwdShape {
  static constexpr int kGroups = SP / kGroup;
  static constexpr int kSub = 4;
  static constexpr int kChunk = 4 * kSub;
  static constexpr int kColumns = SP == 32 ? 128 : 256;
  static constexpr int kThreads = kColumns * kGroups;
};
constexpr int kBwdChunk = BwdShape<16>::kChunk;  // of all
static_assert(BwdShape<8>::kChunk == kBwdChunk && BwdShape<32>::kChunk == kBwdChunk, "");
int bwd_columns(int S) { return scan_padded(S) == 32 ? BwdShape<32>::kColumns : BwdShape<16>::kColumns; }

// The states that a chunk ends with from zero, the gradient that its own outputs
// send to the state before it, and its sum of delta.
template <class T, int SP>
__global__ __launch_bounds__(256) void ends_kernel(ScanBwdArgs g, ScanChunks sh, ScanSpace ws,
                                                                      int colblocks) {
  const ScanArgs& a = g.a;
  const int ch = blockIdx.x / colblocks, b = blockIdx.y;
  const int KC = a.K * a.C;
  const int id = (blockIdx.x - ch * colblocks) * blockDim.x + threadIdx.x;
  const bool here = id < KC;
  const int j = here ? id : 0, c = j % a.C;
  const int len = scan_length(a.lengths, b, a.N);
  const int t0 = ch * sh.chunk, t2 = min(min(a.N, t0 + sh.chunk), len);
  const long long row0 = (long long)b * a.N;
  const T* xp = static_cast<const T*>(a.x) + row0 * KC + j;
  const T* gyp = static_cast<const T*>(g.gy) + row0 * KC + j;
  const T* dp = static_cast<const T*>(a.delta) + row0 * a.C + c;
  const ConstFloats bc = (ConstFloats)(ws.bc + row0 * 2 * SP);
  constexpr int kAhead = 4;
  const float rows_seen = colblocks <= 2 ? touch_rows<SP>(ws.bc + row0 * 2 * SP, t0, t2) : 0.f;
  T dn[kAhead], xn[kAhead], gn[kAhead];  // as stored: widening them here would wait for them
  auto fetch = [&](int tb) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = min(tb + u, t2 - 1);
      dn[u] = dp[(long long)t * a.C];
      xn[u] = xp[(long long)t * KC];
      gn[u] = gyp[(long long)t * KC];
    }
  };
  TokenRows<SP> rows;
  if (t0 < t2) {
    fetch(t0);
    rows.begin(bc, t0);
  }
  float A2[SP], h[SP], r[SP], P[SP];
#pragma unroll
  for (int s = 0; s < SP; ++s) {
    A2[s] = ws.A2[s * a.C + c];
    h[s] = r[s] = 0.f;
    P[s] = 1.f;
  }
  const float bias = a.bias ? a.bias[c] : 0.f;
  float total = 0.f;
  settle_rows(rows_seen);
  auto token = [&](int t, T draw, T xraw, T graw) {
    const float* p = rows.at(t, min(t + 1, t2 - 1));
    const float d = softplus(widen(draw) + bias), dx = d * widen(xraw), gy = widen(graw);
    total += d;
#pragma unroll
    for (int s = 0; s < SP; ++s) {
      const float e = exp2_fast(d * A2[s]);
      h[s] = fmaf(e, h[s], p[s] * dx);
      P[s] *= e;
      r[s] = fmaf(P[s], p[SP + s] * gy, r[s]);
    }
  };
  int tb = t0;
  for (; tb + kAhead <= t2; tb += kAhead) {  // no conditions inside: the rows change registers without copies
    T dc[kAhead], xc[kAhead], gc[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      dc[u] = dn[u];
      xc[u] = xn[u];
      gc[u] = gn[u];
    }
    fetch(tb + kAhead);  // (the last token again at the end: under a condition it would move behind the loop)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) token(tb + u, dc[u], xc[u], gc[u]);
  }
#pragma unroll
  for (int u = 0; u < kAhead - 1; ++u)
    if (tb + u < t2) token(tb + u, dn[u], xn[u], gn[u]);
  if (!here) return;
  const long long at = ((long long)b * sh.chunks + ch) * a.S * KC + j;
#pragma unroll
  for (int s = 0; s < SP; ++s)
    if (s < a.S) {
      ws.hs[at + (long long)s * KC] = h[s];
      ws.rs[at + (long long)s * KC] = r[s];
    }
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
  halve<0x4E, (N / 16 > 0 ? N / 16 : 1)>(v, lane & 2);   // quad_perm 2, 3, 0, 1
  halve<0xB1, (N / 32 > 0 ? N / 32 : 1)>(v, lane & 1);   // quad_perm 1, 0, 3, 2
  return v[0];
}
// Lane bits 5, 4, 3, ... choose the halves from the largest on; the lowest bits
// of fewer than 64 values hold copies.
template <int N>
__device__ __forceinline__ int scatter_index(int lane) { return lane / (64 / N); }

// Block (chunk, column block) of a batch element: `columns` columns k C + c (whole
// waves) x the groups of states, group slowest.  ONE: K = 1, delta's gradient is
// finished here.
template <class T, int SP, bool ONE>
__global__ __launch_bounds__(BwdShape<SP>::kThreads, 4) void scan_bwd_kernel(ScanBwdArgs g,
                                                                                           ScanChunks sh, ScanSpace ws,
                                                                                           int colblocks, int columns) {
  typedef BwdShape<SP> Shape;
  constexpr int kSub = Shape::kSub, kGroups = Shape::kGroups, kWaves = Shape::kColumns / 64;
  constexpr int kPieces = Shape::kChunk / kSub;
  __shared__ float starts[kPieces - 1][kGroup][Shape::kThreads];
  __shared__ float sums[kGroups > 1 ? kSub : 1][2][kGroups > 1 ? Shape::kThreads : 1];
  __shared__ float red[kGroups][kWaves][kSub][2 * kGroup];
  const ScanArgs& a = g.a;
  const int ch = blockIdx.x / colblocks, cb = blockIdx.x - ch * colblocks, b = blockIdx.y;
  const int KC = a.K * a.C, tid = threadIdx.x, lane = tid & 63;
  const int group = __builtin_amdgcn_readfirstlane(kGroups > 1 ? tid / columns : 0);
  const int column = tid - group * columns, wave = column >> 6;
  const int id = cb * columns + column;
  const bool here = id < KC;
  const int j = here ? id : 0, c = ONE ? j : j % a.C;
  const int s0 = group * kGroup;
  const int len = scan_length(a.lengths, b, a.N);
  const int t0 = ch * sh.chunk, t1 = min(a.N, t0 + sh.chunk), t2 = min(t1, len);
  const long long row0 = (long long)b * a.N;
  const T* xp = static_cast<const T*>(a.x) + row0 * KC + j;
  const T* gyp = static_cast<const T*>(g.gy) + row0 * KC + j;
  const T* dp = static_cast<const T*>(a.delta) + row0 * a.C + c;
  T* gxp = static_cast<T*>(g.gx) + row0 * KC + j;
  T* gdp = static_cast<T*>(g.gdelta) + row0 * KC + j;  // ONE
  float* gdk = ws.gd + row0 * KC + j;                  // else
  const ConstFloats bc = (ConstFloats)(ws.bc + row0 * 2 * SP + s0);
  const long long at = (((long long)b * sh.chunks + ch) * a.S + s0) * KC + j;
  const bool carried = here && sh.chunks > 1;
  float A2[kGroup], r[kGroup], gA[kGroup];
  const float bias = a.bias ? a.bias[c] : 0.f, D = a.D ? a.D[c] : 0.f;
  float gD = 0.f, gbias = 0.f;
  const int last = t2 > t0 ? (t2 - t0 - 1) / kSub : -1;  // the last piece
  const float rows_seen = colblocks <= 2 ? touch_rows<SP>(ws.bc + row0 * 2 * SP, t0, t2) : 0.f;
#pragma unroll
  for (int s = 0; s < kGroup; ++s) A2[s] = ws.A2[(s0 + s) * a.C + c];
  auto start = [&](float (&h)[kGroup]) {
#pragma unroll
    for (int s = 0; s < kGroup; ++s) h[s] = carried && s0 + s < a.S ? ws.hs[at + (long long)s * KC] : 0.f;
  };
  {  // the states before every piece but the first
    float h[kGroup];
    T dn[kSub], xn[kSub];
    auto fetch = [&](int ts) {
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        dn[i] = dp[(long long)min(ts + i, t2 - 1) * a.C];
        xn[i] = xp[(long long)min(ts + i, t2 - 1) * KC];
      }
    };
    if (last > 0) fetch(t0);
    start(h);
    settle_rows(rows_seen);
#pragma unroll 1
    for (int piece = 0; piece < last; ++piece) {
      const int ts = t0 + piece * kSub;
      float d[kSub], x[kSub];
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        d[i] = widen(dn[i]);
        x[i] = here ? widen(xn[i]) : 0.f;
      }
      fetch(ts + kSub);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        const float di = softplus(d[i] + bias), dx = di * x[i];
        const ConstFloats p = bc + (long long)(ts + i) * 2 * SP;
#pragma unroll
        for (int s = 0; s < kGroup; ++s) h[s] = fmaf(exp2_fast(di * A2[s]), h[s], p[s] * dx);
      }
#pragma unroll
      for (int s = 0; s < kGroup; ++s) starts[piece][s][tid] = h[s];
    }
  }
#pragma unroll
  for (int s = 0; s < kGroup; ++s) {
    r[s] = carried && s0 + s < a.S ? ws.rs[at + (long long)s * KC] : 0.f;
    gA[s] = 0.f;
  }
  T dn[kSub], xn[kSub], gn[kSub];  // the next piece's, as stored
  auto fetch = [&](int ts) {
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      const int t = max(min(ts + i, t2 - 1), t0);
      dn[i] = dp[(long long)t * a.C];
      xn[i] = xp[(long long)t * KC];
      gn[i] = gyp[(long long)t * KC];
    }
  };
  if (last >= 0) fetch(t0 + last * kSub);
#pragma unroll 1
  for (int piece = last; piece >= 0; --piece) {
    const int ts = t0 + piece * kSub, n = min(kSub, t2 - ts);
    float hist[kSub][kGroup], d[kSub], x[kSub], gy[kSub];  // hist[i]: before token i
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      const bool on = here && i < n;
      d[i] = widen(dn[i]) + bias;
      x[i] = on ? widen(xn[i]) : 0.f;
      gy[i] = on ? widen(gn[i]) : 0.f;
    }
    fetch(ts - kSub);
    __builtin_amdgcn_sched_barrier(0);
    if (piece) {
#pragma unroll
      for (int s = 0; s < kGroup; ++s) hist[0][s] = starts[piece - 1][s][tid];
    } else {
      start(hist[0]);
    }
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
      if (i < n) {  // uniform
        d[i] = softplus(d[i]);
        const float dx = d[i] * x[i];
        const ConstFloats p = bc + (long long)(ts + i) * 2 * SP;
        float v[kGroup];
#pragma unroll
        for (int s = 0; s < kGroup; ++s) {
          const float h = fmaf(exp2_fast(d[i] * A2[s]), hist[i][s], p[s] * dx);
          v[s] = h * gy[i];
          if (i + 1 < kSub) hist[i + 1][s] = h;
        }
        red[group][wave][i][kGroup + scatter_index<kGroup>(lane)] = wave_scatter_sum(v, lane);
      }
    }
    // gradients that add over the states: of x (from `into`) and of delta
    auto finish = [&](int i, float into, float gd) {
      const long long t = ts + i;
      gd = fmaf(gd, kLn2, into * x[i]);
      if (ONE) {
        gd *= __builtin_amdgcn_rcpf(1.f + exp2_fast(-kLog2e * (widen(dp[t * a.C]) + bias)));  // softplus' derivative, delta read again
        gbias += gd;
      }
      if (!here) return;
      if (g.gx) gxp[t * KC] = (T)fmaf(d[i], into, D * gy[i]);
      if (ONE) {
        if (g.gdelta) gdp[t * KC] = (T)gd;
      } else {
        gdk[t * KC] = gd;
      }
    };
#pragma unroll
    for (int i = kSub - 1; i >= 0; --i) {
      if (i < n) {
        const ConstFloats p = bc + (long long)(ts + i) * 2 * SP;
        const float dx = d[i] * x[i];
        float v[kGroup], into = 0.f, gd = 0.f;
#pragma unroll
        for (int s = 0; s < kGroup; ++s) {
          const float gs = fmaf(p[SP + s], gy[i], r[s]);
          v[s] = gs * dx;
          into = fmaf(p[s], gs, into);
          r[s] = exp2_fast(d[i] * A2[s]) * gs;
          const float q = r[s] * hist[i][s];
          gA[s] = fmaf(d[i], q, gA[s]);
          gd = fmaf(A2[s], q, gd);
        }
        gD = fmaf(gy[i], x[i], gD);
        red[group][wave][i][scatter_index<kGroup>(lane)] = wave_scatter_sum(v, lane);
        if (kGroups > 1) {
          sums[i][0][tid] = into;
          sums[i][1][tid] = gd;
        } else {
          finish(i, into, gd);
        }
      }
    }
    __syncthreads();
    if (kGroups > 1) {  // group g finishes tokens g, g + kGroups, ...
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        if (i < n && i % kGroups == group) {
          float into = 0.f, gd = 0.f;
#pragma unroll
          for (int q = 0; q < kGroups; ++q) {
            into += sums[i][0][q * columns + column];
            gd += sums[i][1][q * columns + column];
          }
          finish(i, into, gd);
        }
      }
    }
    const int waves = columns >> 6;
    float* out = ws.gbc + (((long long)cb * a.B + b) * a.N + ts) * 2 * SP;
    for (int o = tid; o < n * 2 * SP; o += blockDim.x) {
      const int i = o / (2 * SP), s = o % SP;
      const bool isC = o % (2 * SP) >= SP;
      float v = 0.f;
      for (int w = 0; w < waves; ++w) v += red[s / kGroup][w][i][(isC ? kGroup : 0) + s % kGroup];
      out[o] = v;
    }
    __syncthreads();
  }
  if (ONE && kGroups > 1) {  // (the last barrier of the pieces was the last reader's)
    sums[0][0][tid] = gbias;
    __syncthreads();
    gbias = 0.f;
#pragma unroll
    for (int q = 0; q < kGroups; ++q) gbias += sums[0][0][q * columns + column];
  }
  if (!here) return;
  if (group == 0) {
    for (int t = max(t0, t2); t < t1; ++t) {
      if (g.gx) gxp[(long long)t * KC] = (T)0.f;
      if (ONE && g.gdelta) gdp[(long long)t * KC] = (T)0.f;
    }
  }
  float* ga = ws.ga + ((long long)b * sh.chunks + ch) * (a.S + 2) * KC + j;
#pragma unroll
  for (int s = 0; s < kGroup; ++s)
    if (s0 + s < a.S) ga[(long long)(s0 + s) * KC] = gA[s];
  if (group == 0) {
    ga[(long long)a.S * KC] = gD;
    if (ONE) ga[(long long)(a.S + 1) * KC] = gbias;
  }
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

// K > 1: graw from the components' parts of gdelta, and its sums over a block's
// tokens.  A block takes `width` channels (a power of two) x 256 / width token
// slots, kBiasRows tokens a slot.
constexpr int kBiasRows = 4;
template <class T>
__global__ __launch_bounds__(256) void delta_kernel(ScanBwdArgs g, ScanSpace ws, int width, int colblocks) {
  __shared__ float lds[256];
  const ScanArgs& a = g.a;
  const int tb = blockIdx.x / colblocks, lane = threadIdx.x & (width - 1), slot = threadIdx.x / width;
  const int slots = 256 / width, c = (blockIdx.x - tb * colblocks) * width + lane;
  const long long rows = (long long)a.B * a.N, r0 = (long long)tb * slots * kBiasRows;
  float sum = 0.f;
  if (c < a.C) {
    const float bias = a.bias ? a.bias[c] : 0.f;
    for (int i = 0; i < kBiasRows; ++i) {
      const long long row = r0 + i * slots + slot;
      if (row >= rows) break;
      const int b = (int)(row / a.N), t = (int)(row - (long long)b * a.N);
      float v = 0.f;
      if (t < scan_length(a.lengths, b, a.N)) {
        const float* p = ws.gd + row * a.K * a.C + c;
        const float raw = load1<T>(a.delta, row * a.C + c) + bias;
#pragma unroll 8
        for (int k = 0; k < a.K; ++k) v += p[(long long)k * a.C];
        v /= 1.f + exp2_fast(-kLog2e * raw);
      }
      if (g.gdelta) static_cast<T*>(g.gdelta)[row * a.C + c] = (T)v;
      sum += v;
    }
  }
  lds[threadIdx.x] = sum;
  __syncthreads();
  if (slot == 0 && c < a.C) {
    for (int i = 1; i < slots; ++i) sum += lds[i * width + lane];
    ws.gbp[(long long)tb * a.C + c] = sum;
  }
}

// Sums over units and components of part[unit][row][k C + c], rows: 64 slices x
// 16 outputs per block.  Output row < rowsA: outA[c rowsA + row]; the two behind
// them: out1[c], out2[c].
constexpr int kSumSlices = 64, kSumLanes = 16;
__global__ __launch_bounds__(kSumSlices * kSumLanes) void sum_units_kernel(const float* __restrict__ part,
                                                                           long long units, int rows, int rowsA, int K,
                                                                           int C, float* outA, float* out1,
                                                                           float* out2) {
  __shared__ float lds[kSumSlices][kSumLanes];
  const int lane = threadIdx.x & (kSumLanes - 1), slice = threadIdx.x / kSumLanes;
  const int o = blockIdx.x * kSumLanes + lane, row = o / C, c = o - row * C;
  float s = 0.f;
  if (row < rows) {
    const float* p = part + (long long)row * K * C + c;
    const long long stride = (long long)rows * K * C;
    if (K == 1) {
#pragma unroll 8
      for (long long u = slice; u < units; u += kSumSlices) s += p[u * stride];
    } else {
      for (long long u = slice; u < units; u += kSumSlices) {
#pragma unroll 8
        for (int k = 0; k < K; ++k) s += p[u * stride + (long long)k * C];
      }
    }
  }
  lds[slice][lane] = s;
  __syncthreads();
  for (int n = kSumSlices / 2; n > 0; n /= 2) {
    if (slice < n) lds[slice][lane] += lds[slice + n][lane];
    __syncthreads();
  }
  if (slice == 0 && row < rows) {
    const float v = lds[0][lane];
    if (row < rowsA) {
      if (outA) outA[(long long)c * rowsA + row] = v;
    } else {
      float* out = row == rowsA ? out1 : out2;
      if (out) out[c] = v;
    }
  }
}

ScanChunks backward_chunks(int64_t N) {
  ScanChunks s;
  s.chunk = kBwdChunk;
  s.chunks = (int)((N + s.chunk - 1) / s.chunk);
  return s;
}

// Lanes over the channels in delta_kernel, and its blocks over the tokens.
int bias_width(int64_t C) {
  int w = 16;
  while (w < 64 && w < C) w *= 2;
  return w;
}
long long bias_blocks(int64_t B, int64_t N, int64_t C) {
  const int rows = 256 / bias_width(C) * kBiasRows;
  return (B * N + rows - 1) / rows;
}

// Column blocks, of equal numbers of waves.
int bwd_colblocks(int64_t KC, int S) { return (int)((KC + bwd_columns(S) - 1) / bwd_columns(S)); }

ScanSpace backward_space(void* base, int64_t B, int64_t N, int K, int64_t C, int S) {
  ScanSpace w;
  const ScanChunks ch = backward_chunks(N);
  const size_t KC = (size_t)K * C, units = (size_t)B * ch.chunks;
  w.place(base, &w.bc, (size_t)B * N * 2 * scan_padded(S));
  w.place(base, &w.A2, (size_t)scan_padded(S) * C);
  if (ch.chunks > 1) {
    w.place(base, &w.hs, units * S * KC);
    w.place(base, &w.rs, units * S * KC);
    w.place(base, &w.ds, units * C);
  }
  w.place(base, &w.gbc, (size_t)bwd_colblocks(KC, S) * B * N * 2 * scan_padded(S));
  w.place(base, &w.ga, units * (S + 2) * KC);
  if (K > 1) {
    w.place(base, &w.gd, (size_t)B * N * KC);
    w.place(base, &w.gbp, (size_t)bias_blocks(B, N, C) * C);
  }
  return w;
}

hipError_t sum_units(const float* part, long long units, int rows, int rowsA, int K, int C, float* outA, float* out1,
                     float* out2, hipStream_t s) {
  hipLaunchKernelGGL(sum_units_kernel, dim3((rows * C + kSumLanes - 1) / kSumLanes), dim3(kSumSlices * kSumLanes), 0, s,
                     part, units, rows, rowsA, K, C, outA, out1, out2);
  return hipGetLastError();
}

template <class T, int SP>
hipError_t run_backward(const ScanBwdArgs& g, const ScanChunks& ch, const ScanSpace& w, hipStream_t s) {
  const ScanArgs& a = g.a;
  const int KC = a.K * a.C;
  const int colblocks = bwd_colblocks(KC, a.S);
  const int columns = ((KC + colblocks - 1) / colblocks + 63) / 64 * 64;
  const long long blocks = (long long)colblocks * ch.chunks;
  if (!launch_fits(blocks, columns * BwdShape<SP>::kGroups)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks, a.B);
  hipError_t e;
  if (ch.chunks > 1) {
    hipLaunchKernelGGL((ends_kernel<T, SP>), grid, dim3(columns), 0, s, g, ch, w, colblocks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if ((e = launch_scan_carry(a, ch, w, nullptr, true, s)) != hipSuccess) return e;
  }
  const dim3 block(columns * BwdShape<SP>::kGroups);
  if (a.K == 1)
    hipLaunchKernelGGL((scan_bwd_kernel<T, SP, true>), grid, block, 0, s, g, ch, w, colblocks, columns);
  else
    hipLaunchKernelGGL((scan_bwd_kernel<T, SP, false>), grid, block, 0, s, g, ch, w, colblocks, columns);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (g.gB || g.gC) {
    const long long n = ((long long)a.B * a.N * 2 * SP + 255) / 256;
    if (!launch_fits(n, 256)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(sum_bc_kernel<T>, dim3((unsigned)n), dim3(256), 0, s, g, w.gbc, colblocks, SP);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.K > 1 && (g.gdelta || g.gbias)) {
    const int width = bias_width(a.C), cbs = (a.C + width - 1) / width;
    const long long tbs = bias_blocks(a.B, a.N, a.C);
    if (!launch_fits(tbs * cbs, 256)) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(delta_kernel<T>, dim3((unsigned)(tbs * cbs)), dim3(256), 0, s, g, w, width, cbs);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (g.gbias && (e = sum_units(w.gbp, tbs, 1, 0, 1, a.C, nullptr, g.gbias, nullptr, s)) != hipSuccess) return e;
  }
  if (g.gA || g.gD || (a.K == 1 && g.gbias))
    return sum_units(w.ga, (long long)a.B * ch.chunks, a.S + 2, a.S, a.K, a.C, g.gA, g.gD,
                     a.K == 1 ? g.gbias : nullptr, s);
  return hipSuccess;
}

template <class T>
hipError_t by_states(const ScanBwdArgs& g, hipStream_t s) {
  const ScanArgs& a = g.a;
  const ScanChunks ch = backward_chunks(a.N);
  const ScanSpace w = backward_space(a.ws, a.B, a.N, a.K, a.C, a.S);
  const hipError_t e = launch_scan_prepare(a, w, scan_padded(a.S), s);
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
