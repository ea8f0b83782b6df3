// Gated delta rule for gfx950: an associative memory per head, written and read
// by keys that are invariants.  With kn, qn the key and query of norm 1 (or as
// they are), per head with a state S of D x V (V = K P values: P channels of all
// K components):
//
//   S_t = e^{g_t} S_{t-1} + beta_t kn_t (v_t - e^{g_t} S_{t-1}^T kn_t)^T,   y_t = scale S_t^T qn_t
//
// Chunks of 64 tokens, G the sum of the decays within the chunk up to a token:
//
//   A_ij = beta_i e^{G_i - G_j} kn_i.kn_j (i > j)       P_ij = scale e^{G_i - G_j} qn_i.kn_j (i >= j)
//   Y = beta (V - e^G Kn S)                             V' = (1 + A)^-1 Y
//   O = scale e^G Qn S + P V'                           S <- e^{G_end} S + (e^{G_end - G} Kn)^T V'
//
// rule_prepare_kernel forms (1 + A)^-1 of all chunks at once; rule_state_kernel
// walks the chunks.  A wave of it owns 16 columns of S, in registers from the
// first chunk to the last; the columns do not meet, so nothing but the chunk's
// keys, queries and triangles, the same for all waves, goes through LDS.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "rule_common.h"
#include "rule_ws.h"

namespace cgconv {

namespace {

using namespace ruledev;

// A decay below this counts as this: e^-1000 is zero in 32 bits, and differences of
// sums stay numbers where a decay is minus infinity.
constexpr float kLowestDecay = -1000.f;

__device__ __forceinline__ int tokens_of(const RuleArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.n.N) : a.n.N;
}

// ---- the triangles ------------------------------------------------------------------

// Eight elements of a token's row as an operand, and their sum of squares.
template <class T>
__device__ __forceinline__ float operand_row(const T* p, int n, Frag (&f)[kParts<T>]) {
  float x[8], s = 0.f;
  row8(p, n, x);
  parts8<T>(x, f);
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
  return s;
}

// Block (chunk, unit) of four waves; wave w has the tile of rows 16 w.
// Bound by latency: a chunk is 20 products of 16 x 16 and a chain of 15 + 3 steps.
template <class T, int KB, bool TRANSPOSED>
__global__ __launch_bounds__(256) void rule_prepare_kernel(RuleArgs a, RuleWs ws) {
  constexpr int NP = kParts<T>, kRow = kT + 1;
  __shared__ float tri[kT * kRow], inv[kT * kRow];
  __shared__ float rk[kT], rq[kT], beta[kT];
  __shared__ double sum[kT];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, q = lane >> 4;
  const int chunk = blockIdx.x, unit = blockIdx.y, b = unit / a.n.H, h = unit - b * a.n.H;
  const int t0 = chunk * kT, tokens = min(tokens_of(a, b) - t0, kT);
  if (tokens <= 0) return;
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk);
  const long long stride = (long long)a.n.Hk * D;
  const long long row0 = ((long long)b * a.n.N + t0) * stride + (long long)hk * D;
  const T* K = static_cast<const T*>(a.k) + row0;
  const T* Q = static_cast<const T*>(a.q) + row0;
  // the own tile's keys, as columns of the product and for the norms
  Frag own[KB][NP];
  const int t = 16 * wave + m;
  float sk = 0.f, sq = 0.f;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const int d = 32 * kb + 8 * q, n = t < tokens ? max(0, D - d) : 0;
    sk += operand_row(K + t * stride + d, n, own[kb]);
    Frag f[NP];
    sq += operand_row(Q + t * stride + d, n, f);
  }
  if (wave == 0) {
    double g = 0.0;
    float bt = 0.f;
    if (lane < tokens) {
      const long long at = ((long long)b * a.n.N + t0 + lane) * a.n.H + h;
      const float x = a.decay[at];
      g = x < kLowestDecay ? kLowestDecay : x;
      bt = a.beta[at];
    }
    beta[lane] = bt;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const double o = __shfl_up(g, s);
      if (lane >= s) g += o;
    }
    sum[lane] = g;
  }
  sk += __shfl_xor(sk, 16);
  sk += __shfl_xor(sk, 32);
  sq += __shfl_xor(sq, 16);
  sq += __shfl_xor(sq, 32);
  if (q == 0) {
    rk[t] = a.normalize ? 1.f / __builtin_sqrtf(sk + kRuleNormEps) : 1.f;
    rq[t] = a.normalize ? 1.f / __builtin_sqrtf(sq + kRuleNormEps) : 1.f;
  }
  v4f acc[kTiles];
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    acc[j] = v4f{0.f, 0.f, 0.f, 0.f};
    if (j > wave) continue;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int u = 16 * j + m, d = 32 * kb + 8 * q;
      Frag f[NP];
      operand_row(K + u * stride + d, u < tokens ? max(0, D - d) : 0, f);
      acc[j] = mma(f, own[kb], acc[j]);  // rows j, columns of the own tile: a lane has four j of its row
    }
  }
  __syncthreads();
  const double mine = sum[t];
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    if (j > wave) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int u = 16 * j + 4 * q + r;
      tri[t * kRow + u] = t > u ? beta[t] * (rk[t] * rk[u]) * expf((float)(mine - sum[u])) * acc[j][r] : 0.f;
    }
  }
  __syncthreads();
  // diagonal blocks: column m of the inverse, row after row
  {
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float s = r == m ? 1.f : 0.f;
#pragma unroll
      for (int c = 0; c < r; ++c) s = fmaf(-tri[(16 * wave + r) * kRow + 16 * wave + c], x[c], s);
      x[r] = s;
    }
    if (q == 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) inv[(16 * wave + r) * kRow + 16 * wave + m] = x[r];
    }
  }
  __syncthreads();
  // block (i, j) = - inv(i, i) sum_{j <= c < i} A(i, c) inv(c, j), by distance i - j
#pragma unroll
  for (int dist = 1; dist < kTiles; ++dist) {
    if (wave >= dist) {
      const int i = wave, j = wave - dist;
      v4f s{0.f, 0.f, 0.f, 0.f};
      for (int c = j; c < i; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s = __builtin_amdgcn_mfma_f32_16x16x4f32(tri[(16 * i + m) * kRow + 16 * c + 4 * q + e],
                                                   inv[(16 * c + 4 * q + e) * kRow + 16 * j + m], s, 0, 0, 0);
      v4f o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o = __builtin_amdgcn_mfma_f32_16x16x4f32(-inv[(16 * i + m) * kRow + 16 * i + 4 * q + e], s[e], o, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) inv[(16 * i + 4 * q + r) * kRow + 16 * j + m] = o[r];
    }
    __syncthreads();
  }
  const long long at = (long long)unit * ws.chunks + chunk;
  for (int n = wave; n < kBlocks; n += 4) {
    const int i = row_of(n), j = n - block_of(i, 0);
    const float* p = inv + (16 * i + m) * kRow + 16 * j + 4 * q;
    ws.inv[(at * kBlocks + n) * 64 + lane] = make_float4(p[0], p[1], p[2], p[3]);
    if (TRANSPOSED) {
      const float* c = inv + (16 * i + 4 * q) * kRow + 16 * j + m;
      ws.invT[(at * kBlocks + n) * 64 + lane] = make_float4(c[0], c[kRow], c[2 * kRow], c[3 * kRow]);
    }
  }
  if (wave == 0) {
    const double g = sum[lane], end = sum[kT - 1];
    const float hi = (float)g;
    float4* to = ws.token + (at * kT + lane) * 2;
    const float e = expf(hi) * (1.f + (float)(g - hi));
    to[0] = make_float4(beta[lane], rk[lane] * e, rk[lane] * expf((float)(end - g)), a.scale * rq[lane] * e);
    to[1] = make_float4(rk[lane], rq[lane], hi, (float)(g - hi));
    if (lane == 0) {
      const float eh = (float)end;
      ws.whole[at] = expf(eh) * (1.f + (float)(end - eh));
    }
  }
}

// ---- the states, chunk after chunk ------------------------------------------------------

// What a walk over the chunks leaves.
enum Walk {
  kOutputs,  // the outputs, and the last state
  kKeep,     // the state before every chunk and V', for the backward
  kSpan,     // of a segment of the chunks: its last state from zero, and from every unit
             // vector with no values written, which is the segment's matrix
};

// Block (group of 16 NW columns, unit, segment).  The columns of kSpan are the VP of the
// values, then those of the matrix.
template <class T, int KB, int NW, int WALK>
__global__ __launch_bounds__(64 * NW) void rule_state_kernel(RuleArgs a, RuleWs ws) {
  constexpr int NP = kParts<T>, ST = row_stride(KB), DT = 2 * KB, kThreads = 64 * NW;
  constexpr bool kOut = WALK == kOutputs;
  __shared__ __attribute__((aligned(16))) bf16 kbuf[NP][kT * ST];
  __shared__ __attribute__((aligned(16))) bf16 qbuf[kOut ? NP : 1][kOut ? kT * ST : 1];
  __shared__ TriangleParts inv, inside;
  __shared__ float4 ta[kT], tb[kT];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, q = lane >> 4;
  const int unit = blockIdx.y, b = unit / a.n.H, h = unit - b * a.n.H, seg = blockIdx.z;
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk), C = a.n.C, KC = a.n.K * C, N = a.n.N;
  const int first = (blockIdx.x * NW + wave) * 16, col = first + m;
  const bool active = first < (kOut ? ws.V : WALK == kKeep ? ws.VP : ws.VP + 32 * KB);
  const bool matrix = WALK == kSpan && first >= ws.VP;
  const Column column(col, ws.V, C / a.n.H, C, h);
  const int length = tokens_of(a, b);
  const int begin = seg * ws.span, last = min(begin + ws.span, ws.chunks);  // of the segment
  const int end = min((length + kT - 1) / kT, last);
  const int stride = a.n.Hk * D;
  const T* K = static_cast<const T*>(a.k) + (long long)b * N * stride + (long long)hk * D;
  const T* Q = static_cast<const T*>(a.q) + (long long)b * N * stride + (long long)hk * D;
  const T* v = static_cast<const T*>(a.v) + (long long)b * N * KC;
  T* y = static_cast<T*>(a.y) + (kOut ? (long long)b * N * KC : 0);
  const long long start = ((long long)unit * ws.segments + seg) * (32 * KB);  // row of a segment's state

  v4f S[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * d + 4 * q + r;
      float x = 0.f;
      if (WALK == kSpan) {
        x = matrix && row == col - ws.VP ? 1.f : 0.f;
      } else if (seg > 0) {
        if (first < ws.VP) x = ws.start[(start + row) * ws.VP + col];
      } else if (a.state_in && column.there && row < D) {
        x = a.state_in[((long long)b * D + row) * KC + column.at];
      }
      S[d][r] = x;
    }

  RowStage<T, KB, kThreads> sk, sq;
  BlockStage<kThreads> si;
  float4 st;
  ColumnStage<T> sv;
  const auto fetch = [&](int c) {
    const int tokens = min(length - c * kT, kT);
    const long long at = (long long)unit * ws.chunks + c;
    sk.load(K + (long long)c * kT * stride, stride, tokens, D, tid);
    if (kOut) sq.load(Q + (long long)c * kT * stride, stride, tokens, D, tid);
    si.load(ws.inv + at * kBlocks * 64, tid);
    st = ws.token[at * 2 * kT + (tid & (2 * kT - 1))];
  };
  const auto fetch_values = [&](int c) {
    sv.load(v + (long long)c * kT * KC, KC, min(length - c * kT, kT), column, q);
  };
  if (begin < end) {
    fetch(begin);
    fetch_values(begin);
  }
  for (int c = begin; c < end; ++c) {
    const int tokens = min(length - c * kT, kT);
    const long long at = (long long)unit * ws.chunks + c;
    __syncthreads();  // the chunk before has been read
    sk.store(kbuf, tokens, D, tid);
    if constexpr (kOut) sq.store(qbuf, tokens, D, tid);
    si.store(inv, tid);
    if (tid < 2 * kT) (tid & 1 ? tb : ta)[tid >> 1] = st;
    const float whole = ws.whole[at];
    __syncthreads();
    if (c + 1 < end) fetch(c + 1);
    // P, transposed: rows j, columns i, so that a lane has four j of its row
    if constexpr (kOut) {
      for (int n = wave; n < kBlocks; n += NW) {
        const int ib = row_of(n), j = n - block_of(ib, 0);
        v4f p{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          Frag fk[NP], fq[NP];
          rows_frag<NP, ST>(kbuf, j, kb, m, q, fk);
          rows_frag<NP, ST>(qbuf, ib, kb, m, q, fq);
          p = mma(fk, fq, p);
        }
        const int i = 16 * ib + m;
        const float4 me = tb[i];
        const float f = a.scale * me.y;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int u = 16 * j + 4 * q + r;
          const float4 other = tb[u];
          p[r] = i >= u ? p[r] * (f * other.x) * decay_between(me, other) : 0.f;
        }
        put_block(inside, n, lane, p[0], p[1], p[2], p[3]);
      }
    }
    v4f X[kTiles], O[kTiles];
    if (active) {
      if constexpr (WALK == kKeep) store_tiles(ws.state + at * (32 * KB) * ws.VP, ws.VP, col, q, S);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) X[i] = O[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        Frag s[3];
        split_tiles(S[2 * kb], S[2 * kb + 1], s);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          Frag f[NP];
          rows_frag<NP, ST>(kbuf, i, kb, m, q, f);
          X[i] = mma(f, s, X[i]);
          if constexpr (kOut) {
            rows_frag<NP, ST>(qbuf, i, kb, m, q, f);
            O[i] = mma(f, s, O[i]);
          }
        }
      }
      // Y, then V' = (1 + A)^-1 Y
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 t = ta[16 * i + 4 * q + r];
          X[i][r] = t.x * fmaf(-t.y, X[i][r], sv.get(i, r, column));
          O[i][r] *= t.w;
        }
      if (c + 1 < end) fetch_values(c + 1);
      Frag fy[2][3];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) split_tiles(X[2 * kb], X[2 * kb + 1], fy[kb]);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        X[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          if (triangle_has<false>(i, kb)) {
            Frag f[3];
            triangle_frag<false>(inv, i, kb, lane, f);
            X[i] = mma(f, fy[kb], X[i]);
          }
      }
    }
    if constexpr (kOut) __syncthreads();  // P is there
    if (!active) continue;
    if constexpr (WALK == kKeep) store_tiles(ws.value + at * kT * ws.VP, ws.VP, col, q, X);
    if constexpr (kOut) {
      Frag fv[2][3];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) split_tiles(X[2 * kb], X[2 * kb + 1], fv[kb]);
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
          if (triangle_has<false>(i, kb)) {
            Frag f[3];
            triangle_frag<false>(inside, i, kb, lane, f);
            O[i] = mma(f, fv[kb], O[i]);
          }
      store_column(y + (long long)c * kT * KC, KC, N - c * kT, tokens, column, q, O);
    }
    // S <- e^{G_end} S + K^T (e^{G_end - G} rk V')
    Frag fz[2][3];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) X[i][r] *= ta[16 * i + 4 * q + r].z;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) split_tiles(X[2 * kb], X[2 * kb + 1], fz[kb]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
      for (int r = 0; r < 4; ++r) S[d][r] *= whole;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        Frag f[NP];
        columns_frag<NP, ST>(kbuf, d, kb, m, q, f);
        S[d] = mma(f, fz[kb], S[d]);
      }
    }
  }
  if constexpr (WALK == kSpan) {
    if (!active) return;
    if (!matrix) {
      store_tiles(ws.span_state + start * ws.VP, ws.VP, col, q, S);
    } else {
      float* to = ws.span_matrix + (start + col - ws.VP) * (32 * KB) + 4 * q;  // its columns are rows here
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<v4f*>(to + 16 * d) = S[d];
    }
  }
  if constexpr (kOut) {
    if (!column.there) return;
    const long long stop = min((long long)last * kT, (long long)N);
    for (long long t = (long long)max(end, begin) * kT + q; t < stop; t += 4) y[t * KC + column.at] = (T)0.f;
    if (!a.state_out || last != ws.chunks) return;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * d + 4 * q + r;
        if (row < D) a.state_out[((long long)b * D + row) * KC + column.at] = S[d][r];
      }
  }
}

// ---- one token ---------------------------------------------------------------------------

// Block (group of columns, unit): LANES vectors of VC columns side by side, 256 / LANES
// rows of the state at a time, all of a thread's rows in registers, so the state is read
// once and written once (bound by its bytes; of few sequences by the latency of one
// chain load - sum - store).  Both sums over the rows come first:
//   y = scale (e^g qn.S + (qn.kn) u),   u = beta (v - e^g kn.S),   S <- e^g S + kn u.
template <class T, int VC, int LANES>
__global__ __launch_bounds__(256) void rule_step_kernel(RuleArgs a, int V) {
  constexpr int kGroups = 256 / LANES, kRows = kRuleMaxDim / kGroups;
  __shared__ float kn[kRuleMaxDim], qn[kRuleMaxDim], dots[4][3];
  __shared__ float part[4][2][LANES * VC];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int unit = blockIdx.y, b = unit / a.n.H, h = unit - b * a.n.H;
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk), C = a.n.C, KC = a.n.K * C;
  const int j = tid % LANES, g = tid / LANES;
  const Column column((blockIdx.x * LANES + j) * VC, V, C / a.n.H, C, h);
  float* state = a.state_out + (long long)b * D * KC + column.at;
  float s[kRows][VC];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
#pragma unroll
    for (int e = 0; e < VC; ++e) s[i][e] = 0.f;
    if (column.there && g + i * kGroups < D) load_vec(state + (long long)(g + i * kGroups) * KC, s[i]);
  }
  float vv[VC];
#pragma unroll
  for (int e = 0; e < VC; ++e) vv[e] = 0.f;
  if (column.there) load_vec(static_cast<const T*>(a.v) + (long long)b * KC + column.at, vv);
  const long long row = ((long long)b * a.n.Hk + hk) * D;
  float xk = 0.f, xq = 0.f;
  if (tid < D) {
    xk = widen(static_cast<const T*>(a.k)[row + tid]);
    xq = widen(static_cast<const T*>(a.q)[row + tid]);
  }
  if (tid < kRuleMaxDim) {
    kn[tid] = xk;
    qn[tid] = xq;
  }
  const float dk = group_sum(xk * xk, 64), dq = group_sum(xq * xq, 64), dkq = group_sum(xk * xq, 64);
  if (lane == 0) {
    dots[wave][0] = dk;
    dots[wave][1] = dq;
    dots[wave][2] = dkq;
  }
  const float decay = expf(a.decay[unit]), beta = a.beta[unit];
  __syncthreads();
  const float sk = dots[0][0] + dots[1][0], sq = dots[0][1] + dots[1][1], skq = dots[0][2] + dots[1][2];
  const float rk = a.normalize ? 1.f / __builtin_sqrtf(sk + kRuleNormEps) : 1.f;
  const float rq = a.scale * (a.normalize ? 1.f / __builtin_sqrtf(sq + kRuleNormEps) : 1.f);
  float x[VC], w[VC];
#pragma unroll
  for (int e = 0; e < VC; ++e) x[e] = w[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const float fk = kn[g + i * kGroups], fq = qn[g + i * kGroups];
#pragma unroll
    for (int e = 0; e < VC; ++e) {
      x[e] = fmaf(fk, s[i][e], x[e]);
      w[e] = fmaf(fq, s[i][e], w[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < VC; ++e) {
#pragma unroll
    for (int o = LANES; o < 64; o *= 2) {
      x[e] += __shfl_xor(x[e], o);
      w[e] += __shfl_xor(w[e], o);
    }
    if (lane < LANES) {
      part[wave][0][j * VC + e] = x[e];
      part[wave][1][j * VC + e] = w[e];
    }
  }
  __syncthreads();
  if (!column.there) return;
  float u[VC], o[VC];
#pragma unroll
  for (int e = 0; e < VC; ++e) {
    const int at = j * VC + e;
    const float xs = (part[0][0][at] + part[1][0][at]) + (part[2][0][at] + part[3][0][at]);
    const float ws = (part[0][1][at] + part[1][1][at]) + (part[2][1][at] + part[3][1][at]);
    u[e] = beta * fmaf(-decay * rk, xs, vv[e]);
    o[e] = rq * fmaf(decay, ws, rk * skq * u[e]);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (g + i * kGroups >= D) continue;
    const float f = rk * kn[g + i * kGroups];
#pragma unroll
    for (int e = 0; e < VC; ++e) s[i][e] = fmaf(f, u[e], decay * s[i][e]);
    store_vec(state + (long long)(g + i * kGroups) * KC, s[i]);
  }
  if (g == 0) store_vec(static_cast<T*>(a.y) + (long long)b * KC + column.at, o);
}

// f of the key width in tiles of 32
template <class F>
hipError_t by_width(int KB, F f) {
  switch (KB) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    default: return f(std::integral_constant<int, 4>());
  }
}

template <class T>
hipError_t prepare(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s) {
  if (!launch_fits(w.chunks, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid(w.chunks, w.units);
  return by_width(w.KB, [&](auto kb) {
    constexpr int KB = decltype(kb)::value;
    if (backward)
      hipLaunchKernelGGL((rule_prepare_kernel<T, KB, true>), grid, dim3(256), 0, s, a, w);
    else
      hipLaunchKernelGGL((rule_prepare_kernel<T, KB, false>), grid, dim3(256), 0, s, a, w);
    return hipGetLastError();
  });
}

template <class T, int NW, int WALK>
hipError_t walk(const RuleArgs& a, const RuleWs& w, hipStream_t s) {
  const int columns = WALK == kOutputs ? w.V : WALK == kKeep ? w.VP : w.VP + 32 * w.KB;
  const dim3 grid((columns + 16 * NW - 1) / (16 * NW), w.units, w.segments);
  return by_width(w.KB, [&](auto kb) {
    hipLaunchKernelGGL((rule_state_kernel<T, decltype(kb)::value, NW, WALK>), grid, dim3(64 * NW), 0, s, a, w);
    return hipGetLastError();
  });
}

template <class T>
hipError_t states(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (w.segments > 1) {
    e = walk<T, 8, kSpan>(a, w, s);
    if (e == hipSuccess) e = launch_rule_join(a.state_in, w, a.n, false, s);
    if (e != hipSuccess) return e;
  }
  if (w.V <= 64) return backward ? walk<T, 4, kKeep>(a, w, s) : walk<T, 4, kOutputs>(a, w, s);
  return backward ? walk<T, 8, kKeep>(a, w, s) : walk<T, 8, kOutputs>(a, w, s);
}

template <class T>
hipError_t step(const RuleArgs& a, hipStream_t s) {
  const int P = a.n.C / a.n.H, V = a.n.K * P, units = a.n.B * a.n.H;
  const auto run = [&](auto kernel, int columns) {
    hipLaunchKernelGGL(kernel, dim3((V + columns - 1) / columns, units), dim3(256), 0, s, a, V);
    return hipGetLastError();
  };
  if (P % 4 == 0) {
    // 64 columns a block, or 16 where those leave CUs without one
    if ((long long)((V + 63) / 64) * units >= 256) return run(rule_step_kernel<T, 4, 16>, 64);
    return run(rule_step_kernel<T, 4, 4>, 16);
  }
  return run(rule_step_kernel<T, 1, 16>, 16);
}

}  // namespace

size_t rule_workspace_bytes(const RuleSizes& n, bool backward) {
  size_t bytes = 0;
  rule_workspace(n, backward, nullptr, &bytes);
  return bytes;
}

hipError_t launch_rule_prepare(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s) {
  return a.type == SEQ_BF16 ? prepare<bf16>(a, w, backward, s) : prepare<float>(a, w, backward, s);
}

hipError_t launch_rule_states(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s) {
  return a.type == SEQ_BF16 ? states<bf16>(a, w, backward, s) : states<float>(a, w, backward, s);
}

hipError_t launch_rule(const RuleArgs& a, hipStream_t s) {
  const RuleWs w = rule_workspace(a.n, false, a.ws, nullptr);
  const hipError_t e = launch_rule_prepare(a, w, false, s);
  return e == hipSuccess ? launch_rule_states(a, w, false, s) : e;
}

hipError_t launch_rule_step(const RuleArgs& a, hipStream_t s) {
  return a.type == SEQ_BF16 ? step<bf16>(a, s) : step<float>(a, s);
}

}  // namespace cgconv
