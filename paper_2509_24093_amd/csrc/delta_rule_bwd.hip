// Backward of the gated delta rule (see delta_rule.hip for the forward's names).
// With gO, gS the gradients of a chunk's outputs and of the state behind it, and per
// token a = rk e^G, z = rk e^(G_end - G), o = scale rq e^G:
//
//   gV' = P^T gO + z K gS           gY = (1 + A)^-T gV'           gv = beta gY
//   gS <- e^{G_end} gS + Q^T (o gO) - K^T (a gv)
//
// rule_reverse_kernel walks these from the last chunk to the first, a wave per 16
// columns as in the forward, and leaves gS and gY of every chunk.  The states and V'
// come from the forward's walk, repeated.  What is left does not depend on the order
// of the chunks, and rule_grads_kernel does it for all of them at once.  With
//
//   M1_ij = scale e^{G_i - G_j} rq_i rk_j gO_i.V'_j (i >= j)
//   M2_ij = - e^{G_i - G_j} rk_i rk_j gY_i.V'_j (i > j)
//   Uq_i = o_i S gO_i + sum_j M1_ij k_j             (rq times the gradient of qn)
//   UL_i = - a_i S gY_i + sum_j M2_ij k_j           (rk times that of kn where A and Y read it, over beta)
//   UR_j = z_j gS V'_j + sum_i beta_i M2_ij k_i + sum_i M1_ij q_i     (where S and P read it)
//   gbeta_i = k_i.UL_i + gY_i.v_i
//   gdecay_t = e^{G_end} <S, gS> + sum_{i >= t} (o_i q_i.S gO_i - beta_i a_i k_i.S gY_i)
//              + sum_{j < t} z_j k_j.gS V'_j + sum_{i >= t > j} (M1_ij q_i.k_j + beta_i M2_ij k_i.k_j)
//     (what a decay stands between; the sum of the gradients of G from the token on is the
//     same, but its terms cancel where decays are small)
//   gk_i = U - rk^2 k_i (k_i.U) with U the sum of beta UL + UR over the heads that share the
//   key; gq alike.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "rule_common.h"
#include "rule_ws.h"

namespace cgconv {

namespace {

using namespace ruledev;

__device__ __forceinline__ int tokens_of(const RuleArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.n.N) : a.n.N;
}

// Block (group of 16 NW columns, unit, segment).  SPAN: only what the segment adds to the
// state's gradient.
template <class T, int KB, int NW, bool SPAN>
__global__ __launch_bounds__(64 * NW) void rule_reverse_kernel(RuleBwdArgs g, RuleWs ws) {
  constexpr int NP = kParts<T>, DT = 2 * KB, kThreads = 64 * NW;
  typedef Stage<T, KB, true, true> Buffer;  // the transposed triangles
  constexpr int ST = Buffer::ST;
  __shared__ Buffer buffers[Buffer::kCount];
  const RuleArgs& a = g.a;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, q = lane >> 4;
  const int unit = blockIdx.y, b = unit / a.n.H, h = unit - b * a.n.H, seg = blockIdx.z;
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk), C = a.n.C, KC = a.n.K * C, N = a.n.N;
  const int col = (blockIdx.x * NW + wave) * 16 + m;
  const bool active = (blockIdx.x * NW + wave) * 16 < ws.VP;
  const Column column(col, ws.V, C / a.n.H, C, h);
  const int length = tokens_of(a, b);
  const int begin = seg * ws.span, last = min(begin + ws.span, ws.chunks);  // of the segment
  const int end = min((length + kT - 1) / kT, last);
  const long long start = ((long long)unit * ws.segments + seg) * (32 * KB);  // row of a segment's state
  const int stride = a.n.Hk * D;
  const T* K = static_cast<const T*>(a.k) + (long long)b * N * stride + (long long)hk * D;
  const T* Q = static_cast<const T*>(a.q) + (long long)b * N * stride + (long long)hk * D;
  const T* gy = static_cast<const T*>(g.gy) + (long long)b * N * KC;
  T* gv = g.gv ? static_cast<T*>(g.gv) + (long long)b * N * KC : nullptr;

  v4f S[DT];  // gS
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * d + 4 * q + r;
      float x = 0.f;
      if (SPAN) {
      } else if (ws.segments > 1) {
        if (active) x = ws.start[(start + row) * ws.VP + col];
      } else if (g.gstate && column.there && row < D) {
        x = g.gstate[((long long)b * D + row) * KC + column.at];
      }
      S[d][r] = x;
    }

  RowStage<T, KB, kThreads> sk, sq;
  BlockStage<kThreads> si, sp;
  float4 st;
  ColumnStage<T> so;
  const auto fetch = [&](int c) {
    const int tokens = min(length - c * kT, kT);
    const long long at = (long long)unit * ws.chunks + c;
    sk.load(K + (long long)c * kT * stride, stride, tokens, D, tid);
    sq.load(Q + (long long)c * kT * stride, stride, tokens, D, tid);
    si.load(ws.invT + at * kBlocks * 64, tid);
    sp.load(ws.inside + at * kBlocks * 64, tid);
    st = ws.token[(at * kT + (tid & (kT - 1))) * 2];
  };
  const auto put = [&](int c, Buffer& to) {
    const int tokens = min(length - c * kT, kT);
    sk.store(to.k, tokens, D, tid);
    sq.store(to.q, tokens, D, tid);
    si.store(to.inv, tid);
    sp.store(to.inside, tid);
    if (tid < kT) to.token[tid] = st;
  };
  if (begin < end) {
    fetch(end - 1);
    so.load(gy + (long long)(end - 1) * kT * KC, KC, min(length - (end - 1) * kT, kT), column, q);
    if (Buffer::kCount == 2) {
      put(end - 1, buffers[0]);
      if (end - 2 >= begin) fetch(end - 2);
    }
  }
  for (int c = end - 1; c >= begin; --c) {
    const int tokens = min(length - c * kT, kT);
    const long long at = (long long)unit * ws.chunks + c;
    Buffer& buf = buffers[(end - 1 - c) & (Buffer::kCount - 1)];
    const float whole = ws.whole[at];
    __syncthreads();  // the chunk is there; the one before has been read
    if (Buffer::kCount == 1) {
      put(c, buf);
      __syncthreads();
      if (c > begin) fetch(c - 1);
    }
    const auto& kbuf = buf.k;
    const auto& qbuf = buf.q;
    const auto& inv = buf.inv;
    const auto& inside = buf.inside;
    const float4* ta = buf.token;
    v4f X[kTiles];
    if (active) {
      if (!SPAN) store_tiles(ws.gstate + at * (32 * KB) * ws.VP, ws.VP, col, q, S);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) X[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        Frag s[3];
        split_tiles(S[2 * kb], S[2 * kb + 1], s);
        Frag f[kTiles][NP];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) rows_frag<NP, ST>(kbuf, i, kb, m, q, f[i]);
        mma_all(f, s, X);
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) X[i][r] *= ta[16 * i + 4 * q + r].z;
    }
    if (Buffer::kCount == 2 && c > begin) {
      put(c - 1, buffers[(end - c) & 1]);
      if (c - 1 > begin) fetch(c - 2);
    }
    if (!active) continue;
    // gV', gY
    Frag fo[2][NP];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = so.get(2 * kb + e / 4, e % 4, column);
      parts8<T>(x, fo[kb]);
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) mma_triangle<true>(inside, kb, lane, fo[kb], X);
    Frag fx[2][3];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) split_tiles(X[2 * kb], X[2 * kb + 1], fx[kb]);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) X[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) mma_triangle<true>(inv, kb, lane, fx[kb], X);
    if (!SPAN) store_tiles(ws.gvalue + at * kT * ws.VP, ws.VP, col, q, X);
    // gS <- e^{G_end} gS + Q^T (o gO) - K^T (a gv)
    v4f o[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float4 tok = ta[16 * i + 4 * q + r];
        X[i][r] *= tok.x;
        o[i][r] = tok.w * so.get(i, r, column);
      }
    if (!SPAN && gv) store_column(gv + (long long)c * kT * KC, KC, N - c * kT, tokens, column, q, X);
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) X[i][r] *= -ta[16 * i + 4 * q + r].y;
    if (c > begin) so.load(gy + (long long)(c - 1) * kT * KC, KC, kT, column, q);
    Frag fz[2][3];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      split_tiles(X[2 * kb], X[2 * kb + 1], fx[kb]);
      split_tiles(o[2 * kb], o[2 * kb + 1], fz[kb]);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[d][r] *= whole;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      Frag f[DT][NP];
#pragma unroll
      for (int d = 0; d < DT; ++d) columns_frag<NP, ST>(kbuf, d, kb, m, q, f[d]);
      mma_all(f, fx[kb], S);
#pragma unroll
      for (int d = 0; d < DT; ++d) columns_frag<NP, ST>(qbuf, d, kb, m, q, f[d]);
      mma_all(f, fz[kb], S);
    }
  }
  if constexpr (SPAN) {
    if (active) store_tiles(ws.span_state + start * ws.VP, ws.VP, col, q, S);
    return;
  }
  if (!column.there) return;
  if (gv) {
    const long long stop = min((long long)last * kT, (long long)N);
    for (long long t = (long long)max(end, begin) * kT + q; t < stop; t += 4) gv[t * KC + column.at] = (T)0.f;
  }
  if (!g.gstate_in || seg > 0) return;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * d + 4 * q + r;
      if (row < D) g.gstate_in[((long long)b * D + row) * KC + column.at] = S[d][r];
    }
}

// ---- gradients of keys, queries, decays and betas -------------------------------------------

// Eight fp32 values of a row as an operand.
__device__ __forceinline__ void wide_frag(const float* p, Frag (&f)[3]) {
  float x[8];
  load_vec(p, x);
  split8(x, f);
}

// Eight columns from col on of a chunk's token (row: its first token), zeros where there is
// no column or no token.  Where eight columns of a head are neighbours in memory (P a
// multiple of eight) they are one load; what is not there is read from a place that is.
template <class T>
__device__ __forceinline__ void columns8(const T* row, int t, int tokens, int stride, int col, int V, int P, int C,
                                         int h, float (&x)[8]) {
  const T* from = row + (long long)min(t, tokens - 1) * stride;
  if (P % 8 == 0) {
    const Column c(col, V, P, C, h);
    load_vec(from + c.at, x);
    const bool there = c.there && t < tokens;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = there ? x[e] : 0.f;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const Column c(col + e, V, P, C, h);
    const float y = widen(from[c.at]);
    x[e] = c.there && t < tokens ? y : 0.f;
  }
}

constexpr int kMStride = kT + 8;  // as row_stride
typedef bf16 Square[3][kT * kMStride];  // a 64 x 64 matrix in three parts

// A tile's accumulator (column m, rows 4 q + r) into the matrix.
__device__ __forceinline__ void put_tile(Square& s, int i, int j, int m, int q, const v4f& v) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int at = (16 * i + 4 * q + r) * kMStride + 16 * j + m;
    float x = v[r];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      const uint16_t bits = (uint16_t)(__float_as_uint(x) >> 16);
      __builtin_memcpy(&s[p][at], &bits, 2);
      x = without_top(x);
    }
  }
}

// Block (chunk, sequence and key head), the heads that share the key one after the other.
// Wave w owns the tiles w, w + 4 of 16 key components (rows of S and gS) for all tokens, and
// of the 64 x 64 matrices the tiles of row w.
template <class T, int KB>
__global__ __launch_bounds__(256) void rule_grads_kernel(RuleBwdArgs g, RuleWs ws) {
  constexpr int NP = kParts<T>, ST = row_stride(KB), DT = 2 * KB, NT = (DT + 3) / 4;
  __shared__ __attribute__((aligned(16))) bf16 kbuf[NP][kT * ST];
  __shared__ __attribute__((aligned(16))) bf16 qbuf[NP][kT * ST];
  __shared__ __attribute__((aligned(16))) Square mat;
  __shared__ float4 ta[kT], tb[kT];
  __shared__ float dots[3][4][kT], behind[4][kT], direct[kT], dleft[kT], whole_dot[4];
  const RuleArgs& a = g.a;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, q = lane >> 4;
  const int chunk = blockIdx.x, b = blockIdx.y / a.n.Hk, hk = blockIdx.y - b * a.n.Hk;
  const int each = a.n.H / a.n.Hk, P = a.n.C / a.n.H;
  const int D = a.n.D, C = a.n.C, KC = a.n.K * C, N = a.n.N;
  const int t0 = chunk * kT, tokens = max(0, min(tokens_of(a, b) - t0, kT)), here = min(N - t0, kT);
  const int stride = a.n.Hk * D;
  const long long key0 = ((long long)b * N + t0) * stride + (long long)hk * D;
  T* gq = g.gq ? static_cast<T*>(g.gq) + key0 : nullptr;
  T* gk = g.gk ? static_cast<T*>(g.gk) + key0 : nullptr;
  const auto gate_at = [&](int t, int h) { return ((long long)b * N + t0 + t) * a.n.H + h; };
  if (tokens == 0) {
    for (int i = tid; i < here * D; i += 256) {
      const int at = (i / D) * stride + i % D;
      if (gq) gq[at] = (T)0.f;
      if (gk) gk[at] = (T)0.f;
    }
    for (int i = tid; i < here * each; i += 256) {
      const long long at = gate_at(i / each, hk * each + i % each);
      if (g.gdecay) g.gdecay[at] = 0.f;
      if (g.gbeta) g.gbeta[at] = 0.f;
    }
    return;
  }
  {
    RowStage<T, KB, 256> s;
    s.load(static_cast<const T*>(a.k) + key0, stride, tokens, D, tid);
    s.store(kbuf, tokens, D, tid);
    s.load(static_cast<const T*>(a.q) + key0, stride, tokens, D, tid);
    s.store(qbuf, tokens, D, tid);
  }
  for (int i = tid; i < 3 * kT * kMStride / 2; i += 256) reinterpret_cast<uint32_t*>(&mat)[i] = 0;  // above the diagonal
  // an element of the keys or queries as stored
  const auto element = [&](const bf16 (&buf)[NP][kT * ST], int t, int d) {
    float x = 0.f;
#pragma unroll
    for (int p = NP - 1; p >= 0; --p) x += (float)buf[p][t * ST + d];
    return x;
  };
  v4f totq[kTiles][NT], totk[kTiles][NT];
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n) totq[i][n] = totk[i][n] = v4f{0.f, 0.f, 0.f, 0.f};

  for (int e = 0; e < each; ++e) {
    const int h = hk * each + e, unit = b * a.n.H + h;
    const long long at = (long long)unit * ws.chunks + chunk;
    const float* S = ws.state + at * (32 * KB) * ws.VP;
    const float* gS = ws.gstate + at * (32 * KB) * ws.VP;
    const float* val = ws.value + at * kT * ws.VP;
    const float* gval = ws.gvalue + at * kT * ws.VP;
    const T* gy = static_cast<const T*>(g.gy) + ((long long)b * N + t0) * KC;
    const T* v = static_cast<const T*>(a.v) + ((long long)b * N + t0) * KC;
    const float whole = ws.whole[at];
    __syncthreads();  // the head before has been read
    if (tid < 2 * kT) (tid & 1 ? tb : ta)[tid >> 1] = ws.token[at * 2 * kT + tid];

    // S gO, S gY, gS V' over the columns, and <S, gS>
    v4f aq[kTiles][NT], al[kTiles][NT], ar[kTiles][NT];
    float both = 0.f;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) aq[i][n] = al[i][n] = ar[i][n] = v4f{0.f, 0.f, 0.f, 0.f};
    if (wave < DT) {
      for (int v0 = 8 * q; v0 < ws.VP; v0 += 32) {
        Frag fs[NT][3], fg[NT][3];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (wave + 4 * n >= DT) continue;
          float x[8], y[8];
          const long long row = (long long)(16 * (wave + 4 * n) + m) * ws.VP + v0;
          load_vec(S + row, x);
          load_vec(gS + row, y);
#pragma unroll
          for (int c = 0; c < 8; ++c) both = fmaf(x[c], y[c], both);
          split8(x, fs[n]);
          split8(y, fg[n]);
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          const int t = 16 * i + m;
          float x[8];
          Frag fo[NP], fy[3], fv[3];
          columns8(gy, t, tokens, KC, v0, ws.V, P, C, h, x);
          parts8<T>(x, fo);
          wide_frag(gval + (long long)t * ws.VP + v0, fy);
          wide_frag(val + (long long)t * ws.VP + v0, fv);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if (wave + 4 * n >= DT) continue;
            aq[i][n] = mma(fo, fs[n], aq[i][n]);
            al[i][n] = mma(fy, fs[n], al[i][n]);
            ar[i][n] = mma(fv, fg[n], ar[i][n]);
          }
        }
      }
    }
    // gO V'^T and gY V'^T of the own row of tiles, and gY.v of its tokens
    v4f mo[kTiles], my[kTiles];
    float yv = 0.f;
#pragma unroll
    for (int j = 0; j < kTiles; ++j) mo[j] = my[j] = v4f{0.f, 0.f, 0.f, 0.f};
    for (int v0 = 8 * q; v0 < ws.VP; v0 += 32) {
      const int t = 16 * wave + m;
      float x[8], y[8];
      Frag fo[NP], fy[3];
      load_vec(gval + (long long)t * ws.VP + v0, y);
      split8(y, fy);
      columns8(v, t, tokens, KC, v0, ws.V, P, C, h, x);
#pragma unroll
      for (int c = 0; c < 8; ++c) yv = fmaf(x[c], y[c], yv);
      columns8(gy, t, tokens, KC, v0, ws.V, P, C, h, x);
      parts8<T>(x, fo);
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        if (j > wave) continue;
        Frag fv[3];
        wide_frag(val + (long long)(16 * j + m) * ws.VP + v0, fv);
        mo[j] = mma(fo, fv, mo[j]);
        my[j] = mma(fy, fv, my[j]);
      }
    }
    yv += __shfl_xor(yv, 16);
    yv += __shfl_xor(yv, 32);
    if (q == 0) direct[16 * wave + m] = yv;
    __syncthreads();  // the tokens' numbers are there, and the matrix has been read
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      if (j > wave) continue;
      const int u = 16 * j + m;
      const float4 other = tb[u];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * wave + 4 * q + r;
        const float4 me = tb[t];
        const float f = other.x * decay_between(me, other);
        mo[j][r] = t >= u ? mo[j][r] * f * (a.scale * me.y) : 0.f;
        my[j][r] = t > u ? -my[j][r] * f * me.x : 0.f;
      }
      put_tile(mat, wave, j, m, q, mo[j]);
    }
    // what the state gives, before the tokens' share: its part of q.Uq, k.UL, k.UR
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + 4 * q + r;
        const float4 tok = ta[t];
        float x = 0.f, y = 0.f, z = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          aq[i][n][r] *= tok.w;
          al[i][n][r] *= -tok.y;
          ar[i][n][r] *= tok.z;
          if (wave + 4 * n >= DT) continue;
          const int d = 16 * (wave + 4 * n) + m;
          const float ke = element(kbuf, t, d);
          x = fmaf(element(qbuf, t, d), aq[i][n][r], x);
          y = fmaf(ke, al[i][n][r], y);
          z = fmaf(ke, ar[i][n][r], z);
        }
        x = group_sum(x, 16);
        y = group_sum(y, 16);
        z = group_sum(z, 16);
        if (m == 0) {
          dots[0][wave][t] = x;
          dots[1][wave][t] = y;
          dots[2][wave][t] = z;
        }
      }
    both = group_sum(both, 64);
    if (lane == 0) whole_dot[wave] = both;
    // the tokens' share, of the own row of tiles: sums over j up to a column, then over i behind it
    {
      v4f left{0.f, 0.f, 0.f, 0.f}, before{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        float column = 0.f;
        if (j <= wave) {
          v4f qk{0.f, 0.f, 0.f, 0.f}, kk{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            Frag f[NP], fj[NP];
            rows_frag<NP, ST>(kbuf, j, kb, m, q, fj);
            rows_frag<NP, ST>(qbuf, wave, kb, m, q, f);
            qk = mma(f, fj, qk);
            rows_frag<NP, ST>(kbuf, wave, kb, m, q, f);
            kk = mma(f, fj, kk);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = 16 * wave + 4 * q + r;
            const float l = my[j][r] * kk[r];
            left[r] += l;
            float x = t > 16 * j + m ? fmaf(mo[j][r], qk[r], ta[t].x * l) : 0.f;
            x += dpp<0x111>(x);  // from the lanes 1, 2, 4, 8 below, zero from outside the 16
            x += dpp<0x112>(x);
            x += dpp<0x114>(x);
            x += dpp<0x118>(x);
            x += before[r];
            before[r] = __shfl(x, 15, 16);
            column += t > 16 * j + m ? x : 0.f;
          }
        }
        column += __shfl_xor(column, 16);
        column += __shfl_xor(column, 32);
        if (q == 0) behind[wave][16 * j + m] = column;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = group_sum(left[r], 16);
        if (m == 0) dleft[16 * wave + 4 * q + r] = x;
      }
    }
    __syncthreads();  // M1 is there
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (wave + 4 * n >= DT) continue;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        Frag fk[NP], fq[NP], f[3];
        columns_frag<NP, ST>(kbuf, wave + 4 * n, kb, m, q, fk);
        columns_frag<NP, ST>(qbuf, wave + 4 * n, kb, m, q, fq);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          if (triangle_has<false>(i, kb)) {
            rows_frag<3, kMStride>(mat, i, kb, m, q, f);
            aq[i][n] = mma(f, fk, aq[i][n]);
          }
          if (triangle_has<true>(i, kb)) {
            columns_frag<3, kMStride>(mat, i, kb, m, q, f);
            ar[i][n] = mma(f, fq, ar[i][n]);
          }
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
      if (j <= wave) put_tile(mat, wave, j, m, q, my[j]);
    __syncthreads();  // M2 is there
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (wave + 4 * n >= DT) continue;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        Frag fk[NP], f[3];
        columns_frag<NP, ST>(kbuf, wave + 4 * n, kb, m, q, fk);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (triangle_has<false>(i, kb)) {
            rows_frag<3, kMStride>(mat, i, kb, m, q, f);
            al[i][n] = mma(f, fk, al[i][n]);
          }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
      if (j <= wave) {
#pragma unroll
        for (int r = 0; r < 4; ++r) my[j][r] *= ta[16 * wave + 4 * q + r].x;
        put_tile(mat, wave, j, m, q, my[j]);
      }
    __syncthreads();  // beta M2 is there
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (wave + 4 * n >= DT) continue;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        Frag fk[NP], f[3];
        columns_frag<NP, ST>(kbuf, wave + 4 * n, kb, m, q, fk);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          if (triangle_has<true>(i, kb)) {
            columns_frag<3, kMStride>(mat, i, kb, m, q, f);
            ar[i][n] = mma(f, fk, ar[i][n]);
          }
      }
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float beta = ta[16 * i + 4 * q + r].x;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          totq[i][n][r] += aq[i][n][r];
          totk[i][n][r] += fmaf(beta, al[i][n][r], ar[i][n][r]);
        }
      }
    if (wave == 0) {
      const auto over = [&](const float (&x)[4][kT], int t) { return (x[0][t] + x[1][t]) + (x[2][t] + x[3][t]); };
      const float left = over(dots[1], lane);
      float from = fmaf(ta[lane].x, left, over(dots[0], lane));  // summed from the token on
      float until = over(dots[2], lane);                         // summed up to the token
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const float x = __shfl_down(from, o), y = __shfl_up(until, o);
        if (lane + o < 64) from += x;
        if (lane >= o) until += y;
      }
      until = __shfl_up(until, 1);
      const float s = whole * ((whole_dot[0] + whole_dot[1]) + (whole_dot[2] + whole_dot[3])) + from +
                      (lane ? until + over(behind, lane - 1) : 0.f);
      if (lane < here) {
        const long long to = gate_at(lane, h);
        if (g.gdecay) g.gdecay[to] = lane < tokens ? s : 0.f;
        if (g.gbeta) g.gbeta[to] = lane < tokens ? left + dleft[lane] + direct[lane] : 0.f;
      }
    }
  }
  // through the norms of key and query, and out
  if (a.normalize) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + 4 * q + r;
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (wave + 4 * n >= DT) continue;
          const int d = 16 * (wave + 4 * n) + m;
          x = fmaf(element(qbuf, t, d), totq[i][n][r], x);
          y = fmaf(element(kbuf, t, d), totk[i][n][r], y);
        }
        x = group_sum(x, 16);
        y = group_sum(y, 16);
        if (i == 0 && r == 0) __syncthreads();  // the last head's dots have been read
        if (m == 0) {
          dots[0][wave][t] = x;
          dots[1][wave][t] = y;
        }
      }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = 16 * i + 4 * q + r;
      float x = 0.f, y = 0.f;
      if (a.normalize) {
        const float4 f = tb[t];
        x = f.y * f.y * ((dots[0][0][t] + dots[0][1][t]) + (dots[0][2][t] + dots[0][3][t]));
        y = f.x * f.x * ((dots[1][0][t] + dots[1][1][t]) + (dots[1][2][t] + dots[1][3][t]));
      }
      if (t >= here) continue;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int d = 16 * (wave + 4 * n) + m;
        if (d >= D) continue;
        const bool there = t < tokens;
        if (gq) gq[t * stride + d] = there ? (T)fmaf(-x, element(qbuf, t, d), totq[i][n][r]) : (T)0.f;
        if (gk) gk[t * stride + d] = there ? (T)fmaf(-y, element(kbuf, t, d), totk[i][n][r]) : (T)0.f;
      }
    }
}

template <class T, int KB>
hipError_t backward(const RuleBwdArgs& g, const RuleWs& w, hipStream_t s) {
  const auto walk = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3((w.VP + 16 * waves - 1) / (16 * waves), w.units, w.segments), dim3(64 * waves), 0, s,
                       g, w);
    return hipGetLastError();
  };
  hipError_t e = hipSuccess;
  if (w.segments > 1) {
    e = w.V <= 64 ? walk(rule_reverse_kernel<T, KB, 4, true>, 4) : walk(rule_reverse_kernel<T, KB, 8, true>, 8);
    if (e == hipSuccess) e = launch_rule_join(g.gstate, w, g.a.n, true, s);
    if (e != hipSuccess) return e;
  }
  e = w.V <= 64 ? walk(rule_reverse_kernel<T, KB, 4, false>, 4) : walk(rule_reverse_kernel<T, KB, 8, false>, 8);
  if (e != hipSuccess || !(g.gq || g.gk || g.gdecay || g.gbeta)) return e;
  hipLaunchKernelGGL((rule_grads_kernel<T, KB>), dim3(w.chunks, g.a.n.B * g.a.n.Hk), dim3(256), 0, s, g, w);
  return hipGetLastError();
}

template <class T>
hipError_t backward_any(const RuleBwdArgs& g, const RuleWs& w, hipStream_t s) {
  switch (w.KB) {
    case 1: return backward<T, 1>(g, w, s);
    case 2: return backward<T, 2>(g, w, s);
    case 3: return backward<T, 3>(g, w, s);
    default: return backward<T, 4>(g, w, s);
  }
}

}  // namespace

hipError_t launch_rule_backward(const RuleBwdArgs& g, hipStream_t s) {
  const RuleWs w = rule_workspace(g.a.n, true, g.a.ws, nullptr);
  hipError_t e = launch_rule_prepare(g.a, w, true, s);
  if (e == hipSuccess) e = launch_rule_states(g.a, w, true, s);
  if (e != hipSuccess) return e;
  return g.a.type == SEQ_BF16 ? backward_any<bf16>(g, w, s) : backward_any<float>(g, w, s);
}

}  // namespace cgconv
