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

// Block (chunk, unit) of four waves; wave w has the tile of rows 16 w.  BACKWARD: the inverse
// also transposed, P only transposed.  4 x 8192 tokens of 16 heads of 128 x 128, bf16: 116 us,
// of which 86 are its 0.45 GB of keys, queries and triangles at the rate of a large copy; the
// chain of 3 + 3 joined blocks does not quite hide behind them.
template <class T, int KB, bool BACKWARD>
__global__ __launch_bounds__(256) void rule_prepare_kernel(RuleArgs a, RuleWs ws) {
  constexpr int NP = kParts<T>, ST = row_stride(KB), kRow = kT + 4;
  constexpr int kRows = 2 * NP * kT * ST * 2, kTriangles = 2 * kT * kRow * 4;
  // the keys and queries, and the triangle and its inverse where they have been
  __shared__ __attribute__((aligned(16))) char space[kRows > kTriangles ? kRows : kTriangles];
  __shared__ float4 tok[kT];  // beta, rk; the second of Token's z, w
  __shared__ float rq[kT];
  __shared__ double sum[kT];
  __shared__ int odd;  // first row of A that is not finite
  auto& kbuf = reinterpret_cast<bf16(*)[NP][kT * ST]>(space)[0];
  auto& qbuf = reinterpret_cast<bf16(*)[NP][kT * ST]>(space)[1];
  float* tri = reinterpret_cast<float*>(space);
  float* inv = tri + kT * kRow;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int m = lane & 15, q = lane >> 4;
  const int chunk = blockIdx.x, unit = blockIdx.y, b = unit / a.n.H, h = unit - b * a.n.H;
  const int t0 = chunk * kT, tokens = min(tokens_of(a, b) - t0, kT);
  if (tokens <= 0) return;
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk), stride = a.n.Hk * D;
  const long long row0 = ((long long)b * a.n.N + t0) * stride + (long long)hk * D;
  const long long at = (long long)unit * ws.chunks + chunk;
  RowStage<T, KB, 256> sk, sq;
  sk.load(static_cast<const T*>(a.k) + row0, stride, tokens, D, tid);
  sq.load(static_cast<const T*>(a.q) + row0, stride, tokens, D, tid);
  if (wave == 0) {
    const long long gate = ((long long)b * a.n.N + t0 + min(lane, tokens - 1)) * a.n.H + h;
    const float x = a.decay[gate], bt = a.beta[gate];
    double g = lane < tokens ? x < kLowestDecay ? kLowestDecay : x : 0.f;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const double o = __shfl_up(g, s);
      if (lane >= s) g += o;
    }
    g *= 1.4426950408889634;  // log2(e)
    sum[lane] = g;
    const float hi = (float)g;
    tok[lane] = make_float4(lane < tokens ? bt : 0.f, 0.f, hi, (float)(g - hi));
  }
  sk.store(kbuf, tokens, D, tid);
  sq.store(qbuf, tokens, D, tid);
  if (tid == 0) odd = kT;
  __syncthreads();
  const int t = 16 * wave + m;
  // products of all pairs on and below the diagonal: kk and (forward) qk with rows j and the own
  // tile's columns i, (backward) kq with rows i and the own tile's columns j; a lane has four of its row
  v4f kk[kTiles], pq[kTiles], qq{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kTiles; ++j) kk[j] = pq[j] = qq;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    Frag ownk[NP], ownq[NP];
    rows_frag<NP, ST>(kbuf, wave, kb, m, q, ownk);
    rows_frag<NP, ST>(qbuf, wave, kb, m, q, ownq);
    qq = mma(ownq, ownq, qq);
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      Frag f[NP];
      if (j <= wave) {
        rows_frag<NP, ST>(kbuf, j, kb, m, q, f);
        kk[j] = mma(f, ownk, kk[j]);
        if (!BACKWARD) pq[j] = mma(f, ownq, pq[j]);
      }
      if (BACKWARD && j >= wave) {
        rows_frag<NP, ST>(qbuf, j, kb, m, q, f);
        pq[j] = mma(f, ownk, pq[j]);
      }
    }
  }
  // the norms are the diagonals
#pragma unroll
  for (int j = 0; j < kTiles; ++j)
    if (j == wave) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * q + r == m) {
          tok[t].y = a.normalize ? 1.f / __builtin_sqrtf(kk[j][r] + kRuleNormEps) : 1.f;
          rq[t] = a.normalize ? 1.f / __builtin_sqrtf(qq[r] + kRuleNormEps) : 1.f;
        }
    }
  __syncthreads();
  const float4 me = tok[t];
  const float sq_ = a.scale * (BACKWARD ? 1.f : rq[t]);
  float zero = 0.f;  // NaN if the lane has an entry of A that is not finite
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    v4f p = pq[j];
    if (j <= wave) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int u = 16 * j + 4 * q + r;
        const float4 other = tok[u];
        const float f = decay_between(me, other) * other.y;
        const float x = t > u ? me.x * me.y * f * kk[j][r] : 0.f;
        tri[t * kRow + u] = x;
        zero = fmaf(x, 0.f, zero);
        if (!BACKWARD) p[r] = t >= u ? p[r] * f * sq_ : 0.f;
      }
      if (!BACKWARD)
        ws.inside[(at * kBlocks + block_of(wave, j)) * 64 + lane] = make_float4(p[0], p[1], p[2], p[3]);
    }
    if (BACKWARD && j >= wave) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int u = 16 * j + 4 * q + r;
        p[r] = u >= t ? p[r] * decay_between(tok[u], me) * (rq[u] * me.y * sq_) : 0.f;
      }
      ws.inside[(at * kBlocks + block_of(j, wave)) * 64 + lane] = make_float4(p[0], p[1], p[2], p[3]);
    }
  }
  if (zero != 0.f) atomicMin(&odd, t);  // the least of them, in whatever order
  __syncthreads();
  // Rows of A from the first that is not finite on stay out of the products, whose zeros would
  // take them to the rows before; those of the inverse are NaN left of the diagonal.
  const int bad = __builtin_amdgcn_readfirstlane(odd);
  if (bad < kT) {
    for (int i = tid; i < (kT - bad) * kT; i += 256) tri[(bad + i / kT) * kRow + i % kT] = 0.f;
    __syncthreads();
  }
  // Diagonal blocks: the inverse of blocks twice as large, X <- X - X C X with C the part of A
  // that joins two of them.  X is held as it accumulates and transposed: the one is an operand
  // of the other's products as it is.
  {
    v4f row, col;  // A: row m, columns 4 q + r; column m, rows 4 q + r
    const float* at = tri + 16 * wave * kRow + 16 * wave;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      row[r] = at[m * kRow + 4 * q + r];
      col[r] = at[(4 * q + r) * kRow + m];
    }
    const auto joins = [](int i, int j, int size) { return ((i ^ j) & -size) == size && (i & size); };
    v4f X, Xt;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * q + r;
      X[r] = (i == m ? 1.f : 0.f) - (joins(i, m, 1) ? col[r] : 0.f);
      Xt[r] = (i == m ? 1.f : 0.f) - (joins(m, i, 1) ? row[r] : 0.f);
    }
#pragma unroll
    for (int size = 2; size < 16; size *= 2) {
      v4f P{0.f, 0.f, 0.f, 0.f}, Q = P;  // C X and its transpose's counterpart
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        P = __builtin_amdgcn_mfma_f32_16x16x4f32(joins(m, 4 * q + e, size) ? row[e] : 0.f, X[e], P, 0, 0, 0);
        Q = __builtin_amdgcn_mfma_f32_16x16x4f32(joins(4 * q + e, m, size) ? col[e] : 0.f, Xt[e], Q, 0, 0, 0);
      }
      const v4f x = X, xt = Xt;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        X = __builtin_amdgcn_mfma_f32_16x16x4f32(-xt[e], P[e], X, 0, 0, 0);
        Xt = __builtin_amdgcn_mfma_f32_16x16x4f32(-x[e], Q[e], Xt, 0, 0, 0);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) inv[(16 * wave + 4 * q + r) * kRow + 16 * wave + m] = X[r];
  }
  __syncthreads();
  // block (i, j) = - inv(i, i) sum_{j <= c < i} A(i, c) inv(c, j), by distance i - j
#pragma unroll
  for (int dist = 1; dist < kTiles; ++dist) {
    if (wave >= dist) {
      const int i = wave, j = wave - dist;
      v4f s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < dist; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = 16 * (j + n) + 4 * q + e;
          s = __builtin_amdgcn_mfma_f32_16x16x4f32(tri[(16 * i + m) * kRow + c], inv[c * kRow + 16 * j + m], s, 0, 0, 0);
        }
      v4f o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o = __builtin_amdgcn_mfma_f32_16x16x4f32(-inv[(16 * i + m) * kRow + 16 * i + 4 * q + e], s[e], o, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) inv[(16 * i + 4 * q + r) * kRow + 16 * j + m] = o[r];
    }
    __syncthreads();
  }
  for (int n = wave; n < kBlocks; n += 4) {
    const int i = row_of(n), j = n - block_of(i, 0);
    // a lane's four entries from (row, column) on, down or along the row
    const auto entries = [&](int row, int column, int down) {
      const float* p = inv + row * kRow + column;
      float4 x = down ? make_float4(p[0], p[kRow], p[2 * kRow], p[3 * kRow]) : make_float4(p[0], p[1], p[2], p[3]);
      if (bad < kT) {
        const auto lost = [&](int e) { return row + e * down >= bad && column + e * !down < row + e * down; };
        const float nan = __builtin_nanf("");
        x = make_float4(lost(0) ? nan : x.x, lost(1) ? nan : x.y, lost(2) ? nan : x.z, lost(3) ? nan : x.w);
      }
      return x;
    };
    ws.inv[(at * kBlocks + n) * 64 + lane] = entries(16 * i + m, 16 * j + 4 * q, 0);
    if (BACKWARD) ws.invT[(at * kBlocks + n) * 64 + lane] = entries(16 * i + 4 * q, 16 * j + m, 1);
  }
  if (wave == 0) {
    const float4 x = tok[lane];
    const double end = sum[kT - 1];
    // a float's exponential is off by its rounding times the number: the rest of the sum makes up for it
    const float e = __builtin_amdgcn_exp2f(x.z) * fmaf(x.w, 0.6931472f, 1.f), eh = (float)end;
    const float until = __builtin_amdgcn_exp2f((float)(end - sum[lane]));
    float4* to = ws.token + (at * kT + lane) * 2;
    to[0] = make_float4(x.x, x.y * e, x.y * until, a.scale * rq[lane] * e);
    to[1] = make_float4(x.y, rq[lane], x.z, x.w);
    if (lane == 0) ws.whole[at] = __builtin_amdgcn_exp2f(eh) * fmaf((float)(end - eh), 0.6931472f, 1.f);
  }
}

// ---- the states, chunk after chunk ------------------------------------------------------

// What a walk over the chunks leaves.
enum Walk {
  kOutputs,  // the outputs, and the last state
  kKeep,     // the state before every chunk and V', for the backward
  kSpan,     // of every segment of the chunks but the last: its last state, of the first from the
             // given one, of others from zero, and of these also from every unit vector with no
             // values written, which is the segment's matrix
};

// Block (128 columns, unit, segment).  The columns of kSpan are the VP of the
// values, then those of the matrix.  A wave's chunk is a chain of products, each waiting for
// the one before, so it is bound by latency: with heads of 128 x 128 and eight waves a block,
// a chunk of 64 tokens takes 8.6 us with its outputs, 5.3 without; the matrix cores are busy 29%
// of the time, the vector units 40%, the LDS 36%.  More of a state's columns in a wave (32: 860
// us of a prompt instead of 688) or fewer waves that share a chunk (four: 1061, and for heads of
// 64 columns, which occupy no more, 195 us instead of 174) are slower; a chunk in LDS ahead, and
// products of one accumulator apart, took 740 to 688.
//
// CAREFUL: what is not finite stays out of the triangles' products.  Returns whether a column of
// the last state is not finite, so that the segment is to be walked again with care; of kSpan
// nothing else is wanted than that the column is.
template <class T, int KB, int WALK>
struct WalkSpace {
  typedef Stage<T, KB, WALK == kOutputs, WALK == kOutputs> Buffer;
  Buffer buffers[Buffer::kCount];
  int again;
};
template <class T, int KB, int WALK>
__device__ __forceinline__ WalkSpace<T, KB, WALK>& walk_space() {
  __shared__ WalkSpace<T, KB, WALK> space;
  return space;
}

template <class T, int KB, int WALK, bool CAREFUL>
__device__ __forceinline__ bool rule_walk(const RuleArgs& a, const RuleWs& ws) {
  constexpr int NP = kParts<T>, DT = 2 * KB, kThreads = 64 * kWalkWaves;
  constexpr bool kOut = WALK == kOutputs;
  typedef typename WalkSpace<T, KB, WALK>::Buffer Buffer;
  constexpr int ST = Buffer::ST;
  auto& space = walk_space<T, KB, WALK>();
  auto& buffers = space.buffers;
  __shared__ float turn[WALK == kSpan ? kWalkWaves : 1][16][20];  // of the matrix: a tile, read along its rows
  // of a second walk the numbers are made anew, rather than held in registers through the first
  const auto lane_number = [](int x) { return CAREFUL ? afresh_lane(x) : x; };
  const auto block_number = [](int x) { return CAREFUL ? afresh(x) : x; };
  const int tid = lane_number(threadIdx.x), wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int m = lane & 15, q = lane >> 4;
  const int unit = block_number(blockIdx.y), b = unit / a.n.H, h = unit - b * a.n.H, seg = block_number(blockIdx.z);
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk), C = a.n.C, KC = a.n.K * C, N = a.n.N;
  const int first = (block_number(blockIdx.x) * kWalkWaves + wave) * 16;
  const bool matrix = WALK == kSpan && first >= ws.VP;
  const bool active = first < (kOut ? ws.V : WALK == kKeep ? ws.VP : ws.VP + 32 * KB) && !(matrix && seg == 0);
  if (WALK == kSpan && seg == 0 && (int)blockIdx.x * kWalkWaves * 16 >= ws.VP) return false;
  const Column column(first + m, ws.V, C / a.n.H, C, h);
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
      const int row = 16 * d + 4 * q + r, col = first + m;
      float x = 0.f;
      if (matrix) {
        x = row == col - ws.VP ? 1.f : 0.f;
      } else if (WALK == kSpan && seg > 0) {
      } else if (seg > 0) {
        if (col < ws.VP) x = ws.start[(start + row) * ws.VP + col];
      } else if (a.state_in && column.there && row < D) {
        x = a.state_in[((long long)b * D + row) * KC + column.at];
      }
      S[d][r] = x;
    }

  RowStage<T, KB, kThreads> sk, sq;
  BlockStage<kThreads> si, sp;
  float4 st;
  ColumnStage<T> sv;
  const auto fetch = [&](int c) {
    const int tokens = min(length - c * kT, kT);
    const long long at = (long long)unit * ws.chunks + c;
    sk.load(K + (long long)c * kT * stride, stride, tokens, D, tid);
    if (kOut) sq.load(Q + (long long)c * kT * stride, stride, tokens, D, tid);
    si.load(ws.inv + at * kBlocks * 64, tid);
    if (kOut) sp.load(ws.inside + at * kBlocks * 64, tid);
    st = ws.token[(at * kT + (tid & (kT - 1))) * 2];
  };
  const auto put = [&](int c, Buffer& to) {
    const int tokens = min(length - c * kT, kT);
    sk.store(to.k, tokens, D, tid);
    if constexpr (kOut) sq.store(to.q, tokens, D, tid);
    si.store(to.inv, tid);
    if constexpr (kOut) sp.store(to.inside, tid);
    if (tid < kT) to.token[tid] = st;
  };
  const auto fetch_values = [&](int c) {
    sv.load(v + (long long)c * kT * KC, KC, min(length - c * kT, kT), column, q);
  };
  if (WALK != kSpan && !CAREFUL && tid == 0) space.again = 0;
  if (begin < end) {
    fetch(begin);
    fetch_values(begin);
    if (Buffer::kCount == 2) {
      put(begin, buffers[0]);
      if (begin + 1 < end) fetch(begin + 1);
    }
  }
  for (int c = begin; c < end; ++c) {
    const int lane = afresh_lane(tid & 63), m = lane & 15, q = lane >> 4;
    const int tokens = min(length - c * kT, kT);
    const long long at = (long long)unit * ws.chunks + c;
    Buffer& buf = buffers[(c - begin) & (Buffer::kCount - 1)];
    const float whole = ws.whole[at];
    __syncthreads();  // the chunk is there; the one before has been read
    if (Buffer::kCount == 1) {
      put(c, buf);
      __syncthreads();
      if (c + 1 < end) fetch(c + 1);
    }
    const auto& kbuf = buf.k;
    const auto& qbuf = buf.q;
    const auto& inv = buf.inv;
    const auto& inside = buf.inside;
    const float4* ta = buf.token;
    v4f X[kTiles], O[kTiles];
    int odd = kT;  // the first place in the lane's column that is not finite
    if (active) {
      if constexpr (WALK == kKeep) {
        store_tiles(ws.state + at * (32 * KB) * ws.VP, ws.VP, first + m, q, S);
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i) X[i] = O[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        Frag s[3];
        split_tiles(S[2 * kb], S[2 * kb + 1], s);
        Frag f[kTiles][NP];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) rows_frag<NP, ST>(kbuf, i, kb, m, q, f[i]);
        mma_all(f, s, X);
        if constexpr (kOut) {
#pragma unroll
          for (int i = 0; i < kTiles; ++i) rows_frag<NP, ST>(qbuf, i, kb, m, q, f[i]);
          mma_all(f, s, O);
        }
      }
      // Y, then V' = (1 + A)^-1 Y
      v4f beta[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 tok = ta[16 * i + 4 * q + r];
          X[i][r] = fmaf(-tok.y, X[i][r], sv.get(i, r, column));
          beta[i][r] = tok.x;
          if constexpr (kOut) O[i][r] *= tok.w;
        }
      if (c + 1 < end) fetch_values(c + 1);
      if constexpr (CAREFUL) {
        odd = min(first_odd<false>(X, q), first_odd<false>(beta, q));
        put_from<false>(X, odd, q, 0.f);
        put_from<false>(beta, odd, q, 0.f);
      }
      Frag fy[2][3];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) split_products(X[2 * kb], beta[2 * kb], X[2 * kb + 1], beta[2 * kb + 1], fy[kb]);
#pragma unroll
      for (int i = 0; i < kTiles; ++i) X[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) mma_triangle<false>(inv, kb, lane, fy[kb], X);
    }
    if (Buffer::kCount == 2 && c + 1 < end) {
      put(c + 1, buffers[(c + 1 - begin) & 1]);
      if (c + 2 < end) fetch(c + 2);
    }
    if (!active) continue;
    if constexpr (CAREFUL) {
      if (kOut) odd = min(odd, first_odd<false>(X, q));  // the inverse has more
      put_from<false>(X, odd, q, kOut ? 0.f : __builtin_nanf(""));
    }
    if constexpr (WALK == kKeep) {
      store_tiles(ws.value + at * kT * ws.VP, ws.VP, first + m, q, X);
    }
    if constexpr (kOut) {
      Frag fv[2][3];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) split_tiles(X[2 * kb], X[2 * kb + 1], fv[kb]);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) mma_triangle<false>(inside, kb, lane, fv[kb], O);
      if constexpr (CAREFUL) {
        put_from<false>(O, odd, q, __builtin_nanf(""));
        put_from<false>(X, odd, q, __builtin_nanf(""));
      }
      store_column(y + (long long)c * kT * KC, KC, N - c * kT, tokens, column, q, O);
    }
    // S <- e^{G_end} S + K^T (e^{G_end - G} rk V')
    Frag fz[2][3];
    v4f late[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) late[i][r] = ta[16 * i + 4 * q + r].z;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) split_products(X[2 * kb], late[2 * kb], X[2 * kb + 1], late[2 * kb + 1], fz[kb]);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[d][r] *= whole;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      Frag f[DT][NP];
#pragma unroll
      for (int d = 0; d < DT; ++d) columns_frag<NP, ST>(kbuf, d, kb, m, q, f[d]);
      mma_all(f, fz[kb], S);
    }
  }
  bool again = false;
  if (WALK != kSpan && !CAREFUL && begin < end) {
    if (any_odd(S)) space.again = 1;
    __syncthreads();
    again = __builtin_amdgcn_readfirstlane(space.again) != 0;
  }
  if constexpr (WALK == kSpan) {
    if (!active) return false;
    const int col = first + m;
    if (!matrix) {
      store_tiles(ws.span_state + start * ws.VP, ws.VP, col, q, S);
    } else {
      const int j = (first - ws.VP) / 16;  // the matrix's columns from 16 j on
      const long long at = ((long long)unit * ws.segments + seg) * (DT * KB * 3 * 64);
      auto& tile = turn[wave];
#pragma unroll
      for (int d = 0; d < DT; ++d) {
#pragma unroll
        for (int r = 0; r < 4; ++r) tile[4 * q + r][m] = S[d][r];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const v4f x = *reinterpret_cast<const v4f*>(&tile[m][4 * q]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        uint2 part[3];
        split2(x[0], x[1], part[0].x, part[1].x, part[2].x);
        split2(x[2], x[3], part[0].y, part[1].y, part[2].y);
        uint4* to = ws.span_matrix + at + ((d * KB + j / 2) * 3) * 64 + lane;
#pragma unroll
        for (int p = 0; p < 3; ++p) reinterpret_cast<uint2*>(to + 64 * p)[j & 1] = part[p];
      }
      if (ws.span_matrixT) {
        uint4* to = ws.span_matrixT + at + (j * KB * 3) * 64 + lane;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          Frag f[3];
          split_tiles(S[2 * kb], S[2 * kb + 1], f);
#pragma unroll
          for (int p = 0; p < 3; ++p) to[64 * (3 * kb + p)] = f[p].all;
        }
      }
    }
  }
  if constexpr (kOut) {
    if (!column.there) return again;
    const long long stop = min((long long)last * kT, (long long)N);
    for (long long n = (long long)max(end, begin) * kT + q; n < stop; n += 4) y[n * KC + column.at] = (T)0.f;
    if (!a.state_out || last != ws.chunks) return again;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * d + 4 * q + r;
        if (row < D) a.state_out[((long long)b * D + row) * KC + column.at] = S[d][r];
      }
  }
  return again;
}

struct WalkArgs {
  RuleArgs a;
  RuleWs ws;
};
template <class T, int KB, int WALK>
__global__ __launch_bounds__(64 * kWalkWaves) void rule_state_kernel(WalkArgs w) {
  const bool again = rule_walk<T, KB, WALK, false>(w.a, w.ws);
  if constexpr (WALK != kSpan) {
    if (again) {
      const auto once_more = argument_anew<WalkArgs>();
      rule_walk<T, KB, WALK, true>(once_more.a, once_more.ws);
    }
  }
}

// ---- one token ---------------------------------------------------------------------------

// Block (group of columns, unit): 16 vectors of VC columns side by side, 16 rows of the state at
// a time, all of a thread's rows in registers, so the state is read once and written once.  Bound
// by its bytes: 64 sequences of 16 heads of 128 x 128, 134 MB, 25.9 us, 5.2 TB/s (38 in blocks of
// 16 columns); of few sequences by the latency of one chain load - sum - store (one sequence
// 4.5 us, as in blocks of 16 columns).  Both sums over the rows come first:
//   y = scale (e^g qn.S + (qn.kn) u),   u = beta (v - e^g kn.S),   S <- e^g S + kn u.
template <class T, int VC>
__global__ __launch_bounds__(256) void rule_step_kernel(RuleArgs a, int V) {
  constexpr int LANES = 16, kGroups = 256 / LANES, kRows = kRuleMaxDim / kGroups;
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

template <class T, int WALK>
hipError_t walk(const RuleArgs& a, const RuleWs& w, hipStream_t s) {
  constexpr int kColumns = 16 * kWalkWaves;
  const int columns = WALK == kOutputs ? w.V : WALK == kKeep ? w.VP : w.VP + 32 * w.KB;
  const dim3 grid((columns + kColumns - 1) / kColumns, w.units, WALK == kSpan ? w.segments - 1 : w.segments);
  return by_width(w.KB, [&](auto kb) {
    hipLaunchKernelGGL((rule_state_kernel<T, decltype(kb)::value, WALK>), grid, dim3(64 * kWalkWaves), 0, s,
                       WalkArgs{a, w});
    return hipGetLastError();
  });
}

template <class T>
hipError_t states(const RuleArgs& a, const RuleWs& w, bool backward, hipStream_t s) {
  if (w.segments > 1) {
    hipError_t e = walk<T, kSpan>(a, w, s);
    if (e == hipSuccess) e = launch_rule_join(w, false, s);
    if (e != hipSuccess) return e;
  }
  return backward ? walk<T, kKeep>(a, w, s) : walk<T, kOutputs>(a, w, s);
}

template <class T>
hipError_t step(const RuleArgs& a, hipStream_t s) {
  const int P = a.n.C / a.n.H, V = a.n.K * P, units = a.n.B * a.n.H;
  const auto run = [&](auto kernel, int columns) {
    hipLaunchKernelGGL(kernel, dim3((V + columns - 1) / columns, units), dim3(256), 0, s, a, V);
    return hipGetLastError();
  };
  return P % 4 == 0 ? run(rule_step_kernel<T, 4>, 64) : run(rule_step_kernel<T, 1>, 16);
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
