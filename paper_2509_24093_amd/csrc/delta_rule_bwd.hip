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

// Block (128 columns, unit, segment).  SPAN: of every segment but the first only
// the gradient of the state before it, of the last from the given one, of others from zero.
// Bound as the forward's walk: a chunk of a 128 x 128 head takes 10 us, 7.3 with SPAN.
// CAREFUL and what it returns: as rule_walk, of the first gradient of the state.
template <class T, int KB>
struct ReverseSpace {
  typedef Stage<T, KB, true, true> Buffer;  // the transposed triangles
  Buffer buffers[Buffer::kCount];
  int again;
};
template <class T, int KB>
__device__ __forceinline__ ReverseSpace<T, KB>& reverse_space() {
  __shared__ ReverseSpace<T, KB> space;
  return space;
}

template <class T, int KB, bool SPAN, bool CAREFUL>
__device__ __forceinline__ bool rule_reverse(const RuleBwdArgs& g, const RuleWs& ws) {
  constexpr int NP = kParts<T>, DT = 2 * KB, kThreads = 64 * kWalkWaves;
  typedef typename ReverseSpace<T, KB>::Buffer Buffer;
  constexpr int ST = Buffer::ST;
  auto& space = reverse_space<T, KB>();
  auto& buffers = space.buffers;
  const RuleArgs& a = g.a;
  const auto lane_number = [](int x) { return CAREFUL ? afresh_lane(x) : x; };
  const auto block_number = [](int x) { return CAREFUL ? afresh(x) : x; };
  const int tid = lane_number(threadIdx.x), wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int m = lane & 15, q = lane >> 4;
  const int unit = block_number(blockIdx.y), b = unit / a.n.H, h = unit - b * a.n.H, seg = block_number(blockIdx.z) + SPAN;
  const int D = a.n.D, hk = h / (a.n.H / a.n.Hk), C = a.n.C, KC = a.n.K * C, N = a.n.N;
  const int first = (block_number(blockIdx.x) * kWalkWaves + wave) * 16, col = first + m;
  const bool active = first < ws.VP;
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
      if (seg + 1 < ws.segments) {
        if (!SPAN && active) x = ws.start[(start + row) * ws.VP + col];
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
  if (!SPAN && !CAREFUL && tid == 0) space.again = 0;
  if (begin < end) {
    fetch(end - 1);
    so.load(gy + (long long)(end - 1) * kT * KC, KC, min(length - (end - 1) * kT, kT), column, q);
    if (Buffer::kCount == 2) {
      put(end - 1, buffers[0]);
      if (end - 2 >= begin) fetch(end - 2);
    }
  }
  for (int c = end - 1; c >= begin; --c) {
    const int lane = afresh_lane(tid & 63), m = lane & 15, q = lane >> 4;
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
    int odd = kT;  // the first place in the lane's column that is not finite, from the last token back
    if constexpr (CAREFUL) {
      v4f o[kTiles];
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[i][r] = so.get(i, r, column);
      odd = first_odd<true>(o, q);
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (place_of<true>(i, r, q) >= odd) so.v[i][r] = (T)0.f;
    }
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
    if constexpr (CAREFUL) {
      odd = min(odd, first_odd<true>(X, q));  // the state's gradient and P have more
      put_from<true>(X, odd, q, 0.f);
    }
    Frag fx[2][3];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) split_tiles(X[2 * kb], X[2 * kb + 1], fx[kb]);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) X[i] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) mma_triangle<true>(inv, kb, lane, fx[kb], X);
    if constexpr (CAREFUL) put_from<true>(X, odd, q, __builtin_nanf(""));
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
  bool again = false;
  if (!SPAN && !CAREFUL && begin < end) {
    if (any_odd(S)) space.again = 1;
    __syncthreads();
    again = __builtin_amdgcn_readfirstlane(space.again) != 0;
  }
  if constexpr (SPAN) {
    if (active) store_tiles(ws.span_state + start * ws.VP, ws.VP, col, q, S);
    return false;
  }
  if (!column.there) return again;
  if (gv) {
    const long long stop = min((long long)last * kT, (long long)N);
    for (long long t = (long long)max(end, begin) * kT + q; t < stop; t += 4) gv[t * KC + column.at] = (T)0.f;
  }
  if (!g.gstate_in || seg > 0) return again;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * d + 4 * q + r;
      if (row < D) g.gstate_in[((long long)b * D + row) * KC + column.at] = S[d][r];
    }
  return again;
}

struct ReverseArgs {
  RuleBwdArgs g;
  RuleWs ws;
};
template <class T, int KB, bool SPAN>
__global__ __launch_bounds__(64 * kWalkWaves) void rule_reverse_kernel(ReverseArgs r) {
  const bool again = rule_reverse<T, KB, SPAN, false>(r.g, r.ws);
  if constexpr (!SPAN) {
    if (again) {
      const auto once_more = argument_anew<ReverseArgs>();
      rule_reverse<T, KB, SPAN, true>(once_more.g, once_more.ws);
    }
  }
}

// ---- gradients of keys, queries, decays and betas -------------------------------------------

// Eight columns from col on of a chunk's token (row: its first token), a slice ahead of their
// use; zeros where there is no column or no token.  PACKED: eight columns of a head are neighbours
// in memory (P a multiple of eight), one load; what is not there is read from a place that is.
template <class T, bool PACKED>
struct SliceStage {
  Raw<T, 8> raw;
  // at: bytes of the token's row from the base
  __device__ __forceinline__ void load(const T* base, uint32_t at, int col, int V, int P, int C, int h) {
    if constexpr (PACKED) {
      raw.load(&place(base, at + Column(col, V, P, C, h).at * (int)sizeof(T)));
    } else {
      T x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = place(base, at + Column(col + e, V, P, C, h).at * (int)sizeof(T));
      __builtin_memcpy(raw.w, x, sizeof x);
    }
  }
  __device__ __forceinline__ void get(bool there, int col, int V, float (&x)[8]) const {
    raw.widen_to(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = there && col + e < V ? x[e] : 0.f;
  }
};

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

// 32 columns of a chunk's V', gY and gO, in parts.
template <class T>
struct Slice {
  static constexpr int ST = row_stride(1);
  alignas(16) bf16 value[3][kT * ST], gvalue[3][kT * ST], gy[kParts<T>][kT * ST];
};

// Operand with a slice's rows 16 i + m: lane group q has the columns 8 q .. 8 q + 7, as it has of
// the other operand's rows.
template <int NP, int N>
__device__ __forceinline__ void slice_frag(const bf16 (&buf)[NP][N], int i, int m, int q, Frag (&f)[NP]) {
#pragma unroll
  for (int p = 0; p < NP; ++p)
    f[p].all = *reinterpret_cast<const uint4*>(buf[p] + (16 * i + m) * (N / kT) + 8 * q);
}

// What a block of rule_grads_kernel shares.  The slices make room for the matrices M1 and beta
// M2; two of each where they fit, so that the waves meet once a slice, or once for both.
template <class T, int KB>
struct GradsSpace {
  static constexpr int NP = kParts<T>, ST = row_stride(KB);
  alignas(16) bf16 k[NP][kT * ST];
  alignas(16) bf16 q[NP][kT * ST];
  float4 ta[kT], tb[kT];
  float dots[3][8][kT], behind[8][kT], direct[kT], dleft[kT], whole_dot[8];
  static constexpr int kLeft = 160 * 1024 - 4 * NP * kT * ST - 32 * kT - 4 * kT * 34 - 64;
  static constexpr int kSlices = 2 * (int)sizeof(Slice<T>) <= kLeft ? 2 : 1;
  static constexpr int kSquares = 2 * (int)sizeof(Square) <= kLeft ? 2 : 1;
  union {
    Slice<T> slice[kSlices];
    Square mat[kSquares];
  };
};

// Block (chunk, sequence and key head) of eight waves, the heads that share the key one after
// the other.  Wave w owns the tile of the 16 key components from 16 w on (rows of S and gS) for
// all tokens; of the 64 x 64 matrices wave w < 4 has the row of tiles w of M1, wave w + 4 that
// of M2.  1024 chunks of 128 x 128 heads in bf16: 134 us, four rounds of blocks (a block's
// accumulators fill the registers of a CU), 0.23 GB at 1.7 TB/s; half of the time is waiting,
// for the slices' loads and at the meetings, and the LDS is busy 42%.  With four waves that read
// and split the columns each for itself 313 us, with branches around the slices' loads 228.
template <class T, int KB, bool PACKED>
__global__ __launch_bounds__(512) void rule_grads_kernel(RuleBwdArgs g, RuleWs ws) {
  typedef GradsSpace<T, KB> Space;
  constexpr int NP = kParts<T>, ST = row_stride(KB), DT = 2 * KB, SS = Slice<T>::ST;
  __shared__ Space space;
  auto& kbuf = space.k;
  auto& qbuf = space.q;
  auto& ta = space.ta;
  auto& tb = space.tb;
  auto& dots = space.dots;
  const RuleArgs& a = g.a;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int m = lane & 15, q = lane >> 4;
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
    for (int i = tid; i < here * D; i += 512) {
      const int at = (i / D) * stride + i % D;
      if (gq) gq[at] = (T)0.f;
      if (gk) gk[at] = (T)0.f;
    }
    for (int i = tid; i < here * each; i += 512) {
      const long long at = gate_at(i / each, hk * each + i % each);
      if (g.gdecay) g.gdecay[at] = 0.f;
      if (g.gbeta) g.gbeta[at] = 0.f;
    }
    return;
  }
  {
    RowStage<T, KB, 512> k, q;
    k.load(static_cast<const T*>(a.k) + key0, stride, tokens, D, tid);
    q.load(static_cast<const T*>(a.q) + key0, stride, tokens, D, tid);
    k.store(kbuf, tokens, D, tid);
    q.store(qbuf, tokens, D, tid);
  }
  // an element of the keys or queries as stored
  const auto element = [&](const bf16 (&buf)[NP][kT * ST], int t, int d) {
    float x = 0.f;
#pragma unroll
    for (int p = NP - 1; p >= 0; --p) x += (float)buf[p][t * ST + d];
    return x;
  };
  const bool owner = wave < DT, second = wave >= 4;  // has key components; has a row of M2
  const int row = wave & 3, own = 16 * wave + m;
  const int st = (tid & 255) >> 2, sc = (tid & 3) * 8;  // token and columns of a slice that a thread brings
  v4f totq[kTiles], totk[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) totq[i] = totk[i] = v4f{0.f, 0.f, 0.f, 0.f};

  for (int e = 0; e < each; ++e) {
    const int lane = afresh_lane(tid & 63), m = lane & 15, q = lane >> 4, own = 16 * wave + m;
    const int h = hk * each + e, unit = b * a.n.H + h;
    const long long at = (long long)unit * ws.chunks + chunk;
    const float* S = ws.state + at * (32 * KB) * ws.VP;
    const float* gS = ws.gstate + at * (32 * KB) * ws.VP;
    const float* wide = (second ? ws.value : ws.gvalue) + at * kT * ws.VP;
    const uint32_t state_at = 4 * (__umul24(owner ? own : 0, ws.VP) + 8 * q), wide_at = 4 * (__umul24(st, ws.VP) + sc);
    const uint32_t row_at = __umul24(min(st, tokens - 1), KC * (int)sizeof(T));
    const T* rows = static_cast<const T*>(second ? g.gy : a.v) + ((long long)b * N + t0) * KC;
    const float whole = ws.whole[at];
    const float4 token = ws.token[at * 2 * kT + (tid & (2 * kT - 1))];

    // S gO, S gY, gS V' over the columns, <S, gS>, gO V'^T or gY V'^T of the own row of tiles, and gY.v
    v4f aq[kTiles], al[kTiles], ar[kTiles], w[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) aq[i] = al[i] = ar[i] = w[i] = v4f{0.f, 0.f, 0.f, 0.f};
    float both = 0.f, yv = 0.f;
    Raw<float, 8> wide_raw;
    Raw<float, 8> state_raw, gstate_raw;
    SliceStage<T, PACKED> narrow;
    // asked for a slice ahead, the last one twice: a branch here would wait for it
    const auto fetch = [&](int v0) {
      wide_raw.load(&place(wide, wide_at + 4 * v0));
      narrow.load(rows, row_at, v0 + sc, ws.V, P, C, h);
      state_raw.load(&place(S, state_at + 4 * v0));
      gstate_raw.load(&place(gS, state_at + 4 * v0));
    };
    fetch(0);
    __syncthreads();  // the head before has been read
    if (tid < 2 * kT) (tid & 1 ? tb : ta)[tid >> 1] = token;
    for (int v0 = 0, n = 0; v0 < ws.VP; v0 += 32, ++n) {
      auto& slice = space.slice[n & (Space::kSlices - 1)];
      if (Space::kSlices == 1 && n) __syncthreads();  // the one before has been read
      {
        float x[8], wx[8];
        Frag f[3];
        wide_raw.widen_to(wx);
        narrow.get(st < tokens, v0 + sc, ws.V, x);
        split8(wx, f);
#pragma unroll
        for (int p = 0; p < 3; ++p)
          *reinterpret_cast<Frag*>((second ? slice.value : slice.gvalue)[p] + st * SS + sc) = f[p];
        if (second) {
          Frag o[NP];
          parts8<T>(x, o);
#pragma unroll
          for (int p = 0; p < NP; ++p) *reinterpret_cast<Frag*>(slice.gy[p] + st * SS + sc) = o[p];
        } else {
#pragma unroll
          for (int c = 0; c < 8; ++c) yv = fmaf(x[c], wx[c], yv);
        }
      }
      Frag fs[3], fg[3];
      {
        float x[8], y[8];
        state_raw.widen_to(x);
        gstate_raw.widen_to(y);
        if (owner) {
#pragma unroll
          for (int c = 0; c < 8; ++c) both = fmaf(x[c], y[c], both);
        }
        split8(x, fs);
        split8(y, fg);
      }
      fetch(min(v0 + 32, ws.VP - 32));
      __syncthreads();  // the slice is there
      Frag fv[kTiles][3];
#pragma unroll
      for (int i = 0; i < kTiles; ++i) slice_frag(slice.value, i, m, q, fv[i]);
      if (owner) mma_all(fv, fg, ar);
      if (second) {
        Frag f[3];
        slice_frag(slice.gvalue, row, m, q, f);
        mma_each(f, fv, w);
      } else {
        Frag f[NP];
        slice_frag(slice.gy, row, m, q, f);
        mma_each(f, fv, w);
      }
      if (owner) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i) slice_frag(slice.gvalue, i, m, q, fv[i]);
        mma_all(fv, fs, al);
        Frag fo[kTiles][NP];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) slice_frag(slice.gy, i, m, q, fo[i]);
        mma_all(fo, fs, aq);
      }
    }
    yv = group_sum(yv, 4);
    if (!second && (lane & 3) == 0) space.direct[st] = yv;
    // M1 or M2 (the tiles past the diagonal are not used)
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      if (j > row) continue;
      const int u = 16 * j + m;
      const float4 other = tb[u];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * row + 4 * q + r;
        const float4 me = tb[t];
        const float f = other.x * decay_between(me, other) * (second ? -me.x : a.scale * me.y);
        w[j][r] = t > u || (t == u && !second) ? w[j][r] * f : 0.f;
      }
    }
    // what the state gives, before the tokens' share: its part of q.Uq, k.UL, k.UR
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + 4 * q + r;
        const float4 tok = ta[t];
        float x = 0.f, y = 0.f, z = 0.f;
        if (owner) {
          const float ke = element(kbuf, t, own), qo = tok.w * aq[i][r], ko = -tok.y * al[i][r];
          const float kr = tok.z * ar[i][r];
          x = element(qbuf, t, own) * qo;
          y = ke * ko;
          z = ke * kr;
          totq[i][r] += qo;
          totk[i][r] += fmaf(tok.x, ko, kr);
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
    if (lane == 0) space.whole_dot[wave] = both;
    // the tokens' share, of the own row of tiles: sums over j up to a column, then over i behind
    // it; that of M2 times beta, as M2 is used from here on
    {
      v4f left{0.f, 0.f, 0.f, 0.f}, before{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        float column = 0.f;
        if (j <= row) {
          v4f p{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            Frag f[NP], fj[NP];
            rows_frag<NP, ST>(kbuf, j, kb, m, q, fj);
            rows_frag<NP, ST>(second ? kbuf : qbuf, row, kb, m, q, f);
            p = mma(f, fj, p);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = 16 * row + 4 * q + r;
            const float beta = second ? ta[t].x : 1.f;
            left[r] = fmaf(w[j][r], p[r], left[r]);
            w[j][r] *= beta;
            float x = t > 16 * j + m ? w[j][r] * p[r] : 0.f;
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
        if (q == 0) space.behind[wave][16 * j + m] = column;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = group_sum(left[r], 16);
        if (second && m == 0) space.dleft[16 * row + 4 * q + r] = x;
      }
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
      if (j > row) w[j] = v4f{0.f, 0.f, 0.f, 0.f};
    // Uq += M1 k, U += M1^T q + beta M2 k + (beta M2)^T k; of the tiles past the diagonal only the
    // neighbour of an even row's own is read
    const auto put = [&](Square& mat) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j)
        if (j <= row || (j == row + 1 && row % 2 == 0)) put_tile(mat, row, j, m, q, w[j]);
    };
    const auto add = [&](const Square& mat, v4f (&down)[kTiles], const bf16 (&other)[NP][kT * ST]) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        Frag fk[NP], fo[NP], f[3];
        columns_frag<NP, ST>(kbuf, wave, kb, m, q, fk);
        columns_frag<NP, ST>(other, wave, kb, m, q, fo);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          if (triangle_has<false>(i, kb)) {
            rows_frag<3, kMStride>(mat, i, kb, m, q, f);
            down[i] = mma(f, fk, down[i]);
          }
          if (triangle_has<true>(i, kb)) {
            columns_frag<3, kMStride>(mat, i, kb, m, q, f);
            totk[i] = mma(f, fo, totk[i]);
          }
        }
      }
    };
    __syncthreads();  // the slices have been read
    if (!second || Space::kSquares == 2) put(space.mat[second ? Space::kSquares - 1 : 0]);
    __syncthreads();  // M1 is there
    if (owner) add(space.mat[0], totq, qbuf);
    if (Space::kSquares == 1) {
      __syncthreads();
      if (second) put(space.mat[0]);
      __syncthreads();
    }
    if (owner) add(space.mat[Space::kSquares - 1], totk, kbuf);
    if (wave == 0) {
      const auto over = [&](const float (&x)[8][kT], int t) {
        return ((x[0][t] + x[1][t]) + (x[2][t] + x[3][t])) + ((x[4][t] + x[5][t]) + (x[6][t] + x[7][t]));
      };
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
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += space.whole_dot[i];
      const float s = whole * ss + from + (lane ? until + over(space.behind, lane - 1) : 0.f);
      if (lane < here) {
        const long long to = gate_at(lane, h);
        if (g.gdecay) g.gdecay[to] = lane < tokens ? s : 0.f;
        if (g.gbeta) g.gbeta[to] = lane < tokens ? left + space.dleft[lane] + space.direct[lane] : 0.f;
      }
    }
  }
  // through the norms of key and query, and out
  if (a.normalize) {
    __syncthreads();  // the last head's dots have been read
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + 4 * q + r;
        float x = 0.f, y = 0.f;
        if (owner) {
          x = element(qbuf, t, own) * totq[i][r];
          y = element(kbuf, t, own) * totk[i][r];
        }
        x = group_sum(x, 16);
        y = group_sum(y, 16);
        if (m == 0) {
          dots[0][wave][t] = x;
          dots[1][wave][t] = y;
        }
      }
    __syncthreads();
    if (tid < 2 * kT) {
      const int t = tid >> 1, k = tid & 1;
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) x += dots[k][i][t];
      const float f = k ? tb[t].x : tb[t].y;
      (k ? space.dleft : space.direct)[t] = f * f * x;
    }
    __syncthreads();
  }
  const auto results = [&](int i, int r, float& gqi, float& gki) {
    const int t = 16 * i + 4 * q + r;
    gqi = totq[i][r];
    gki = totk[i][r];
    if (a.normalize) {
      gqi = fmaf(-space.direct[t], element(qbuf, t, own), gqi);
      gki = fmaf(-space.dleft[t], element(kbuf, t, own), gki);
    }
    if (t >= tokens) gqi = gki = 0.f;
  };
  if constexpr (NP == 1) {
    // in the place of the keys and queries, from where whole rows go out, rather than in 2-byte
    // stores of a wave's 16 components
    if (owner) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = (16 * i + 4 * q + r) * ST + own;
          float x, y;
          results(i, r, x, y);
          qbuf[0][at] = (bf16)x;
          kbuf[0][at] = (bf16)y;
        }
    }
    __syncthreads();
    const auto store_raw = [](T* to, const bf16* from) {
      Raw<T, 8> piece;
      __builtin_memcpy(piece.w, __builtin_assume_aligned(from, 16), 16);
#pragma unroll
      for (int i = 0; i < Words<T, 8>::kWords; ++i) reinterpret_cast<typename Words<T, 8>::Unaligned*>(to)[i] = piece.w[i];
    };
    const auto out = [&](T* to, const bf16* from) {
      if (!to) return;
      if (D % 8 == 0) {
        const int pieces = D / 8;
        for (int i = tid; i < here * pieces; i += 512) {
          const int t = i / pieces, c = (i - t * pieces) * 8;
          store_raw(to + t * stride + c, from + t * ST + c);
        }
      } else {
        for (int i = tid; i < here * D; i += 512) {
          const int t = i / D, c = i - t * D;
          to[t * stride + c] = from[t * ST + c];
        }
      }
    };
    out(gq, qbuf[0]);
    out(gk, kbuf[0]);
  } else if (owner && own < D) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + 4 * q + r;
        float x, y;
        results(i, r, x, y);
        if (t >= here) continue;
        if (gq) gq[t * stride + own] = x;
        if (gk) gk[t * stride + own] = y;
      }
  }
}

template <class T, int KB>
hipError_t backward(const RuleBwdArgs& g, const RuleWs& w, hipStream_t s) {
  constexpr int kColumns = 16 * kWalkWaves;
  const auto walk = [&](auto kernel, int segments) {
    hipLaunchKernelGGL(kernel, dim3((w.VP + kColumns - 1) / kColumns, w.units, segments), dim3(64 * kWalkWaves), 0, s,
                       ReverseArgs{g, w});
    return hipGetLastError();
  };
  hipError_t e = hipSuccess;
  if (w.segments > 1) {
    e = walk(rule_reverse_kernel<T, KB, true>, w.segments - 1);
    if (e == hipSuccess) e = launch_rule_join(w, true, s);
    if (e != hipSuccess) return e;
  }
  e = walk(rule_reverse_kernel<T, KB, false>, w.segments);
  if (e != hipSuccess || !(g.gq || g.gk || g.gdecay || g.gbeta)) return e;
  const dim3 grid(w.chunks, g.a.n.B * g.a.n.Hk);
  if (g.a.n.C / g.a.n.H % 8 == 0)
    hipLaunchKernelGGL((rule_grads_kernel<T, KB, true>), grid, dim3(512), 0, s, g, w);
  else
    hipLaunchKernelGGL((rule_grads_kernel<T, KB, false>), grid, dim3(512), 0, s, g, w);
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
