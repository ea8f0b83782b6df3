// Gated delta rule: the states between the segments of a long sequence.  A segment of
// chunks takes the state S before it to M S + R, and the gradient of the state behind it to
// M^T gS + R'; M and R (or R') come from walks of all segments at once, and the segments are
// joined one after the other here: a product of D x D with D x V each.
#include <hip/hip_runtime.h>

#include "rule_common.h"
#include "rule_ws.h"

namespace cgconv {

namespace {

using namespace ruledev;

// Block (tile of 16 columns, unit); wave w has the rows of the tiles w, w + 4.  The next
// segment's matrix is asked for before the state is exchanged.
template <int KB, bool REVERSE>
__global__ __launch_bounds__(256) void rule_join_kernel(const float* first, RuleWs ws, RuleSizes n) {
  constexpr int DT = 2 * KB, NT = (DT + 3) / 4, DP = 32 * KB;
  __shared__ v4f S[DT][64];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int m = lane & 15, q = lane >> 4;
  const int unit = blockIdx.y, b = unit / n.H, h = unit - b * n.H, col = blockIdx.x * 16 + m;
  const Column column(col, ws.V, n.C / n.H, n.C, h);
  const long long KC = (long long)n.K * n.C;
  v4f own[NT];
  float M[NT][KB][8];
  const auto tile = [&](int i) { return wave + 4 * i; };
  const auto matrix = [&](int seg) {
    const float* p = ws.span_matrix + ((long long)unit * ws.segments + seg) * DP * DP;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (tile(i) >= DT) continue;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int row = 16 * tile(i) + m, k = 32 * kb + 4 * q + (e & 3) + (e & 4) * 4;
          M[i][kb][e] = REVERSE ? p[row * DP + k] : p[k * DP + row];
        }
    }
  };
  const int from = REVERSE ? ws.segments - 1 : 0, by = REVERSE ? -1 : 1;
  matrix(from);
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * tile(i) + 4 * q + r;
      own[i][r] = first && column.there && row < n.D ? first[((long long)b * n.D + row) * KC + column.at] : 0.f;
    }
  for (int step = 0; step < ws.segments; ++step) {
    const int seg = from + by * step;
    const long long at = ((long long)unit * ws.segments + seg) * DP;
    v4f add[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      if (tile(i) >= DT) continue;
      S[tile(i)][lane] = own[i];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const long long to = (at + 16 * tile(i) + 4 * q + r) * ws.VP + col;
        ws.start[to] = own[i][r];
        add[i][r] = ws.span_state[to];
      }
    }
    if (step + 1 == ws.segments) break;
    Frag f[NT][KB][3];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) split8(M[i][kb], f[i][kb]);
    if (step + 2 < ws.segments) matrix(seg + by);
    __syncthreads();
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      Frag s[3];
      split_tiles(S[2 * kb][lane], S[2 * kb + 1][lane], s);
#pragma unroll
      for (int i = 0; i < NT; ++i)
        if (tile(i) < DT) add[i] = mma(f[i][kb], s, add[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) own[i] = add[i];
  }
}

}  // namespace

hipError_t launch_rule_join(const float* first, const RuleWs& w, const RuleSizes& n, bool reverse, hipStream_t s) {
  const dim3 grid(w.VP / 16, w.units);
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, first, w, n);
    return hipGetLastError();
  };
  switch (w.KB) {
    case 1: return reverse ? run(rule_join_kernel<1, true>) : run(rule_join_kernel<1, false>);
    case 2: return reverse ? run(rule_join_kernel<2, true>) : run(rule_join_kernel<2, false>);
    case 3: return reverse ? run(rule_join_kernel<3, true>) : run(rule_join_kernel<3, false>);
    default: return reverse ? run(rule_join_kernel<4, true>) : run(rule_join_kernel<4, false>);
  }
}

}  // namespace cgconv
