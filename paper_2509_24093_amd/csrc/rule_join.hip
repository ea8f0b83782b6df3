// Gated delta rule: the states between the segments of a long sequence.  A segment of
// chunks takes the state S before it to M S + R, and the gradient of the state behind it to
// M^T gS + R'; M and R (or R') come from walks of all segments at once, and the segments are
// joined one after the other here: a product of D x D with D x V each.  The walk of the first
// segment begins with the given state, so its R is the state behind it and its M is not
// needed; nor is anything of the last segment.
#include <hip/hip_runtime.h>

#include "rule_common.h"
#include "rule_ws.h"

namespace cgconv {

namespace {

using namespace ruledev;

// Block (unit, tile of 16 columns; so those of a unit that is a multiple of 8 from the next one
// have their matrices in the same XCD's L2), wave w with the rows of tile w.  Bound by the latency of a
// step, of which nothing but the products and the exchange of the state's parts depends on the
// step before: the matrices come in parts, asked for two steps ahead.  16 segments of 128 x 128
// for 16 units 30 us, 2 us a step; 36 with a unit's blocks on all XCDs, 60 with the matrices in
// fp32 and split here.
template <int KB>
__global__ __launch_bounds__(128 * KB) void rule_join_kernel(const uint4* matrix, RuleWs ws, bool reverse) {
  constexpr int DT = 2 * KB, DP = 32 * KB;
  __shared__ uint2 S[2][3][DT][64];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int m = lane & 15, q = lane >> 4, row = 16 * wave + 4 * q;
  const int unit = blockIdx.x, col = blockIdx.y * 16 + m, steps = ws.segments;
  const auto segment = [&](int step) { return (long long)unit * steps + (reverse ? steps - 1 - step : step); };
  struct Next {
    Frag M[KB][3];
    v4f add;
  } next[2];
  const auto fetch = [&](int step, Next& to) {  // past the last one that is needed that one again
    const long long at = segment(max(min(step, steps - 2), 0));
    const uint4* p = matrix + (at * DT + wave) * (KB * 3 * 64) + lane;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 3; ++i) to.M[kb][i].all = p[64 * (3 * kb + i)];
#pragma unroll
    for (int r = 0; r < 4; ++r) to.add[r] = ws.span_state[(at * DP + row + r) * ws.VP + col];
  };
  v4f own;  // behind the first segment
#pragma unroll
  for (int r = 0; r < 4; ++r) own[r] = ws.span_state[(segment(0) * DP + row + r) * ws.VP + col];
  fetch(1, next[0]);
  fetch(2, next[1]);
  const auto once = [&](int step, Next& now, uint2 (&parts)[3][DT][64]) {
    const long long at = segment(step) * DP;
#pragma unroll
    for (int r = 0; r < 4; ++r) ws.start[(at + row + r) * ws.VP + col] = own[r];
    if (step + 1 == steps) return;
    uint2 p[3];
    split2(own[0], own[1], p[0].x, p[1].x, p[2].x);
    split2(own[2], own[3], p[0].y, p[1].y, p[2].y);
#pragma unroll
    for (int i = 0; i < 3; ++i) parts[i][wave][lane] = p[i];
    __syncthreads();
    v4f acc[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      Frag s[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        s[i].h[0] = parts[i][2 * kb][lane];
        s[i].h[1] = parts[i][2 * kb + 1][lane];
      }
      acc[kb] = mma(now.M[kb], s, v4f{0.f, 0.f, 0.f, 0.f});
    }
    own = now.add;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) own += acc[kb];
    fetch(step + 2, now);
  };
  for (int step = 1; step < steps; step += 2) {
    once(step, next[0], S[0]);
    if (step + 1 < steps) once(step + 1, next[1], S[1]);
  }
}

}  // namespace

hipError_t launch_rule_join(const RuleWs& w, bool reverse, hipStream_t s) {
  const dim3 grid(w.units, w.VP / 16);
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(128 * w.KB), 0, s, reverse ? w.span_matrixT : w.span_matrix, w,
                       reverse);
    return hipGetLastError();
  };
  switch (w.KB) {
    case 1: return run(rule_join_kernel<1>);
    case 2: return run(rule_join_kernel<2>);
    case 3: return run(rule_join_kernel<3>);
    default: return run(rule_join_kernel<4>);
  }
}

}  // namespace cgconv
