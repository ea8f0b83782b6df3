// Device side shared by the selective scan's forward (scan.hip) and backward
// (scan_bwd.hip).
//
//   delta = softplus(raw[t,c] + bias[c])
//   h_t[s,k,c] = exp(delta A[c,s]) h_{t-1}[s,k,c] + delta B_t[s] x_t[k,c]
//   y_t[k,c] = sum_s C_t[s] h_t[s,k,c] + D[c] x_t[k,c]
//
// Lanes are channels (of one or several components), so B_t and C_t are the
// same for a whole wave: a preparing kernel writes them as fp32 rows of SP
// states each (SP = S rounded up as each direction takes it, zeros behind S), and the scans read them
// through the scalar cache as scalar operands, a token ahead of their use.  The
// states stay in registers.
#pragma once

#include "seq_common.h"

namespace cgconv {
namespace seqdev {

typedef const __attribute__((address_space(4))) float* ConstFloats;

constexpr float kLog2e = 1.44269504088896340736f;

// exp(v) as 2^(v log2 e) of the hardware.  a is pre-scaled by log2 e.
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|) in (0, 1]; log1p(e) = 2
// atanh(u), u = e / (2 + e) <= 1/3, by its series in u^2 <= 1/9: the terms
// left out, from u^17 2/17 on, are below 2^-29 of the sum.
__device__ __forceinline__ float softplus(float v) {
  const float e = exp2_fast(-fabsf(v) * kLog2e);
  const float u = e * __builtin_amdgcn_rcpf(2.f + e), q = u * u;
  float p = 2.f / 15.f;
  p = fmaf(p, q, 2.f / 13.f);
  p = fmaf(p, q, 2.f / 11.f);
  p = fmaf(p, q, 2.f / 9.f);
  p = fmaf(p, q, 2.f / 7.f);
  p = fmaf(p, q, 2.f / 5.f);
  p = fmaf(p, q, 2.f / 3.f);
  p = fmaf(p, q, 2.f);
  return fmaxf(v, 0.f) + p * u;
}

__device__ __forceinline__ int scan_length(const int* lengths, int b, int N) {
  return lengths ? min(max(lengths[b], 0), N) : N;
}

// B_t (v[0..SP)) and C_t (v[SP..2SP)) of one token, in scalar registers.
template <int SP>
struct TokenRow {
  float v[2 * SP];
  __device__ __forceinline__ void load(ConstFloats p) {
#pragma unroll
    for (int s = 0; s < 2 * SP; ++s) v[s] = p[s];
  }
};

// The rows of consecutive tokens: at(t) gives token t's, asked for a token ahead
// where two rows fit the scalar registers.  Scalar loads return in any order, so
// a wait is for all of them: the next row is asked for behind the wait for this
// one, or this one's first use would wait for both; and the scheduler would move
// the request to the row's use.
template <int SP>
struct TokenRows {
  static constexpr bool kAhead = SP <= 16;
  TokenRow<SP> row, next;
  ConstFloats base;
  __device__ __forceinline__ void begin(ConstFloats p, int t) {
    base = p;
    if (kAhead) next.load(base + (long long)t * 2 * SP);
  }
  __device__ __forceinline__ const float* at(int t, int following) {
    if (kAhead) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
      __builtin_amdgcn_sched_barrier(0);
      row = next;
      next.load(base + (long long)following * 2 * SP);
      __builtin_amdgcn_sched_barrier(0);
    } else {
      row.load(base + (long long)t * 2 * SP);
    }
    return row.v;
  }
};

// Brings the rows of tokens t0 .. t2 - 1, at most 64, into the caches near this
// block: where only one or two blocks share them, a scalar load of every token
// would otherwise wait for memory on its own (2 x 8192 tokens of 49 x 32, forward:
// 218 -> 209 us; 4 x 8192 of 2048, 8 blocks a chunk, 346 -> 353).  Returns a value
// for settle_rows, behind the block's other first loads.
template <int SP>
__device__ __forceinline__ float touch_rows(const float* rows, int t0, int t2) {
  constexpr int kLine = 32;  // floats of a cache line
  const int n = min(t2 - t0, 64) * 2 * SP;
  const float* p = rows + (long long)t0 * 2 * SP;
  float v = 0.f;
  for (int i = threadIdx.x * kLine; i < n; i += blockDim.x * kLine) v += p[i];
  return v;
}
__device__ __forceinline__ void settle_rows(float v) { asm volatile("" ::"v"(v)); }

template <class T>
__device__ __forceinline__ float load1(const void* p, long long i) {
  return widen(static_cast<const T*>(p)[i]);
}

}  // namespace seqdev

constexpr int kScanThreads = 256;

// Tokens in chunks; a chunk's states at its start are [B][chunks][S][K C].
struct ScanChunks {
  int chunk, chunks;
};
// States of the backward's rows and registers: groups of eight, one, two or four of
// them (rows of 4, 12 and 24 took as long or longer, forward and backward of 4 x 2048 x
// 1024 bf16: S 4 181 and 181 us, 12 282 and 321, 24 535 and 521; 4 x 1024 of 16 x 64
// fp32: 24 326 and 333).
inline int scan_padded(int S) { return S <= 8 ? 8 : S <= 16 ? 16 : 32; }

// Workspace: parts of one allocation, 256-byte aligned.
struct ScanSpace {
  float* bc = nullptr;   // [B][N][2 SP]: B_t, C_t
  float* A2 = nullptr;   // [SP][C]: A log2 e
  float* hs = nullptr;   // [B][chunks][S][K C]: states at the chunks' ends, then starts
  float* ds = nullptr;   // [B][chunks][C]: sum of delta over a chunk
  // backward
  float* rs = nullptr;   // [B][chunks][S][K C]: gradients of the states behind a chunk
  float* gbc = nullptr;  // [column blocks][B][N][2 SP]: of B_t, C_t
  float* gd = nullptr;   // [B][N][K][C]: the components' parts of delta's (K > 1)
  float* ga = nullptr;   // [B][chunks][S + 2][K C]: of A, D and (K = 1) the bias over a chunk
  float* gbp = nullptr;  // [token blocks][C]: of the bias (K > 1)
  size_t bytes = 0;
  void place(void* base, float** p, size_t floats) {
    *p = reinterpret_cast<float*>(static_cast<char*>(base) + bytes);
    bytes += (floats * sizeof(float) + 255) / 256 * 256;
  }
};

size_t scan_forward_bytes(int64_t B, int64_t N, int K, int64_t C, int S);
size_t scan_backward_bytes(int64_t B, int64_t N, int K, int64_t C, int S);

// bc and A2 for rows of SP states
hipError_t launch_scan_prepare(const ScanArgs& a, const ScanSpace& w, int SP, hipStream_t s);
// hs: what the chunks add to what they start with; rs (or nullptr) likewise, in reverse
hipError_t launch_scan_carry(const ScanArgs& a, const ScanChunks& ch, const ScanSpace& w, const float* first, bool reverse,
                             hipStream_t s);

}  // namespace cgconv
