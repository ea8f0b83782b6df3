// Activation checkpoints in 8 bits (format: seq_common.h): rows of C channels
// of any tensor to int8 codes and one power-of-two scale byte per 32 channels,
// and back.  Both directions are streams, bound by HBM.  A tensor larger than the
// chip's caches (kPackNtBytes) is read and written with nontemporal accesses: it
// leaves the caches before anybody reads it again (410 MB of bf16 there and back
// 216 -> 192 us; 57 MB, which stay cached between the two, would go 28.5 -> 30).
#include <hip/hip_runtime.h>

#include "seq_common.h"

namespace cgconv {

namespace {

using namespace seqdev;

constexpr int kThreads = 256;
constexpr long long kPackNtBytes = 256LL << 20;

// A thread takes 16 bytes of x: the 32 / V lanes of a scale's channels are
// neighbours, and a row's last group leaves lanes idle.  TAIL: C is no multiple of
// V, so rows start anywhere and end inside a vector.
template <class T, int V, bool PACK, bool NT, bool TAIL>
__global__ __launch_bounds__(kThreads) void pack_kernel(const T* __restrict__ x, const int8_t* __restrict__ codes_in,
                                                        const uint8_t* __restrict__ scales_in, T* __restrict__ out,
                                                        int8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                        long long groups, int C, int nb) {
  constexpr int kLanes = kPackBlock / V;
  const long long thread = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long g = thread / kLanes;
  if (g >= groups) return;
  const int j = (int)(thread % kLanes);
  const long long row = g / nb;
  const int c = (int)(g - row * nb) * kPackBlock + j * V;
  const int n = C - c;
  const bool here = n > 0;
  const long long at = row * C + c;
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.f;
  if (PACK) {
    if (here) load_part<TAIL, NT>(x + at, n, v);
    const uint32_t scale = pack_scale(group_max_bits(max_bits(v), kLanes));
    if (here) store_codes<TAIL>(codes + at, n, v, scale);
    if (j == 0) scales[g] = (uint8_t)scale;
  } else if (here) {
    load_codes<TAIL>(codes_in + at, n, scales_in[g], v);
    store_part<TAIL, NT>(out + at, n, v);
  }
}

template <class T, int V, bool PACK>
hipError_t launch(const void* x, int8_t* codes, uint8_t* scales, void* out, long long rows, int C, hipStream_t s) {
  const int nb = (int)pack_blocks(C);
  const long long groups = rows * nb;
  const long long blocks = (groups * (kPackBlock / V) + kThreads - 1) / kThreads;
  if (!launch_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  const auto run = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, static_cast<const T*>(x), codes, scales,
                       static_cast<T*>(out), codes, scales, groups, C, nb);
    return hipGetLastError();
  };
  const bool nt = rows * C * (long long)sizeof(T) > kPackNtBytes;
  if (C % V) return nt ? run(pack_kernel<T, V, PACK, true, true>) : run(pack_kernel<T, V, PACK, false, true>);
  return nt ? run(pack_kernel<T, V, PACK, true, false>) : run(pack_kernel<T, V, PACK, false, false>);
}

template <bool PACK>
hipError_t launch_any(int type, const void* x, int8_t* codes, uint8_t* scales, void* out, long long rows, int C,
                      hipStream_t s) {
  return type == SEQ_BF16 ? launch<bf16, 8, PACK>(x, codes, scales, out, rows, C, s)
                          : launch<float, 4, PACK>(x, codes, scales, out, rows, C, s);
}

}  // namespace

hipError_t launch_pack(int type, const void* x, int8_t* codes, uint8_t* scales, long long rows, int C, hipStream_t s) {
  return launch_any<true>(type, x, codes, scales, nullptr, rows, C, s);
}

hipError_t launch_unpack(int type, const int8_t* codes, const uint8_t* scales, void* x, long long rows, int C,
                         hipStream_t s) {
  return launch_any<false>(type, nullptr, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), x, rows, C, s);
}

}  // namespace cgconv
