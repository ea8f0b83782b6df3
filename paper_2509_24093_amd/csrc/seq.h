// Internal interface between the sequence plan (sequence.cpp) and its kernels:
// layer norm by degree (norm.hip), 8-bit checkpoints (pack.hip), the short
// causal convolution (conv.hip) and the selective scan (scan.hip,
// scan_bwd.hip).  Features x, y are [B][N][K][C], channel fastest, in fp32 or
// bfloat16; parameters, states and statistics are fp32.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace cgconv {

// the message of cgconv_last_error(), shared by both translation units of the ABI
void set_last_error(const char* fmt, ...) __attribute__((format(printf, 1, 2)));
void clear_last_error();

enum SeqType : int { SEQ_F32 = 0, SEQ_BF16 = 1 };
inline int64_t seq_type_size(int type) { return type == SEQ_BF16 ? 2 : 4; }

// Channels that share one scale of an 8-bit checkpoint.
constexpr int kPackBlock = 32;
inline int64_t pack_blocks(int64_t C) { return (C + kPackBlock - 1) / kPackBlock; }

// ---- layer norm by degree ------------------------------------------------------

struct NormArgs {
  int type;
  const void* x;
  const float* weight;  // [L+1][C] or nullptr (ones)
  const float* bias;    // [C] or nullptr (zeros)
  float eps;
  void* y;
  float* mean;      // [tokens] or nullptr
  float* rstd;      // [tokens][L+1] or nullptr
  int8_t* codes;    // [tokens][K][C] or nullptr: the checkpoint of x
  uint8_t* scales;  // [tokens][K][pack_blocks(C)]
  long long tokens;
  int L, K, C;
};

struct NormBwdArgs {
  int type;
  const void* x;          // or nullptr: codes and scales hold it
  const int8_t* codes;
  const uint8_t* scales;
  const float* weight;    // or nullptr
  const float* mean;
  const float* rstd;
  const void* gy;
  void* gx;               // or nullptr
  float* gw;              // [L+1][C] or nullptr
  float* gb;              // [C] or nullptr
  float* part;            // norm_bwd_blocks(...) * (K + 1) * C floats
  long long tokens;
  int L, K, C;
};

// Longest (2L+1) C: one block holds the largest degree of a token.
constexpr int kNormMaxSegment = 16384;

hipError_t launch_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormBwdArgs& a, hipStream_t s);
// bytes of NormBwdArgs::part
size_t norm_bwd_part_bytes(long long tokens, int L, int C);

// ---- 8-bit checkpoints ---------------------------------------------------------

hipError_t launch_pack(int type, const void* x, int8_t* codes, uint8_t* scales, long long rows, int C, hipStream_t s);
hipError_t launch_unpack(int type, const int8_t* codes, const uint8_t* scales, void* x, long long rows, int C,
                         hipStream_t s);

}  // namespace cgconv
