// Internal interface between the sequence plan (sequence.cpp) and its kernels:
// layer norm by degree (norm.hip), alone and around a residual connection
// (residual.hip), 8-bit checkpoints (pack.hip), the short causal convolution
// (conv.hip), the selective scan (scan.hip, scan_bwd.hip), the gated delta rule
// (delta_rule.hip, delta_rule_bwd.hip, rule_join.hip) and the clipping of gradients
// (clip.hip).  Features x, y are
// [B][N][K][C], channel fastest, in fp32 or bfloat16; parameters, states and
// statistics are fp32.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace cgconv {

// the message of cgconv_last_error(), shared by both translation units of the ABI
void set_last_error(const char* fmt, ...) __attribute__((format(printf, 1, 2)));
void clear_last_error();

enum SeqType : int { SEQ_F32 = 0, SEQ_BF16 = 1 };
// A launch counts its threads along an axis in 32 bits.  A launcher that would pass
// that returns hipErrorInvalidConfiguration (CGCONV_ERR_UNSUPPORTED to the caller).
inline bool launch_fits(long long blocks, int threads) {
  return blocks <= INT32_MAX && blocks * threads <= UINT32_MAX;
}

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
  float* part;            // norm_bwd_part_bytes, or nullptr if neither gw nor gb is wanted
  long long tokens;
  int L, K, C;
};

hipError_t launch_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormBwdArgs& a, hipStream_t s);
// bytes of NormBwdArgs::part
size_t norm_bwd_part_bytes(long long tokens, int L, int C);

// ---- norms around a residual connection -------------------------------------------

struct ResidualArgs {
  int type;
  const void* x;             // [tokens][K][C]
  const void* u;
  const void* gate;          // [tokens][C] or nullptr (ones in place of its silu)
  const float* post_weight;  // [L+1][C] or nullptr (ones)
  const float* scale;        // [C] or nullptr (ones)
  const float* weight;       // [L+1][C] or nullptr (ones)
  const float* bias;         // [C] or nullptr (zeros)
  float eps;
  void* r;
  void* y;
  float* stats;  // [tokens][2 (L+2)]: mean of u, its factors, mean of r, its factors; or nullptr
  long long tokens;
  int L, K, C;
};
struct ResidualBwdArgs {
  ResidualArgs a;  // r, y, bias and eps unused
  const void* gr;  // or nullptr (zeros)
  const void* gy;
  void* gx;        // any may be nullptr
  void* gu;
  void* ggate;
  float* gpost;
  float* gscale;
  float* gw;
  float* gb;
  float* part;  // residual_part_bytes, or nullptr if no parameter's gradient is wanted
};
hipError_t launch_residual(const ResidualArgs& a, hipStream_t s);
hipError_t launch_residual_backward(const ResidualBwdArgs& g, hipStream_t s);
size_t residual_part_bytes(long long tokens, int L, int C);

// ---- 8-bit checkpoints ---------------------------------------------------------

hipError_t launch_pack(int type, const void* x, int8_t* codes, uint8_t* scales, long long rows, int C, hipStream_t s);
hipError_t launch_unpack(int type, const int8_t* codes, const uint8_t* scales, void* x, long long rows, int C,
                         hipStream_t s);

// ---- short causal convolution --------------------------------------------------

constexpr int kConvMaxWidth = 8;
struct ConvArgs {
  int type;
  const void* x;        // [B][N][K][C] (a step: [B][K][C])
  const float* weight;  // [W][L+1][C]
  const float* bias;    // [C] or nullptr
  const int* lengths;   // [B] or nullptr
  const void* state_in;  // [B][W-1][K][C] or nullptr (zeros)
  void* y;
  void* state_out;       // or nullptr; a step's state, in place
  int B, N, L, K, C, W;
  int activation;
};
struct ConvBwdArgs {
  ConvArgs a;  // y and the states unused
  const void* gy;
  void* gx;    // or nullptr
  float* gw;   // [W][L+1][C] or nullptr
  float* gb;   // [C] or nullptr
  float* part;  // conv_bwd_part_bytes, or nullptr if neither gw nor gb is wanted
};
hipError_t launch_conv(const ConvArgs& a, hipStream_t s);
hipError_t launch_conv_step(const ConvArgs& a, hipStream_t s);
hipError_t launch_conv_backward(const ConvBwdArgs& g, hipStream_t s);
size_t conv_bwd_part_bytes(int64_t B, int64_t N, int K, int64_t C);

// ---- selective scan --------------------------------------------------------------

struct ScanArgs {
  int type;
  const void* x;      // [B][N][K][C] (a step: [B][K][C])
  const void* delta;  // [B][N][C]
  const float* A;     // [C][S]
  const void* Bt;     // [B][N][S]
  const void* Ct;
  const float* D;     // [C] or nullptr
  const float* bias;  // [C] or nullptr
  const int* lengths;  // [B] or nullptr
  const float* state_in;  // [B][S][K][C] or nullptr (zeros)
  void* y;
  float* state_out;  // or nullptr; a step's state, in place
  int B, N, K, C, S;
  float* ws;  // scan_workspace_bytes
};
struct ScanBwdArgs {
  ScanArgs a;  // y and the states unused
  const void* gy;
  void* gx;      // the gradients, in the inputs' types (fp32 for A, D, bias);
  void* gdelta;  // any may be nullptr
  float* gA;
  void* gB;
  void* gC;
  float* gD;
  float* gbias;
};
hipError_t launch_scan(const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_step(const ScanArgs& a, hipStream_t s);
hipError_t launch_scan_backward(const ScanBwdArgs& g, hipStream_t s);
// workspace of both directions
size_t scan_workspace_bytes(int64_t B, int64_t N, int K, int64_t C, int S);

// ---- clipping by the global norm ------------------------------------------------------

struct ClipArgs {
  long long n;             // tensors; the arrays are the host's
  const int32_t* types;
  const int64_t* counts;
  const void* const* grads;
  void* const* out;        // each its gradient's own address, or an array of its own
  float max_norm, eps;
  float* norm;
  double* ws;  // clip_workspace_bytes
};
hipError_t launch_clip(const ClipArgs& a, hipStream_t s);
size_t clip_workspace_bytes(long long n, const int64_t* counts);

// ---- gated delta rule ---------------------------------------------------------------

constexpr int kRuleMaxDim = 128;   // key width
constexpr float kRuleNormEps = 1e-6f;  // under the root of a key's norm
constexpr int kRuleChunk = 64;     // tokens whose products are formed at once
constexpr int kRuleTriangle = 10;  // 16 x 16 blocks on and below the diagonal of a chunk

struct RuleSizes {
  int B, N, K, C;  // C = H P: P channels of every component a head
  int H, Hk, D;    // heads, key heads (Hk divides H), key width
};
struct RuleArgs {
  int type;
  RuleSizes n;
  const void* q;       // [B][N][Hk][D] (a step: [B][Hk][D])
  const void* k;
  const void* v;       // [B][N][K][C]
  const float* decay;  // [B][N][H], logarithms
  const float* beta;   // [B][N][H]
  const int* lengths;  // [B] or nullptr
  const float* state_in;  // [B][D][K][C] or nullptr (zeros)
  void* y;
  float* state_out;  // or nullptr; a step's state, in place
  float scale;
  int normalize;
  char* ws;  // rule_workspace_bytes
};
struct RuleBwdArgs {
  RuleArgs a;  // y and state_out unused
  const void* gy;
  const float* gstate;  // [B][D][K][C] or nullptr (zeros)
  void* gq;             // any may be nullptr
  void* gk;
  void* gv;
  float* gdecay;
  float* gbeta;
  float* gstate_in;
};
hipError_t launch_rule(const RuleArgs& a, hipStream_t s);
hipError_t launch_rule_step(const RuleArgs& a, hipStream_t s);
hipError_t launch_rule_backward(const RuleBwdArgs& g, hipStream_t s);
size_t rule_workspace_bytes(const RuleSizes& n, bool backward);

}  // namespace cgconv
