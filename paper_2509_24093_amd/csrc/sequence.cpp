// Sequence plan and the entry points of the operators around the convolution
// (see include/cgconv.h, "Sequence operators"): checks of arguments, the
// plan's workspace, launches.  Kernels: norm.hip, residual.hip, pack.hip, conv.hip,
// scan.hip, scan_bwd.hip, delta_rule.hip, delta_rule_bwd.hip, rule_join.hip,
// clip.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>
#include <vector>

#include "cgconv.h"
#include "seq.h"

using namespace cgconv;

struct cgconv_seq_plan {
  int64_t B = 0, N = 0, C = 0;
  int L = 0, K = 0, S = 0;
  int H = 0, Hk = 0, D = 0;     // the delta rule's heads, key heads and key width; H = 0: none
  bool rule_backward = false;   // its backward's workspace is there
  int device = 0;
  size_t ws_bytes = 0;
  void* ws = nullptr;
};

namespace {

// A device array of a call: its name, whether the call needs it and whether it
// is written.
struct Arg {
  const char* name;
  const void* ptr;
  size_t bytes;
  bool needed, written;
};

// Presence, alignment (of `align` bytes) and overlap: what a call writes shares
// no byte with any other array of the call.
int check_arrays(const Arg* args, int n, unsigned align = 16) {
  for (int i = 0; i < n; ++i) {
    if (args[i].needed && !args[i].ptr) {
      set_last_error("%s must be a non-NULL device pointer", args[i].name);
      return CGCONV_ERR_INVALID_ARG;
    }
  }
  for (int i = 0; i < n; ++i) {
    if (args[i].ptr && (reinterpret_cast<uintptr_t>(args[i].ptr) & (align - 1)) != 0) {
      set_last_error("%s must be %u-byte aligned", args[i].name, align);
      return CGCONV_ERR_ALIGNMENT;
    }
  }
  for (int i = 0; i < n; ++i) {
    if (!args[i].ptr || !args[i].written) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(args[i].ptr);
    for (int j = 0; j < n; ++j) {
      if (j == i || !args[j].ptr) continue;
      const uintptr_t b = reinterpret_cast<uintptr_t>(args[j].ptr);
      if (a < b + args[j].bytes && b < a + args[i].bytes) {
        set_last_error("%s must not overlap %s", args[i].name, args[j].name);
        return CGCONV_ERR_INVALID_ARG;
      }
    }
  }
  return CGCONV_OK;
}

int check_type(int32_t dtype) {
  if (dtype != CGCONV_F32 && dtype != CGCONV_BF16) {
    set_last_error("dtype=%d is neither CGCONV_F32 nor CGCONV_BF16", dtype);
    return CGCONV_ERR_INVALID_ARG;
  }
  return CGCONV_OK;
}

int check_plan(const cgconv_seq_plan* p, int32_t dtype) {
  if (!p) {
    set_last_error("plan is NULL");
    return CGCONV_ERR_INVALID_ARG;
  }
  const int st = check_type(dtype);
  if (st != CGCONV_OK) return st;
  int cur = -1;
  if (hipGetDevice(&cur) != hipSuccess || cur != p->device) {
    set_last_error("the plan's device (%d) is not current (%d)", p->device, cur);
    return CGCONV_ERR_INVALID_ARG;
  }
  return CGCONV_OK;
}

int launched(hipError_t e) {
  if (e == hipSuccess) return CGCONV_OK;
  if (e == hipErrorInvalidConfiguration) {
    set_last_error("unsupported sizes: more threads than one launch takes");
    return CGCONV_ERR_UNSUPPORTED;
  }
  set_last_error("kernel launch failed: %s", hipGetErrorString(e));
  return CGCONV_ERR_HIP;
}

RuleSizes rule_sizes(const cgconv_seq_plan* p) {
  return {(int)p->B, (int)p->N, p->K, (int)p->C, p->H, p->Hk, p->D};
}

cgconv_seq_plan* create_plan(int64_t batch, int64_t N, int32_t L_max, int64_t C, int32_t states, int32_t heads,
                             int32_t key_heads, int32_t key_dim, bool rule_backward) {
  clear_last_error();
  if (batch < 1 || batch > 65535 || N < 1 || C < 1 || states < 0) {
    set_last_error("invalid sizes: batch=%lld N=%lld C=%lld states=%d (need 1 <= batch <= 65535, N >= 1, C >= 1, "
                   "states >= 0)", (long long)batch, (long long)N, (long long)C, states);
    return nullptr;
  }
  if (L_max < 0 || L_max > CGCONV_LMAX) {
    set_last_error("unsupported L_max=%d: 0..%d", L_max, CGCONV_LMAX);
    return nullptr;
  }
  if (states > CGCONV_SEQ_STATES) {
    set_last_error("unsupported states=%d: at most %d", states, CGCONV_SEQ_STATES);
    return nullptr;
  }
  const int K = (L_max + 1) * (L_max + 1);
  if ((int64_t)(2 * L_max + 1) * C > CGCONV_SEQ_SEGMENT) {
    set_last_error("unsupported C=%lld at L_max=%d: (2 L_max + 1) C at most %d", (long long)C, L_max,
                   CGCONV_SEQ_SEGMENT);
    return nullptr;
  }
  if (N > CGCONV_SEQ_TOKENS / batch) {
    set_last_error("unsupported batch*N: at most %lld tokens", (long long)CGCONV_SEQ_TOKENS);
    return nullptr;
  }
  if ((int64_t)batch * N > CGCONV_SEQ_VALUES / (K * C)) {
    set_last_error("unsupported batch*N*K*C: at most %lld values", (long long)CGCONV_SEQ_VALUES);
    return nullptr;
  }
  cgconv_seq_plan* p = new (std::nothrow) cgconv_seq_plan;
  if (!p) {
    set_last_error("host allocation failed");
    return nullptr;
  }
  p->B = batch;
  p->N = N;
  p->C = C;
  p->L = L_max;
  p->K = K;
  p->S = states;
  p->H = heads;
  p->Hk = key_heads;
  p->D = key_dim;
  p->rule_backward = rule_backward;
  hipError_t e = hipGetDevice(&p->device);
  if (e != hipSuccess) {
    set_last_error("hipGetDevice failed: %s", hipGetErrorString(e));
    delete p;
    return nullptr;
  }
  p->ws_bytes = std::max(norm_bwd_part_bytes(batch * N, L_max, (int)C), conv_bwd_part_bytes(batch, N, K, C));
  p->ws_bytes = std::max(p->ws_bytes, residual_part_bytes(batch * N, L_max, (int)C));
  if (states) p->ws_bytes = std::max(p->ws_bytes, scan_workspace_bytes(batch, N, K, C, states));
  if (heads) p->ws_bytes = std::max(p->ws_bytes, rule_workspace_bytes(rule_sizes(p), rule_backward));
  if ((e = hipMalloc(&p->ws, p->ws_bytes)) != hipSuccess) {
    set_last_error("workspace allocation of %zu bytes failed: %s", p->ws_bytes, hipGetErrorString(e));
    (void)hipGetLastError();
    delete p;
    return nullptr;
  }
  return p;
}

}  // namespace

extern "C" {

cgconv_seq_plan_t cgconv_seq_plan_create(int64_t batch, int64_t N, int32_t L_max, int64_t C, int32_t states) {
  return create_plan(batch, N, L_max, C, states, 0, 0, 0, false);
}

cgconv_seq_plan_t cgconv_seq_plan_create_rule(int64_t batch, int64_t N, int32_t L_max, int64_t C, int32_t states,
                                              int32_t heads, int32_t key_heads, int32_t key_dim, int32_t backward) {
  clear_last_error();
  if (heads < 1 || key_heads < 1 || key_dim < 1) {
    set_last_error("invalid sizes: heads=%d key_heads=%d key_dim=%d (need at least 1 each)", heads, key_heads, key_dim);
    return nullptr;
  }
  if (C % heads != 0 || heads % key_heads != 0) {
    set_last_error("invalid sizes: C=%lld must be a multiple of heads=%d, heads a multiple of key_heads=%d",
                   (long long)C, heads, key_heads);
    return nullptr;
  }
  if (key_dim > CGCONV_SEQ_KEY_DIM) {
    set_last_error("unsupported key_dim=%d: at most %d", key_dim, CGCONV_SEQ_KEY_DIM);
    return nullptr;
  }
  if (batch >= 1 && batch > 65535 / heads) {
    set_last_error("unsupported batch*heads: at most 65535");
    return nullptr;
  }
  return create_plan(batch, N, L_max, C, states, heads, key_heads, key_dim, backward != 0);
}

void cgconv_seq_plan_destroy(cgconv_seq_plan_t plan) {
  if (!plan) return;
  int cur = 0;
  (void)hipGetDevice(&cur);
  (void)hipSetDevice(plan->device);
  (void)hipFree(plan->ws);
  (void)hipSetDevice(cur);
  delete plan;
}

int cgconv_seq_plan_info(cgconv_seq_plan_t plan, size_t* workspace_bytes) {
  if (!plan) {
    set_last_error("plan is NULL");
    return CGCONV_ERR_INVALID_ARG;
  }
  if (workspace_bytes) *workspace_bytes = plan->ws_bytes;
  return CGCONV_OK;
}

int cgconv_seq_norm(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const float* weight, const float* bias,
                    float eps, void* y, float* mean, float* rstd, int8_t* codes, uint8_t* scales,
                    hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  if (!(eps >= 0.f)) {
    set_last_error("eps=%g must be >= 0", (double)eps);
    return CGCONV_ERR_INVALID_ARG;
  }
  if (!mean != !rstd || !codes != !scales) {
    set_last_error("mean and rstd, and codes and scales, are given together or not at all");
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t tokens = plan->B * plan->N, n = tokens * plan->K * plan->C;
  const Arg args[] = {{"x", x, n * seq_type_size(dtype), true, false},
                      {"weight", weight, (plan->L + 1) * (size_t)plan->C * 4, false, false},
                      {"bias", bias, (size_t)plan->C * 4, false, false},
                      {"y", y, n * seq_type_size(dtype), true, true},
                      {"mean", mean, tokens * 4, false, true},
                      {"rstd", rstd, tokens * (plan->L + 1) * 4, false, true},
                      {"codes", codes, n, false, true},
                      {"scales", scales, tokens * plan->K * pack_blocks(plan->C), false, true}};
  if ((st = check_arrays(args, 8)) != CGCONV_OK) return st;
  NormArgs a{dtype, x, weight, bias, eps, y, mean, rstd, codes, scales, (long long)tokens, plan->L, plan->K,
             (int)plan->C};
  return launched(launch_norm(a, stream));
}

int cgconv_seq_norm_backward(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const int8_t* codes,
                             const uint8_t* scales, const float* weight, const float* mean, const float* rstd,
                             const void* grad_y, void* grad_x, float* grad_weight, float* grad_bias,
                             hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  if (!codes != !scales || !x == !codes) {
    set_last_error("either x or both codes and scales must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  if (!grad_x && !grad_weight && !grad_bias) {
    set_last_error("at least one of grad_x, grad_weight and grad_bias must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t tokens = plan->B * plan->N, n = tokens * plan->K * plan->C;
  const size_t nw = (plan->L + 1) * (size_t)plan->C * 4;
  const Arg args[] = {{"x", x, n * seq_type_size(dtype), false, false},
                      {"codes", codes, n, false, false},
                      {"scales", scales, tokens * plan->K * pack_blocks(plan->C), false, false},
                      {"weight", weight, nw, false, false},
                      {"mean", mean, tokens * 4, true, false},
                      {"rstd", rstd, tokens * (plan->L + 1) * 4, true, false},
                      {"grad_y", grad_y, n * seq_type_size(dtype), true, false},
                      {"grad_x", grad_x, n * seq_type_size(dtype), false, true},
                      {"grad_weight", grad_weight, nw, false, true},
                      {"grad_bias", grad_bias, (size_t)plan->C * 4, false, true}};
  if ((st = check_arrays(args, 10)) != CGCONV_OK) return st;
  NormBwdArgs a{dtype, x, codes, scales, weight, mean, rstd, grad_y, grad_x, grad_weight, grad_bias,
                grad_weight || grad_bias ? static_cast<float*>(plan->ws) : nullptr, (long long)tokens, plan->L,
                plan->K, (int)plan->C};
  return launched(launch_norm_backward(a, stream));
}

int cgconv_seq_residual_norm(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const void* u, const void* gate,
                             const float* post_weight, const float* scale, const float* weight, const float* bias,
                             float eps, void* r, void* y, float* stats, hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  if (!(eps >= 0.f)) {
    set_last_error("eps=%g must be >= 0", (double)eps);
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t tokens = plan->B * plan->N, C = plan->C, n = tokens * plan->K * C * seq_type_size(dtype);
  const size_t nw = (plan->L + 1) * C * 4;
  const Arg args[] = {{"x", x, n, true, false},
                      {"u", u, n, true, false},
                      {"gate", gate, tokens * C * seq_type_size(dtype), false, false},
                      {"post_weight", post_weight, nw, false, false},
                      {"scale", scale, C * 4, false, false},
                      {"weight", weight, nw, false, false},
                      {"bias", bias, C * 4, false, false},
                      {"r", r, n, true, true},
                      {"y", y, n, true, true},
                      {"stats", stats, tokens * 2 * (plan->L + 2) * 4, false, true}};
  if ((st = check_arrays(args, 10)) != CGCONV_OK) return st;
  ResidualArgs a{dtype, x, u, gate, post_weight, scale, weight, bias, eps, r, y, stats, (long long)tokens, plan->L,
                 plan->K, (int)C};
  return launched(launch_residual(a, stream));
}

int cgconv_seq_residual_norm_backward(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const void* u,
                                      const void* gate, const float* post_weight, const float* scale,
                                      const float* weight, const float* stats, const void* grad_r, const void* grad_y,
                                      void* grad_x, void* grad_u, void* grad_gate, float* grad_post_weight,
                                      float* grad_scale, float* grad_weight, float* grad_bias, hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  if (!grad_x && !grad_u && !grad_gate && !grad_post_weight && !grad_scale && !grad_weight && !grad_bias) {
    set_last_error("at least one gradient must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  if (grad_gate && !gate) {
    set_last_error("grad_gate is given without a gate");
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t tokens = plan->B * plan->N, C = plan->C, n = tokens * plan->K * C * seq_type_size(dtype);
  const size_t nw = (plan->L + 1) * C * 4, ng = tokens * C * seq_type_size(dtype);
  const Arg args[] = {{"x", x, n, true, false},
                      {"u", u, n, true, false},
                      {"gate", gate, ng, false, false},
                      {"post_weight", post_weight, nw, false, false},
                      {"scale", scale, C * 4, false, false},
                      {"weight", weight, nw, false, false},
                      {"stats", stats, tokens * 2 * (plan->L + 2) * 4, true, false},
                      {"grad_r", grad_r, n, false, false},
                      {"grad_y", grad_y, n, true, false},
                      {"grad_x", grad_x, n, false, true},
                      {"grad_u", grad_u, n, false, true},
                      {"grad_gate", grad_gate, ng, false, true},
                      {"grad_post_weight", grad_post_weight, nw, false, true},
                      {"grad_scale", grad_scale, C * 4, false, true},
                      {"grad_weight", grad_weight, nw, false, true},
                      {"grad_bias", grad_bias, C * 4, false, true}};
  if ((st = check_arrays(args, 16)) != CGCONV_OK) return st;
  ResidualBwdArgs g{};
  g.a = {dtype, x, u, gate, post_weight, scale, weight, nullptr, 0.f, nullptr, nullptr, const_cast<float*>(stats),
         (long long)tokens, plan->L, plan->K, (int)C};
  g.gr = grad_r;
  g.gy = grad_y;
  g.gx = grad_x;
  g.gu = grad_u;
  g.ggate = grad_gate;
  g.gpost = grad_post_weight;
  g.gscale = grad_scale;
  g.gw = grad_weight;
  g.gb = grad_bias;
  g.part = grad_post_weight || grad_scale || grad_weight || grad_bias ? static_cast<float*>(plan->ws) : nullptr;
  return launched(launch_residual_backward(g, stream));
}

}  // extern "C"

namespace {

int check_width(int32_t width) {
  if (width < 2 || width > CGCONV_SEQ_WIDTH) {
    set_last_error("unsupported width=%d: 2..%d", width, CGCONV_SEQ_WIDTH);
    return CGCONV_ERR_UNSUPPORTED;
  }
  return CGCONV_OK;
}

ConvArgs conv_args(const cgconv_seq_plan* p, int32_t dtype, int32_t width, const void* x, const float* weight,
                   const float* bias, int32_t activation, const int32_t* lengths) {
  ConvArgs a{};
  a.type = dtype;
  a.x = x;
  a.weight = weight;
  a.bias = bias;
  a.lengths = lengths;
  a.B = (int)p->B;
  a.N = (int)p->N;
  a.L = p->L;
  a.K = p->K;
  a.C = (int)p->C;
  a.W = width;
  a.activation = activation != 0;
  return a;
}

int check_scan_plan(const cgconv_seq_plan* p, int32_t dtype) {
  const int st = check_plan(p, dtype);
  if (st == CGCONV_OK && p->S == 0) {
    set_last_error("the plan has no states (cgconv_seq_plan_create with states >= 1)");
    return CGCONV_ERR_INVALID_ARG;
  }
  return st;
}

ScanArgs scan_args(const cgconv_seq_plan* p, int32_t dtype, const void* x, const void* delta, const float* A,
                   const void* Bt, const void* Ct, const float* D, const float* delta_bias, const int32_t* lengths) {
  ScanArgs a{};
  a.type = dtype;
  a.x = x;
  a.delta = delta;
  a.A = A;
  a.Bt = Bt;
  a.Ct = Ct;
  a.D = D;
  a.bias = delta_bias;
  a.lengths = lengths;
  a.B = (int)p->B;
  a.N = (int)p->N;
  a.K = p->K;
  a.C = (int)p->C;
  a.S = p->S;
  a.ws = static_cast<float*>(p->ws);
  return a;
}

}  // namespace

extern "C" {

int cgconv_seq_conv(cgconv_seq_plan_t plan, int32_t dtype, int32_t width, const void* x, const float* weight,
                    const float* bias, int32_t activation, const int32_t* lengths, const void* state_in, void* y,
                    void* state_out, hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK || (st = check_width(width)) != CGCONV_OK) return st;
  const size_t row = (size_t)plan->K * plan->C * seq_type_size(dtype), n = plan->B * plan->N * row;
  const Arg args[] = {{"x", x, n, true, false},
                      {"weight", weight, width * (plan->L + 1) * (size_t)plan->C * 4, true, false},
                      {"bias", bias, (size_t)plan->C * 4, false, false},
                      {"lengths", lengths, (size_t)plan->B * 4, false, false},
                      {"state_in", state_in, plan->B * (width - 1) * row, false, false},
                      {"y", y, n, true, true},
                      {"state_out", state_out, plan->B * (width - 1) * row, false, true}};
  if ((st = check_arrays(args, 7)) != CGCONV_OK) return st;
  ConvArgs a = conv_args(plan, dtype, width, x, weight, bias, activation, lengths);
  a.state_in = state_in;
  a.y = y;
  a.state_out = state_out;
  return launched(launch_conv(a, stream));
}

int cgconv_seq_conv_step(cgconv_seq_plan_t plan, int32_t dtype, int32_t width, const void* x, const float* weight,
                         const float* bias, int32_t activation, void* state, void* y, hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK || (st = check_width(width)) != CGCONV_OK) return st;
  const size_t n = (size_t)plan->B * plan->K * plan->C * seq_type_size(dtype);
  const Arg args[] = {{"x", x, n, true, false},
                      {"weight", weight, width * (plan->L + 1) * (size_t)plan->C * 4, true, false},
                      {"bias", bias, (size_t)plan->C * 4, false, false},
                      {"state", state, (width - 1) * n, true, true},
                      {"y", y, n, true, true}};
  if ((st = check_arrays(args, 5)) != CGCONV_OK) return st;
  ConvArgs a = conv_args(plan, dtype, width, x, weight, bias, activation, nullptr);
  a.y = y;
  a.state_out = state;
  return launched(launch_conv_step(a, stream));
}

int cgconv_seq_conv_backward(cgconv_seq_plan_t plan, int32_t dtype, int32_t width, const void* x,
                             const float* weight, const float* bias, int32_t activation, const int32_t* lengths,
                             const void* grad_y, void* grad_x, float* grad_weight, float* grad_bias,
                             hipStream_t stream) {
  int st = check_plan(plan, dtype);
  if (st != CGCONV_OK || (st = check_width(width)) != CGCONV_OK) return st;
  if (!grad_x && !grad_weight && !grad_bias) {
    set_last_error("at least one of grad_x, grad_weight and grad_bias must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t n = (size_t)plan->B * plan->N * plan->K * plan->C * seq_type_size(dtype);
  const size_t nw = width * (plan->L + 1) * (size_t)plan->C * 4;
  const Arg args[] = {{"x", x, n, true, false},
                      {"weight", weight, nw, true, false},
                      {"bias", bias, (size_t)plan->C * 4, false, false},
                      {"lengths", lengths, (size_t)plan->B * 4, false, false},
                      {"grad_y", grad_y, n, true, false},
                      {"grad_x", grad_x, n, false, true},
                      {"grad_weight", grad_weight, nw, false, true},
                      {"grad_bias", grad_bias, (size_t)plan->C * 4, false, true}};
  if ((st = check_arrays(args, 8)) != CGCONV_OK) return st;
  ConvBwdArgs g{};
  g.a = conv_args(plan, dtype, width, x, weight, bias, activation, lengths);
  g.gy = grad_y;
  g.gx = grad_x;
  g.gw = grad_weight;
  g.gb = grad_bias;
  g.part = grad_weight || grad_bias ? static_cast<float*>(plan->ws) : nullptr;
  return launched(launch_conv_backward(g, stream));
}

int cgconv_seq_scan(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const void* delta, const float* A,
                    const void* Bt, const void* Ct, const float* D, const float* delta_bias, const int32_t* lengths,
                    const float* state_in, void* y, float* state_out, hipStream_t stream) {
  int st = check_scan_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  const size_t ts = seq_type_size(dtype), tokens = plan->B * plan->N, C = plan->C;
  const size_t state = plan->B * plan->S * plan->K * C * 4;
  const Arg args[] = {{"x", x, tokens * plan->K * C * ts, true, false},
                      {"delta", delta, tokens * C * ts, true, false},
                      {"A", A, C * plan->S * 4, true, false},
                      {"Bt", Bt, tokens * plan->S * ts, true, false},
                      {"Ct", Ct, tokens * plan->S * ts, true, false},
                      {"D", D, C * 4, false, false},
                      {"delta_bias", delta_bias, C * 4, false, false},
                      {"lengths", lengths, (size_t)plan->B * 4, false, false},
                      {"state_in", state_in, state, false, false},
                      {"y", y, tokens * plan->K * C * ts, true, true},
                      {"state_out", state_out, state, false, true}};
  if ((st = check_arrays(args, 11)) != CGCONV_OK) return st;
  ScanArgs a = scan_args(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, lengths);
  a.state_in = state_in;
  a.y = y;
  a.state_out = state_out;
  return launched(launch_scan(a, stream));
}

int cgconv_seq_scan_step(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const void* delta, const float* A,
                         const void* Bt, const void* Ct, const float* D, const float* delta_bias, float* state,
                         void* y, hipStream_t stream) {
  int st = check_scan_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  const size_t ts = seq_type_size(dtype), B = plan->B, C = plan->C;
  const Arg args[] = {{"x", x, B * plan->K * C * ts, true, false},
                      {"delta", delta, B * C * ts, true, false},
                      {"A", A, C * plan->S * 4, true, false},
                      {"Bt", Bt, B * plan->S * ts, true, false},
                      {"Ct", Ct, B * plan->S * ts, true, false},
                      {"D", D, C * 4, false, false},
                      {"delta_bias", delta_bias, C * 4, false, false},
                      {"state", state, B * plan->S * plan->K * C * 4, true, true},
                      {"y", y, B * plan->K * C * ts, true, true}};
  if ((st = check_arrays(args, 9)) != CGCONV_OK) return st;
  ScanArgs a = scan_args(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, nullptr);
  a.y = y;
  a.state_out = state;
  return launched(launch_scan_step(a, stream));
}

int cgconv_seq_scan_backward(cgconv_seq_plan_t plan, int32_t dtype, const void* x, const void* delta, const float* A,
                             const void* Bt, const void* Ct, const float* D, const float* delta_bias,
                             const int32_t* lengths, const void* grad_y, void* grad_x, void* grad_delta,
                             float* grad_A, void* grad_Bt, void* grad_Ct, float* grad_D, float* grad_delta_bias,
                             hipStream_t stream) {
  int st = check_scan_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  if (!grad_x && !grad_delta && !grad_A && !grad_Bt && !grad_Ct && !grad_D && !grad_delta_bias) {
    set_last_error("at least one gradient must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t ts = seq_type_size(dtype), tokens = plan->B * plan->N, C = plan->C;
  const size_t n = tokens * plan->K * C * ts, nd = tokens * C * ts, na = C * plan->S * 4, nb = tokens * plan->S * ts;
  const Arg args[] = {{"x", x, n, true, false},
                      {"delta", delta, nd, true, false},
                      {"A", A, na, true, false},
                      {"Bt", Bt, nb, true, false},
                      {"Ct", Ct, nb, true, false},
                      {"D", D, C * 4, false, false},
                      {"delta_bias", delta_bias, C * 4, false, false},
                      {"lengths", lengths, (size_t)plan->B * 4, false, false},
                      {"grad_y", grad_y, n, true, false},
                      {"grad_x", grad_x, n, false, true},
                      {"grad_delta", grad_delta, nd, false, true},
                      {"grad_A", grad_A, na, false, true},
                      {"grad_Bt", grad_Bt, nb, false, true},
                      {"grad_Ct", grad_Ct, nb, false, true},
                      {"grad_D", grad_D, C * 4, false, true},
                      {"grad_delta_bias", grad_delta_bias, C * 4, false, true}};
  if ((st = check_arrays(args, 16)) != CGCONV_OK) return st;
  ScanBwdArgs g{};
  g.a = scan_args(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, lengths);
  g.gy = grad_y;
  g.gx = grad_x;
  g.gdelta = grad_delta;
  g.gA = grad_A;
  g.gB = grad_Bt;
  g.gC = grad_Ct;
  g.gD = grad_D;
  g.gbias = grad_delta_bias;
  return launched(launch_scan_backward(g, stream));
}

}  // extern "C"

namespace {

int check_rule_plan(const cgconv_seq_plan* p, int32_t dtype) {
  const int st = check_plan(p, dtype);
  if (st == CGCONV_OK && p->H == 0) {
    set_last_error("the plan has no delta rule (cgconv_seq_plan_create_rule)");
    return CGCONV_ERR_INVALID_ARG;
  }
  return st;
}

RuleArgs rule_args(const cgconv_seq_plan* p, int32_t dtype, const void* q, const void* k, const void* v,
                   const float* decay, const float* beta, float scale, int32_t normalize, const int32_t* lengths) {
  RuleArgs a{};
  a.type = dtype;
  a.n = rule_sizes(p);
  a.q = q;
  a.k = k;
  a.v = v;
  a.decay = decay;
  a.beta = beta;
  a.lengths = lengths;
  a.scale = scale;
  a.normalize = normalize != 0;
  a.ws = static_cast<char*>(p->ws);
  return a;
}

}  // namespace

extern "C" {

int cgconv_seq_delta_rule(cgconv_seq_plan_t plan, int32_t dtype, const void* q, const void* k, const void* v,
                          const float* decay, const float* beta, float scale, int32_t normalize,
                          const int32_t* lengths, const float* state_in, void* y, float* state_out,
                          hipStream_t stream) {
  int st = check_rule_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  const size_t ts = seq_type_size(dtype), tokens = plan->B * plan->N, row = (size_t)plan->K * plan->C;
  const size_t keys = tokens * plan->Hk * plan->D * ts, gates = tokens * plan->H * 4, state = plan->B * plan->D * row * 4;
  const Arg args[] = {{"q", q, keys, true, false},
                      {"k", k, keys, true, false},
                      {"v", v, tokens * row * ts, true, false},
                      {"decay", decay, gates, true, false},
                      {"beta", beta, gates, true, false},
                      {"lengths", lengths, (size_t)plan->B * 4, false, false},
                      {"state_in", state_in, state, false, false},
                      {"y", y, tokens * row * ts, true, true},
                      {"state_out", state_out, state, false, true}};
  if ((st = check_arrays(args, 9)) != CGCONV_OK) return st;
  RuleArgs a = rule_args(plan, dtype, q, k, v, decay, beta, scale, normalize, lengths);
  a.state_in = state_in;
  a.y = y;
  a.state_out = state_out;
  return launched(launch_rule(a, stream));
}

int cgconv_seq_delta_rule_step(cgconv_seq_plan_t plan, int32_t dtype, const void* q, const void* k, const void* v,
                               const float* decay, const float* beta, float scale, int32_t normalize, float* state,
                               void* y, hipStream_t stream) {
  int st = check_rule_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  const size_t ts = seq_type_size(dtype), B = plan->B, row = (size_t)plan->K * plan->C;
  const Arg args[] = {{"q", q, B * plan->Hk * plan->D * ts, true, false},
                      {"k", k, B * plan->Hk * plan->D * ts, true, false},
                      {"v", v, B * row * ts, true, false},
                      {"decay", decay, B * plan->H * 4, true, false},
                      {"beta", beta, B * plan->H * 4, true, false},
                      {"state", state, B * plan->D * row * 4, true, true},
                      {"y", y, B * row * ts, true, true}};
  if ((st = check_arrays(args, 7)) != CGCONV_OK) return st;
  RuleArgs a = rule_args(plan, dtype, q, k, v, decay, beta, scale, normalize, nullptr);
  a.y = y;
  a.state_out = state;
  return launched(launch_rule_step(a, stream));
}

int cgconv_seq_delta_rule_backward(cgconv_seq_plan_t plan, int32_t dtype, const void* q, const void* k, const void* v,
                                   const float* decay, const float* beta, float scale, int32_t normalize,
                                   const int32_t* lengths, const float* state_in, const void* grad_y,
                                   const float* grad_state, void* grad_q, void* grad_k, void* grad_v,
                                   float* grad_decay, float* grad_beta, float* grad_state_in, hipStream_t stream) {
  int st = check_rule_plan(plan, dtype);
  if (st != CGCONV_OK) return st;
  if (!plan->rule_backward) {
    set_last_error("the plan has no workspace for the delta rule's backward (cgconv_seq_plan_create_rule with backward)");
    return CGCONV_ERR_INVALID_ARG;
  }
  if (!grad_q && !grad_k && !grad_v && !grad_decay && !grad_beta && !grad_state_in) {
    set_last_error("at least one gradient must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  const size_t ts = seq_type_size(dtype), tokens = plan->B * plan->N, row = (size_t)plan->K * plan->C;
  const size_t keys = tokens * plan->Hk * plan->D * ts, gates = tokens * plan->H * 4, state = plan->B * plan->D * row * 4;
  const Arg args[] = {{"q", q, keys, true, false},
                      {"k", k, keys, true, false},
                      {"v", v, tokens * row * ts, true, false},
                      {"decay", decay, gates, true, false},
                      {"beta", beta, gates, true, false},
                      {"lengths", lengths, (size_t)plan->B * 4, false, false},
                      {"state_in", state_in, state, false, false},
                      {"grad_y", grad_y, tokens * row * ts, true, false},
                      {"grad_state", grad_state, state, false, false},
                      {"grad_q", grad_q, keys, false, true},
                      {"grad_k", grad_k, keys, false, true},
                      {"grad_v", grad_v, tokens * row * ts, false, true},
                      {"grad_decay", grad_decay, gates, false, true},
                      {"grad_beta", grad_beta, gates, false, true},
                      {"grad_state_in", grad_state_in, state, false, true}};
  if ((st = check_arrays(args, 15)) != CGCONV_OK) return st;
  RuleBwdArgs g{};
  g.a = rule_args(plan, dtype, q, k, v, decay, beta, scale, normalize, lengths);
  g.a.state_in = state_in;
  g.gy = grad_y;
  g.gstate = grad_state;
  g.gq = grad_q;
  g.gk = grad_k;
  g.gv = grad_v;
  g.gdecay = grad_decay;
  g.gbeta = grad_beta;
  g.gstate_in = grad_state_in;
  return launched(launch_rule_backward(g, stream));
}

static int check_pack(int32_t dtype, int64_t rows, int64_t C) {
  const int st = check_type(dtype);
  if (st != CGCONV_OK) return st;
  if (rows < 1 || C < 1 || C > INT32_MAX || rows > (INT64_MAX >> 8) / C) {
    set_last_error("invalid sizes: rows=%lld C=%lld", (long long)rows, (long long)C);
    return CGCONV_ERR_INVALID_ARG;
  }
  constexpr int64_t kGroups = (1LL << 29) - 32;  // whole blocks of 32 groups, 8 threads each, below 2^32 threads
  if (rows > kGroups / pack_blocks(C)) {
    set_last_error("unsupported rows=%lld at C=%lld: too many for one launch", (long long)rows, (long long)C);
    return CGCONV_ERR_UNSUPPORTED;
  }
  return CGCONV_OK;
}

int cgconv_pack8(int32_t dtype, int64_t rows, int64_t C, const void* x, int8_t* codes, uint8_t* scales,
                 hipStream_t stream) {
  clear_last_error();
  int st = check_pack(dtype, rows, C);
  if (st != CGCONV_OK) return st;
  const size_t n = (size_t)rows * C;
  const Arg args[] = {{"x", x, n * seq_type_size(dtype), true, false},
                      {"codes", codes, n, true, true},
                      {"scales", scales, (size_t)rows * pack_blocks(C), true, true}};
  if ((st = check_arrays(args, 3)) != CGCONV_OK) return st;
  return launched(launch_pack(dtype, x, codes, scales, rows, (int)C, stream));
}

int cgconv_unpack8(int32_t dtype, int64_t rows, int64_t C, const int8_t* codes, const uint8_t* scales, void* x,
                   hipStream_t stream) {
  clear_last_error();
  int st = check_pack(dtype, rows, C);
  if (st != CGCONV_OK) return st;
  const size_t n = (size_t)rows * C;
  const Arg args[] = {{"codes", codes, n, true, false},
                      {"scales", scales, (size_t)rows * pack_blocks(C), true, false},
                      {"x", x, n * seq_type_size(dtype), true, true}};
  if ((st = check_arrays(args, 3)) != CGCONV_OK) return st;
  return launched(launch_unpack(dtype, codes, scales, x, rows, (int)C, stream));
}

}  // extern "C"

namespace {

// Sizes of a list of tensors: whole, and together below 2^60 values.
int check_counts(int64_t n, const int64_t* counts) {
  if (n < 0 || (n > 0 && !counts)) {
    set_last_error("invalid list of tensors: n=%lld", (long long)n);
    return CGCONV_ERR_INVALID_ARG;
  }
  int64_t total = 0;
  for (int64_t i = 0; i < n; ++i) {
    if (counts[i] < 0 || counts[i] > (1LL << 60) - total) {
      set_last_error("invalid number of values of tensor %lld: %lld", (long long)i, (long long)counts[i]);
      return CGCONV_ERR_INVALID_ARG;
    }
    total += counts[i];
  }
  if (n > CGCONV_CLIP_TENSORS) {
    set_last_error("unsupported n=%lld: at most %d tensors", (long long)n, CGCONV_CLIP_TENSORS);
    return CGCONV_ERR_UNSUPPORTED;
  }
  return CGCONV_OK;
}

// What a list's call writes shares no byte with anything else of the call, but for an output
// in its own gradient's place: the spans in the order of their addresses, each against the
// ends of those before it.
int check_spans(const ClipArgs& a, size_t ws_bytes) {
  struct Span {
    uintptr_t from, to;
    bool written;
  };
  std::vector<Span> spans;
  try {
    spans.reserve(2 * (size_t)a.n + 2);
  } catch (const std::bad_alloc&) {
    set_last_error("host allocation failed");
    return CGCONV_ERR_OUT_OF_MEMORY;
  }
  const auto add = [&](const void* p, size_t bytes, bool written) {
    if (bytes) spans.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
  };
  for (int64_t i = 0; i < a.n; ++i) {
    const size_t bytes = (size_t)a.counts[i] * seq_type_size(a.types[i]);
    add(a.out[i], bytes, true);
    if (a.grads[i] != a.out[i]) add(a.grads[i], bytes, false);
  }
  add(a.norm, 4, true);
  add(a.ws, ws_bytes, true);
  std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.from < y.from; });
  uintptr_t any = 0, written = 0;
  for (const Span& s : spans) {
    if (s.from < (s.written ? any : written)) {
      set_last_error("what is written must not overlap another array of the call");
      return CGCONV_ERR_INVALID_ARG;
    }
    any = std::max(any, s.to);
    if (s.written) written = std::max(written, s.to);
  }
  return CGCONV_OK;
}

}  // namespace

extern "C" {

int64_t cgconv_clip_workspace(int64_t n, const int64_t* counts) {
  clear_last_error();
  const int st = check_counts(n, counts);
  return st != CGCONV_OK ? st : (int64_t)clip_workspace_bytes(n, counts);
}

int cgconv_clip(int64_t n, const int32_t* dtypes, const int64_t* counts, const void* const* grads, void* const* out,
                float max_norm, float eps, float* norm, void* workspace, int64_t workspace_bytes,
                hipStream_t stream) {
  clear_last_error();
  int st = check_counts(n, counts);
  if (st != CGCONV_OK) return st;
  if (n > 0 && (!dtypes || !grads || !out)) {
    set_last_error("dtypes, grads and out must be given");
    return CGCONV_ERR_INVALID_ARG;
  }
  if (!(max_norm >= 0.f) || !(eps >= 0.f)) {
    set_last_error("max_norm=%g and eps=%g must be >= 0", (double)max_norm, (double)eps);
    return CGCONV_ERR_INVALID_ARG;
  }
  const Arg args[] = {{"norm", norm, 4, true, true}, {"workspace", workspace, 0, true, true}};
  if ((st = check_arrays(args, 2, 4)) != CGCONV_OK) return st;
  if ((reinterpret_cast<uintptr_t>(workspace) & 7) != 0) {
    set_last_error("workspace must be 8-byte aligned");
    return CGCONV_ERR_ALIGNMENT;
  }
  const size_t needed = clip_workspace_bytes(n, counts);
  if (workspace_bytes < 0 || (size_t)workspace_bytes < needed) {
    set_last_error("workspace of %lld bytes, %zu are needed", (long long)workspace_bytes, needed);
    return CGCONV_ERR_INVALID_ARG;
  }
  for (int64_t i = 0; i < n; ++i) {
    if ((st = check_type(dtypes[i])) != CGCONV_OK) return st;
    if (counts[i] == 0) continue;
    if (!grads[i] || !out[i]) {
      set_last_error("tensor %lld must be a non-NULL device pointer", (long long)i);
      return CGCONV_ERR_INVALID_ARG;
    }
    const uintptr_t low = (reinterpret_cast<uintptr_t>(grads[i]) | reinterpret_cast<uintptr_t>(out[i]));
    if (low & (seq_type_size(dtypes[i]) - 1)) {
      set_last_error("tensor %lld must be aligned to its values", (long long)i);
      return CGCONV_ERR_ALIGNMENT;
    }
  }
  const ClipArgs a{n, dtypes, counts, grads, out, max_norm, eps, norm, static_cast<double*>(workspace)};
  if ((st = check_spans(a, needed)) != CGCONV_OK) return st;
  return launched(launch_clip(a, stream));
}

}  // extern "C"
