// Sequence plan and the entry points of the operators around the convolution
// (see include/cgconv.h, "Sequence operators"): checks of arguments, the
// plan's workspace, launches.  Kernels: norm.hip, pack.hip, conv.hip, scan.hip,
// scan_bwd.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>

#include "cgconv.h"
#include "seq.h"

using namespace cgconv;

struct cgconv_seq_plan {
  int64_t B = 0, N = 0, C = 0;
  int L = 0, K = 0, S = 0;
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

}  // namespace

extern "C" {

cgconv_seq_plan_t cgconv_seq_plan_create(int64_t batch, int64_t N, int32_t L_max, int64_t C, int32_t states) {
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
  hipError_t e = hipGetDevice(&p->device);
  if (e != hipSuccess) {
    set_last_error("hipGetDevice failed: %s", hipGetErrorString(e));
    delete p;
    return nullptr;
  }
  p->ws_bytes = std::max(norm_bwd_part_bytes(batch * N, L_max, (int)C), conv_bwd_part_bytes(batch, N, K, C));
  if (states) p->ws_bytes = std::max(p->ws_bytes, scan_workspace_bytes(batch, N, K, C, states));
  if ((e = hipMalloc(&p->ws, p->ws_bytes)) != hipSuccess) {
    set_last_error("workspace allocation of %zu bytes failed: %s", p->ws_bytes, hipGetErrorString(e));
    (void)hipGetLastError();
    delete p;
    return nullptr;
  }
  return p;
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
