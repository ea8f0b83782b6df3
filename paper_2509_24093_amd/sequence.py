"""Operators around the convolution on [batch, tokens, (L+1)^2, C] features:
layer norm by degree, the short causal convolution and the selective state space
scan (whole sequences and single tokens), and activation checkpoints in 8 bits
(``include/cgconv.h``, "Sequence operators").  As in the package's main module, every step runs in the
library's HIP kernels; this module checks and marshals arguments.
"""

from __future__ import annotations

import ctypes
import math

CGCONV_F32 = 0
CGCONV_BF16 = 1
CGCONV_SEQ_TOKENS = 1 << 30
CGCONV_SEQ_VALUES = 1 << 38
CGCONV_SEQ_SEGMENT = 16384
CGCONV_SEQ_STATES = 32
CGCONV_SEQ_WIDTH = 8
CGCONV_SEQ_KEY_DIM = 128

_vp, _i64, _i32, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float

# name: (argument types, result type); bound when the library is loaded
SIGNATURES = {
    "cgconv_seq_plan_create": ([_i64, _i64, _i32, _i64, _i32], _vp),
    "cgconv_seq_plan_destroy": ([_vp], None),
    "cgconv_seq_plan_info": ([_vp, ctypes.POINTER(ctypes.c_size_t)], ctypes.c_int),
    "cgconv_seq_norm": ([_vp, _i32, _vp, _vp, _vp, _f32, _vp, _vp, _vp, _vp, _vp, _vp], ctypes.c_int),
    "cgconv_seq_norm_backward": ([_vp, _i32] + [_vp] * 11, ctypes.c_int),
    "cgconv_seq_conv": ([_vp, _i32, _i32, _vp, _vp, _vp, _i32] + [_vp] * 5, ctypes.c_int),
    "cgconv_seq_conv_step": ([_vp, _i32, _i32, _vp, _vp, _vp, _i32] + [_vp] * 3, ctypes.c_int),
    "cgconv_seq_conv_backward": ([_vp, _i32, _i32, _vp, _vp, _vp, _i32] + [_vp] * 6, ctypes.c_int),
    "cgconv_seq_scan": ([_vp, _i32] + [_vp] * 12, ctypes.c_int),
    "cgconv_seq_scan_step": ([_vp, _i32] + [_vp] * 10, ctypes.c_int),
    "cgconv_seq_scan_backward": ([_vp, _i32] + [_vp] * 17, ctypes.c_int),
    "cgconv_seq_plan_create_rule": ([_i64, _i64, _i32, _i64] + [_i32] * 5, _vp),
    "cgconv_seq_delta_rule": ([_vp, _i32] + [_vp] * 5 + [_f32, _i32] + [_vp] * 5, ctypes.c_int),
    "cgconv_seq_delta_rule_step": ([_vp, _i32] + [_vp] * 5 + [_f32, _i32] + [_vp] * 3, ctypes.c_int),
    "cgconv_seq_delta_rule_backward": ([_vp, _i32] + [_vp] * 5 + [_f32, _i32] + [_vp] * 11, ctypes.c_int),
    "cgconv_seq_residual_norm": ([_vp, _i32] + [_vp] * 7 + [_f32] + [_vp] * 4, ctypes.c_int),
    "cgconv_seq_residual_norm_backward": ([_vp, _i32] + [_vp] * 17, ctypes.c_int),
    "cgconv_clip_workspace": ([_i64, _vp], _i64),
    "cgconv_clip": ([_i64] + [_vp] * 4 + [_f32, _f32, _vp, _vp, _i64, _vp], ctypes.c_int),
    "cgconv_pack8": ([_i32, _i64, _i64] + [_vp] * 4, ctypes.c_int),
    "cgconv_unpack8": ([_i32, _i64, _i64] + [_vp] * 4, ctypes.c_int),
}


def bind(lib) -> None:
    for name, (args, res) in SIGNATURES.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res


def _main():
    import paper_2509_24093_amd as P
    return P


# ---- C ABI, same names -------------------------------------------------------

def cgconv_seq_plan_create(batch: int, N: int, L_max: int, C: int, states: int = 0) -> int:
    P = _main()
    h = P.library().cgconv_seq_plan_create(batch, N, L_max, C, states)
    if not h:
        raise P.CgconvError(P.CGCONV_ERR_INVALID_ARG, P.cgconv_last_error())
    return h


def cgconv_seq_plan_create_rule(batch: int, N: int, L_max: int, C: int, states: int, heads: int, key_heads: int,
                                key_dim: int, backward: bool = True) -> int:
    P = _main()
    h = P.library().cgconv_seq_plan_create_rule(batch, N, L_max, C, states, heads, key_heads, key_dim, int(backward))
    if not h:
        raise P.CgconvError(P.CGCONV_ERR_INVALID_ARG, P.cgconv_last_error())
    return h


def cgconv_seq_plan_destroy(plan: int) -> None:
    _main().library().cgconv_seq_plan_destroy(plan)


def cgconv_seq_plan_info(plan: int) -> int:
    """Workspace bytes."""
    P = _main()
    n = ctypes.c_size_t()
    P._check(P.library().cgconv_seq_plan_info(plan, ctypes.byref(n)))
    return n.value


def cgconv_seq_norm(plan, dtype, x, weight, bias, eps, y, mean, rstd, codes, scales, stream) -> int:
    """Layer norm by degree (device pointers; weight, bias, the statistics and
    the checkpoint may be None)."""
    P = _main()
    return P._check(P.library().cgconv_seq_norm(plan, dtype, x, weight, bias, eps, y, mean, rstd, codes, scales,
                                                stream))


def cgconv_seq_norm_backward(plan, dtype, x, codes, scales, weight, mean, rstd, grad_y, grad_x, grad_weight,
                             grad_bias, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_norm_backward(plan, dtype, x, codes, scales, weight, mean, rstd, grad_y,
                                                         grad_x, grad_weight, grad_bias, stream))


def cgconv_seq_residual_norm(plan, dtype, x, u, gate, post_weight, scale, weight, bias, eps, r, y, stats, stream) -> int:
    """Norms around a residual connection (gate, parameters and stats may be None)."""
    P = _main()
    return P._check(P.library().cgconv_seq_residual_norm(plan, dtype, x, u, gate, post_weight, scale, weight, bias, eps,
                                                         r, y, stats, stream))


def cgconv_seq_residual_norm_backward(plan, dtype, x, u, gate, post_weight, scale, weight, stats, grad_r, grad_y,
                                      grad_x, grad_u, grad_gate, grad_post_weight, grad_scale, grad_weight, grad_bias,
                                      stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_residual_norm_backward(
        plan, dtype, x, u, gate, post_weight, scale, weight, stats, grad_r, grad_y, grad_x, grad_u, grad_gate,
        grad_post_weight, grad_scale, grad_weight, grad_bias, stream))


def cgconv_seq_conv(plan, dtype, width, x, weight, bias, activation, lengths, state_in, y, state_out, stream) -> int:
    """Short causal convolution (bias, lengths and the states may be None)."""
    P = _main()
    return P._check(P.library().cgconv_seq_conv(plan, dtype, width, x, weight, bias, activation, lengths, state_in, y,
                                                state_out, stream))


def cgconv_seq_conv_step(plan, dtype, width, x, weight, bias, activation, state, y, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_conv_step(plan, dtype, width, x, weight, bias, activation, state, y, stream))


def cgconv_seq_conv_backward(plan, dtype, width, x, weight, bias, activation, lengths, grad_y, grad_x, grad_weight,
                             grad_bias, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_conv_backward(plan, dtype, width, x, weight, bias, activation, lengths,
                                                         grad_y, grad_x, grad_weight, grad_bias, stream))


def cgconv_seq_scan(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, lengths, state_in, y, state_out, stream) -> int:
    """Selective scan (D, delta_bias, lengths and the states may be None)."""
    P = _main()
    return P._check(P.library().cgconv_seq_scan(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, lengths, state_in, y,
                                                state_out, stream))


def cgconv_seq_scan_step(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, state, y, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_scan_step(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, state, y,
                                                     stream))


def cgconv_seq_scan_backward(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, lengths, grad_y, grad_x, grad_delta,
                             grad_A, grad_Bt, grad_Ct, grad_D, grad_delta_bias, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_scan_backward(plan, dtype, x, delta, A, Bt, Ct, D, delta_bias, lengths,
                                                         grad_y, grad_x, grad_delta, grad_A, grad_Bt, grad_Ct, grad_D,
                                                         grad_delta_bias, stream))


def cgconv_seq_delta_rule(plan, dtype, q, k, v, decay, beta, scale, normalize, lengths, state_in, y, state_out,
                          stream) -> int:
    """Gated delta rule (lengths and the states may be None)."""
    P = _main()
    return P._check(P.library().cgconv_seq_delta_rule(plan, dtype, q, k, v, decay, beta, scale, normalize, lengths,
                                                      state_in, y, state_out, stream))


def cgconv_seq_delta_rule_step(plan, dtype, q, k, v, decay, beta, scale, normalize, state, y, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_delta_rule_step(plan, dtype, q, k, v, decay, beta, scale, normalize, state,
                                                           y, stream))


def cgconv_seq_delta_rule_backward(plan, dtype, q, k, v, decay, beta, scale, normalize, lengths, state_in, grad_y,
                                   grad_state, grad_q, grad_k, grad_v, grad_decay, grad_beta, grad_state_in,
                                   stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_seq_delta_rule_backward(plan, dtype, q, k, v, decay, beta, scale, normalize,
                                                               lengths, state_in, grad_y, grad_state, grad_q, grad_k,
                                                               grad_v, grad_decay, grad_beta, grad_state_in, stream))


def cgconv_pack8(dtype, rows, C, x, codes, scales, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_pack8(dtype, rows, C, x, codes, scales, stream))


def cgconv_unpack8(dtype, rows, C, codes, scales, x, stream) -> int:
    P = _main()
    return P._check(P.library().cgconv_unpack8(dtype, rows, C, codes, scales, x, stream))


def cgconv_clip_workspace(counts) -> int:
    """Workspace bytes of a clipping of tensors of these numbers of values."""
    P = _main()
    n = P.library().cgconv_clip_workspace(len(counts), (ctypes.c_int64 * len(counts))(*counts))
    P._check(min(n, 0))
    return n


def cgconv_clip(dtypes, counts, grads, out, max_norm, eps, norm, workspace, workspace_bytes, stream) -> int:
    """Clipping of a list of tensors by their global norm (lists of type codes,
    numbers of values and device pointers)."""
    P, n = _main(), len(counts)
    return P._check(P.library().cgconv_clip(
        n, (ctypes.c_int32 * n)(*dtypes), (ctypes.c_int64 * n)(*counts), (_vp * n)(*grads), (_vp * n)(*out), max_norm, eps,
        norm, workspace, workspace_bytes, stream))


# ---- tensors -------------------------------------------------------------------

_codes = {}  # torch dtype: CGCONV_* code


def _dtype_code(name, dtype) -> int:
    if not _codes:
        import torch
        _codes.update({torch.float32: CGCONV_F32, torch.bfloat16: CGCONV_BF16})
    code = _codes.get(dtype)
    if code is None:
        raise ValueError(f"{name} must be float32 or bfloat16")
    return code


def _tensor(name, t, shape, dtype, device):
    """t's address after its checks; None stays None.  A step's call spends most
    of its time here: the accepted case is five cheap queries."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.device.index != device:
        raise ValueError(f"{name} is on GPU {t.device.index}, expected GPU {device}")
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")


def _features_dtype(name, t):
    """dtype and code of a feature tensor."""
    dtype = getattr(t, "dtype", None)
    return dtype, _dtype_code(name, dtype)


def _scale_shape(shape):
    return tuple(shape[:-1]) + ((shape[-1] + 31) // 32,)


def checkpoint_pack(x):
    """8-bit checkpoint of a contiguous fp32 or bf16 GPU tensor of any shape
    [..., C]: int8 codes of its shape and one power-of-two scale byte per 32
    channels, [..., ceil(C / 32)]; 1.03 bytes a value instead of 4 or 2."""
    import torch
    P = _main()
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.ndim < 1 or not x.is_contiguous():
        raise ValueError("x must be a contiguous GPU tensor")
    code = _dtype_code("x", x.dtype)
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scales = torch.empty(_scale_shape(x.shape), dtype=torch.uint8, device=x.device)
    if x.numel() == 0:
        return codes, scales
    if x.device.index != torch.cuda.current_device():
        raise ValueError(f"x is on GPU {x.device.index}, which is not current")
    C = x.shape[-1]
    cgconv_pack8(code, x.numel() // C, C, x.data_ptr(), codes.data_ptr(), scales.data_ptr(), P._current_stream(torch))
    return codes, scales


def checkpoint_unpack(codes, scales, dtype=None, out=None):
    """The values of a checkpoint, in float32 (default) or bfloat16."""
    import torch
    P = _main()
    dtype = (out.dtype if out is not None else torch.float32) if dtype is None else dtype
    code = _dtype_code("dtype", dtype)
    if not isinstance(codes, torch.Tensor) or not codes.is_cuda or codes.ndim < 1:
        raise ValueError("codes must be a GPU tensor")
    device = codes.device.index
    if out is None:
        out = torch.empty(codes.shape, dtype=dtype, device=codes.device)
    args = (_tensor("codes", codes, codes.shape, torch.int8, device),
            _tensor("scales", scales, _scale_shape(codes.shape), torch.uint8, device),
            _tensor("out", out, codes.shape, dtype, device))
    if codes.numel() == 0:
        return out
    if device != torch.cuda.current_device():
        raise ValueError(f"codes is on GPU {device}, which is not current")
    C = codes.shape[-1]
    cgconv_unpack8(code, codes.numel() // C, C, *args, P._current_stream(torch))
    return out


def _list_of(name, tensors, device):
    """Type codes, sizes and addresses of a list of contiguous GPU tensors.  A
    list of few tensors spends its call's time here: cheap queries, and the
    explanation only for a list that is refused."""
    import torch
    _dtype_code(name, torch.float32)
    try:
        if all([t.is_contiguous() and t.get_device() == device for t in tensors]):
            return ([_codes[t.dtype] for t in tensors], [t.numel() for t in tensors], [t.data_ptr() for t in tensors])
    except (AttributeError, KeyError):
        pass
    for i, t in enumerate(tensors):
        if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name}[{i}] must be a contiguous GPU tensor")
        if t.get_device() != device:
            raise ValueError(f"{name}[{i}] is on GPU {t.get_device()}, which is not current")
        _dtype_code(f"{name}[{i}]", t.dtype)
    raise ValueError(f"{name} must be tensors")


def clip_gradients(grads, max_norm: float, eps: float = 1e-6, out=None):
    """Clips contiguous fp32 or bf16 GPU tensors of any shapes by their global
    norm: each is multiplied by min(1, max_norm / (norm + eps)), in place or into
    the tensors of ``out``.  Returns the norm before, a float32 tensor of no
    dimensions (nothing waits for the GPU).  max_norm = inf: the norm alone."""
    import torch
    P = _main()
    grads = list(grads)
    device = torch.cuda.current_device()
    codes, counts, addresses = _list_of("grads", grads, device)
    to = addresses
    if out is not None:
        out = list(out)
        out_codes, out_counts, to = _list_of("out", out, device)
        if out_codes != codes or out_counts != counts:
            raise ValueError("out must hold tensors of the gradients' types and sizes")
    on = torch.device("cuda", device)
    size = cgconv_clip_workspace(counts)
    workspace, norm = torch.empty(size, dtype=torch.uint8, device=on), torch.empty((), dtype=torch.float32, device=on)
    cgconv_clip(codes, counts, addresses, to, max_norm, eps, norm.data_ptr(), workspace.data_ptr(), size,
                P._current_stream(torch))
    return norm


def _want_checkpoint(checkpoint) -> bool:
    if checkpoint not in (None, "int8"):
        raise ValueError("checkpoint must be None or 'int8'")
    return checkpoint == "int8"


def keep(ctx, checkpoint: bool, tensors, others=()):
    """Saves tensors for the backward pass, whole or as 8-bit checkpoints, and
    others as they are."""
    if checkpoint:
        saved = [s for t in tensors for s in checkpoint_pack(t)]
        ctx.kept_dtypes = [t.dtype for t in tensors]
    else:
        saved = list(tensors)
        ctx.kept_dtypes = None
    ctx.n_kept = len(tensors)
    ctx.save_for_backward(*saved, *others)


def kept(ctx):
    """(the tensors, the others) of :func:`keep`, unpacked."""
    saved = ctx.saved_tensors
    if ctx.kept_dtypes is None:
        return saved[:ctx.n_kept], saved[ctx.n_kept:]
    n = 2 * ctx.n_kept
    return [checkpoint_unpack(saved[2 * i], saved[2 * i + 1], dtype) for i, dtype in enumerate(ctx.kept_dtypes)], saved[n:]


class SequencePlan:
    """Sizes and workspace of the sequence operators for features
    [batch, N, (L_max+1)^2, C] (fp32 or bf16) on the current GPU; states: S of
    the selective scan (0: no scans, a smaller workspace).  heads, key_heads
    (default: heads) and key_dim: of the gated delta rule (0: none), with the
    workspace of its backward unless backward is False."""

    def __init__(self, batch: int, N: int, L_max: int, C: int, states: int = 0, heads: int = 0, key_heads: int = None,
                 key_dim: int = 0, backward: bool = True):
        import torch
        self._h = None
        self.heads, self.key_dim = int(heads), int(key_dim)
        self.key_heads = self.heads if key_heads is None else int(key_heads)
        if self.heads or self.key_heads or self.key_dim:
            self._h = cgconv_seq_plan_create_rule(int(batch), int(N), int(L_max), int(C), int(states), self.heads,
                                                  self.key_heads, self.key_dim, bool(backward))
        else:
            self._h = cgconv_seq_plan_create(int(batch), int(N), int(L_max), int(C), int(states))
        self._lib = _main().library()
        self.device = torch.cuda.current_device()
        self.batch, self.N, self.L_max, self.C, self.states = int(batch), int(N), int(L_max), int(C), int(states)
        self.shape = (self.batch, self.N, (self.L_max + 1) ** 2, self.C)
        self.token_shape = (self.batch,) + self.shape[2:]  # of a step
        self.state_shape = (self.batch, self.states) + self.shape[2:]  # of a scan
        self.memory_shape = (self.batch, self.key_dim) + self.shape[2:]  # of a delta rule's state
        self._scale = 1.0 / math.sqrt(self.key_dim) if self.key_dim > 0 else 1.0
        self._on = torch.device("cuda", self.device)
        self._f32, self._empty = torch.float32, torch.empty
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._raw_stream = raw or (lambda device: torch.cuda.current_stream(device).cuda_stream)

    def info(self) -> int:
        """Workspace bytes."""
        return cgconv_seq_plan_info(self._h)

    def _done(self, status: int) -> None:
        if status < 0:
            P = _main()
            raise P.CgconvError(status, P.cgconv_last_error())

    def _out(self, out, like, shape):
        """(out, its address); a new tensor if out is None."""
        if out is None:
            out = self._empty(shape, dtype=like.dtype, device=self._on)
            return out, out.data_ptr()
        return out, _tensor("out", out, shape, like.dtype, self.device)

    def _new(self, shape, dtype, wanted=True):
        return self._empty(shape, dtype=dtype, device=self._on) if wanted else None

    def norm(self, x, weight=None, bias=None, eps: float = 1e-5, checkpoint: bool = False, out=None):
        """Layer norm by degree (L_max = 0: the ordinary layer norm): weight
        [L_max+1, C] and bias [C], fp32 or None.  Returns (y, mean [batch, N],
        rstd [batch, N, L_max+1]), and the 8-bit checkpoint (codes, scales) of x
        behind them if asked for."""
        dtype, code = _features_dtype("x", x)
        f32, dev = self._f32, self.device
        px = _tensor("x", x, self.shape, dtype, dev)
        pw, pb = _tensor("weight", weight, (self.L_max + 1, self.C), f32, dev), _tensor("bias", bias, (self.C,), f32, dev)
        out, po = self._out(out, x, self.shape)
        mean, rstd = self._new(self.shape[:2], f32), self._new(self.shape[:2] + (self.L_max + 1,), f32)
        codes = scales = None
        if checkpoint:
            import torch
            codes, scales = self._new(self.shape, torch.int8), self._new(_scale_shape(self.shape), torch.uint8)
        self._done(self._lib.cgconv_seq_norm(self._h, code, px, pw, pb, eps, po, mean.data_ptr(), rstd.data_ptr(),
                                             codes.data_ptr() if checkpoint else None,
                                             scales.data_ptr() if checkpoint else None, self._raw_stream(dev)))
        return (out, mean, rstd, codes, scales) if checkpoint else (out, mean, rstd)

    def norm_backward(self, x, weight, mean, rstd, grad_y, need_x: bool = True, need_weight: bool = True,
                      need_bias: bool = True):
        """(grad_x, grad_weight, grad_bias) given grad_y and the forward's
        statistics; x is the input or its checkpoint (codes, scales).  A
        gradient that is not needed is None."""
        if not (need_x or need_weight or need_bias):
            return None, None, None
        dtype, code = _features_dtype("grad_y", grad_y)
        f32, dev = self._f32, self.device
        px = pc = ps = None
        if isinstance(x, (tuple, list)):
            import torch
            codes, scales = x
            pc = _tensor("codes", codes, self.shape, torch.int8, dev)
            ps = _tensor("scales", scales, _scale_shape(self.shape), torch.uint8, dev)
        else:
            px = _tensor("x", x, self.shape, dtype, dev)
        args = (self._h, code, px, pc, ps, _tensor("weight", weight, (self.L_max + 1, self.C), f32, dev),
                _tensor("mean", mean, self.shape[:2], f32, dev),
                _tensor("rstd", rstd, self.shape[:2] + (self.L_max + 1,), f32, dev),
                _tensor("grad_y", grad_y, self.shape, dtype, dev))
        grads = (self._new(self.shape, dtype, need_x), self._new((self.L_max + 1, self.C), f32, need_weight),
                 self._new((self.C,), f32, need_bias))
        self._done(self._lib.cgconv_seq_norm_backward(*args, *(None if t is None else t.data_ptr() for t in grads),
                                                      self._raw_stream(dev)))
        return grads

    # ---- norms around a residual connection

    def _residual_args(self, x, u, gate, post_weight, scale, weight):
        dtype, code = _features_dtype("x", x)
        dev, f32, per = self.device, self._f32, (self.L_max + 1, self.C)
        return dtype, (self._h, code, _tensor("x", x, self.shape, dtype, dev), _tensor("u", u, self.shape, dtype, dev),
                       _tensor("gate", gate, self.shape[:2] + (self.C,), dtype, dev),
                       _tensor("post_weight", post_weight, per, f32, dev), _tensor("scale", scale, (self.C,), f32, dev),
                       _tensor("weight", weight, per, f32, dev))

    def residual_norm(self, x, u, gate=None, post_weight=None, scale=None, weight=None, bias=None, eps: float = 1e-5,
                      out_r=None, out_y=None):
        """The norms on both sides of a residual connection: r = x + scale
        silu(gate) post_weight norm(u) and y = weight norm(r) + bias, norms by
        degree.  gate [batch, N, C] of x's type, post_weight and weight [L_max+1,
        C], scale and bias [C] in fp32; each may be None.  Returns (r, y, stats
        [batch, N, 2 (L_max+2)])."""
        dtype, args = self._residual_args(x, u, gate, post_weight, scale, weight)
        pb = _tensor("bias", bias, (self.C,), self._f32, self.device)
        r, pr = self._out(out_r, x, self.shape)
        y, py = self._out(out_y, x, self.shape)
        stats = self._new(self.shape[:2] + (2 * (self.L_max + 2),), self._f32)
        self._done(self._lib.cgconv_seq_residual_norm(*args, pb, eps, pr, py, stats.data_ptr(),
                                                      self._raw_stream(self.device)))
        return r, y, stats

    def residual_norm_backward(self, x, u, gate, post_weight, scale, weight, stats, grad_r, grad_y, need=(True,) * 7):
        """Gradients of (x, u, gate, post_weight, scale, weight, bias) given those
        of r (or None) and y and the forward's stats; None where ``need`` is False."""
        if not any(need):
            return (None,) * 7
        dtype, args = self._residual_args(x, u, gate, post_weight, scale, weight)
        dev, f32, lead = self.device, self._f32, self.shape[:2]
        args += (_tensor("stats", stats, lead + (2 * (self.L_max + 2),), f32, dev),
                 _tensor("grad_r", grad_r, self.shape, dtype, dev), _tensor("grad_y", grad_y, self.shape, dtype, dev))
        per, one = ((self.L_max + 1, self.C), f32), ((self.C,), f32)
        shapes = ((self.shape, dtype), (self.shape, dtype), (lead + (self.C,), dtype), per, one, per, one)
        grads = tuple(self._new(*s, n) for s, n in zip(shapes, need))
        self._done(self._lib.cgconv_seq_residual_norm_backward(
            *args, *(None if t is None else t.data_ptr() for t in grads), self._raw_stream(dev)))
        return grads

    # ---- short causal convolution

    def _conv_args(self, x, weight, bias, shape):
        dtype, code = _features_dtype("x", x)
        width = len(weight) if getattr(weight, "ndim", 0) == 3 else 0
        dev, f32 = self.device, self._f32
        return dtype, width, (self._h, code, width, _tensor("x", x, shape, dtype, dev),
                              _tensor("weight", weight, (width, self.L_max + 1, self.C), f32, dev),
                              _tensor("bias", bias, (self.C,), f32, dev))

    def _lengths(self, lengths):
        if lengths is None:
            return None
        import torch
        return _tensor("lengths", lengths, (self.batch,), torch.int32, self.device)

    def _conv_state_shape(self, width):
        return (self.batch, max(width - 1, 0)) + self.shape[2:]

    def conv_state(self, width: int, dtype=None):
        """The state before the first token: zeros [batch, width - 1, K, C]."""
        return self._new(self._conv_state_shape(width), dtype or self._f32).zero_()

    def conv(self, x, weight, bias=None, lengths=None, state=None, activation: bool = True, out=None):
        """Short causal convolution over the tokens: weight [width, L_max+1, C]
        and bias [C], fp32; the invariants pass z sigmoid(z) unless activation
        is False.  lengths (int32 [batch]): what tokens behind them hold does
        not matter, their outputs are zero.  Returns (y, state): the width - 1 inputs before
        every sequence's end, [batch, width - 1, K, C], for conv_step or the
        next piece (state=)."""
        dtype, width, args = self._conv_args(x, weight, bias, self.shape)
        shape, pl = self._conv_state_shape(width), self._lengths(lengths)
        ps = _tensor("state", state, shape, dtype, self.device)
        out, po = self._out(out, x, self.shape)
        last = self._new(shape, dtype)
        self._done(self._lib.cgconv_seq_conv(*args, 1 if activation else 0, pl, ps, po, last.data_ptr(),
                                             self._raw_stream(self.device)))
        return out, last

    def conv_step(self, x, weight, bias, state, activation: bool = True, out=None):
        """One token of every sequence: x [batch, K, C]; state is moved on in
        place.  Returns y [batch, K, C]."""
        dtype, width, args = self._conv_args(x, weight, bias, self.token_shape)
        ps = _tensor("state", state, self._conv_state_shape(width), dtype, self.device)
        out, po = self._out(out, x, self.token_shape)
        self._done(self._lib.cgconv_seq_conv_step(*args, 1 if activation else 0, ps, po,
                                                  self._raw_stream(self.device)))
        return out

    def conv_backward(self, x, weight, bias, grad_y, lengths=None, activation: bool = True, need_x: bool = True,
                      need_weight: bool = True, need_bias: bool = True):
        """(grad_x, grad_weight, grad_bias) given grad_y, from the zero state; a
        gradient that is not needed is None."""
        if not (need_x or need_weight or need_bias):
            return None, None, None
        dtype, width, args = self._conv_args(x, weight, bias, self.shape)
        args += (1 if activation else 0, self._lengths(lengths),
                 _tensor("grad_y", grad_y, self.shape, dtype, self.device))
        grads = (self._new(self.shape, dtype, need_x), self._new(weight.shape, self._f32, need_weight),
                 self._new((self.C,), self._f32, need_bias))
        self._done(self._lib.cgconv_seq_conv_backward(*args, *(None if t is None else t.data_ptr() for t in grads),
                                                      self._raw_stream(self.device)))
        return grads

    # ---- selective scan

    def _scan_args(self, x, delta, A, Bt, Ct, D, delta_bias, lead, shape):
        dtype, code = _features_dtype("x", x)
        S, C, dev, f32 = self.states, self.C, self.device, self._f32
        rows = lead + (S,)
        return dtype, (self._h, code, _tensor("x", x, shape, dtype, dev),
                       _tensor("delta", delta, lead + (C,), dtype, dev), _tensor("A", A, (C, S), f32, dev),
                       _tensor("Bt", Bt, rows, dtype, dev), _tensor("Ct", Ct, rows, dtype, dev),
                       _tensor("D", D, (C,), f32, dev), _tensor("delta_bias", delta_bias, (C,), f32, dev))

    def scan_state(self):
        """The state before the first token: fp32 zeros [batch, S, K, C]."""
        return self._new(self.state_shape, self._f32).zero_()

    def scan(self, x, delta, A, Bt, Ct, D=None, delta_bias=None, lengths=None, state=None, out=None):
        """Selective scan of whole sequences: delta [batch, N, C], Bt and Ct
        [batch, N, S] of x's type, A [C, S], D and delta_bias [C] in fp32.
        Returns (y, state): the state [batch, S, K, C] (fp32) after every
        sequence's last token, for scan_step or the next piece (state=)."""
        _, args = self._scan_args(x, delta, A, Bt, Ct, D, delta_bias, self.shape[:2], self.shape)
        pl, ps = self._lengths(lengths), _tensor("state", state, self.state_shape, self._f32, self.device)
        out, po = self._out(out, x, self.shape)
        last = self._new(self.state_shape, self._f32)
        self._done(self._lib.cgconv_seq_scan(*args, pl, ps, po, last.data_ptr(), self._raw_stream(self.device)))
        return out, last

    def scan_step(self, x, delta, A, Bt, Ct, D, state, delta_bias=None, out=None):
        """One token of every sequence: x [batch, K, C], delta [batch, C], Bt
        and Ct [batch, S]; state is moved on in place.  Returns y [batch, K, C]."""
        _, args = self._scan_args(x, delta, A, Bt, Ct, D, delta_bias, self.shape[:1], self.token_shape)
        ps = _tensor("state", state, self.state_shape, self._f32, self.device)
        out, po = self._out(out, x, self.token_shape)
        self._done(self._lib.cgconv_seq_scan_step(*args, ps, po, self._raw_stream(self.device)))
        return out

    def scan_backward(self, x, delta, A, Bt, Ct, D, grad_y, delta_bias=None, lengths=None, need=(True,) * 7):
        """Gradients of (x, delta, A, Bt, Ct, D, delta_bias) given grad_y, from
        the zero state; None where ``need`` is False."""
        if not any(need):
            return (None,) * 7
        lead, f32 = self.shape[:2], self._f32
        dtype, args = self._scan_args(x, delta, A, Bt, Ct, D, delta_bias, lead, self.shape)
        args += (self._lengths(lengths), _tensor("grad_y", grad_y, self.shape, dtype, self.device))
        rows = (lead + (self.states,), dtype)
        shapes = ((self.shape, dtype), (lead + (self.C,), dtype), ((self.C, self.states), f32), rows, rows,
                  ((self.C,), f32), ((self.C,), f32))
        grads = tuple(self._new(*s, n) for s, n in zip(shapes, need))
        self._done(self._lib.cgconv_seq_scan_backward(*args, *(None if t is None else t.data_ptr() for t in grads),
                                                      self._raw_stream(self.device)))
        return grads

    # ---- gated delta rule

    def _rule_args(self, q, k, v, decay, beta, scale, normalize, lead, shape):
        dtype, code = _features_dtype("v", v)
        dev, f32 = self.device, self._f32
        keys, gates = lead + (self.key_heads, self.key_dim), lead + (self.heads,)
        return dtype, (self._h, code, _tensor("q", q, keys, dtype, dev), _tensor("k", k, keys, dtype, dev),
                       _tensor("v", v, shape, dtype, dev), _tensor("decay", decay, gates, f32, dev),
                       _tensor("beta", beta, gates, f32, dev), self._scale if scale is None else scale,
                       1 if normalize else 0)

    def delta_rule_state(self):
        """The state before the first token: fp32 zeros [batch, key_dim, K, C]."""
        return self._new(self.memory_shape, self._f32).zero_()

    def delta_rule(self, q, k, v, decay, beta, scale=None, normalize: bool = True, lengths=None, state=None, out=None):
        """Gated delta rule of whole sequences: q and k [batch, N, key_heads,
        key_dim], v [batch, N, K, C] (head h: channels h C / heads and on), decay
        (logarithms) and beta [batch, N, heads] in fp32; scale: 1 / sqrt(key_dim)
        if None; normalize: q and k are taken at norm 1.  Returns (y, state): the
        state [batch, key_dim, K, C] (fp32) after every sequence's last token, for
        delta_rule_step or the next piece (state=)."""
        _, args = self._rule_args(q, k, v, decay, beta, scale, normalize, self.shape[:2], self.shape)
        pl, ps = self._lengths(lengths), _tensor("state", state, self.memory_shape, self._f32, self.device)
        out, po = self._out(out, v, self.shape)
        last = self._new(self.memory_shape, self._f32)
        self._done(self._lib.cgconv_seq_delta_rule(*args, pl, ps, po, last.data_ptr(), self._raw_stream(self.device)))
        return out, last

    def delta_rule_step(self, q, k, v, decay, beta, state, scale=None, normalize: bool = True, out=None):
        """One token of every sequence: q and k [batch, key_heads, key_dim], v
        [batch, K, C], decay and beta [batch, heads]; state is moved on in place.
        Returns y [batch, K, C]."""
        _, args = self._rule_args(q, k, v, decay, beta, scale, normalize, self.shape[:1], self.token_shape)
        ps = _tensor("state", state, self.memory_shape, self._f32, self.device)
        out, po = self._out(out, v, self.token_shape)
        self._done(self._lib.cgconv_seq_delta_rule_step(*args, ps, po, self._raw_stream(self.device)))
        return out

    def delta_rule_backward(self, q, k, v, decay, beta, grad_y, scale=None, normalize: bool = True, lengths=None,
                            state=None, grad_state=None, need=(True,) * 6):
        """Gradients of (q, k, v, decay, beta, state) given those of y and, if
        there is one, of the final state; None where ``need`` is False."""
        if not any(need):
            return (None,) * 6
        dtype, args = self._rule_args(q, k, v, decay, beta, scale, normalize, self.shape[:2], self.shape)
        dev, f32, lead = self.device, self._f32, self.shape[:2]
        args += (self._lengths(lengths), _tensor("state", state, self.memory_shape, f32, dev),
                 _tensor("grad_y", grad_y, self.shape, dtype, dev),
                 _tensor("grad_state", grad_state, self.memory_shape, f32, dev))
        keys, gates = (lead + (self.key_heads, self.key_dim), dtype), (lead + (self.heads,), f32)
        shapes = (keys, keys, (self.shape, dtype), gates, gates, (self.memory_shape, f32))
        grads = tuple(self._new(*s, n) for s, n in zip(shapes, need))
        self._done(self._lib.cgconv_seq_delta_rule_backward(*args, *(None if t is None else t.data_ptr() for t in grads),
                                                            self._raw_stream(dev)))
        return grads

    def close(self):
        if getattr(self, "_h", None):
            cgconv_seq_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_functions = {}


def _whole(grad):
    """An incoming gradient as the entry points take it: contiguous, at a 16-byte
    boundary (that of a part of a concatenation may start anywhere)."""
    grad = grad.contiguous()
    return grad if grad.data_ptr() % 16 == 0 else grad.clone()


def _grad_wanted(*tensors) -> bool:
    import torch
    return torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors)


def _norm_function():
    import torch
    from torch.autograd.function import once_differentiable

    class _NormFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, plan, eps, checkpoint):
            y, *rest = plan.norm(x, weight, bias, eps, checkpoint=checkpoint)
            stats, held = rest[:2], rest[2:] if checkpoint else [x]
            ctx.save_for_backward(weight, *stats, *held)
            ctx.plan = plan
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_y):
            weight, mean, rstd, *held = ctx.saved_tensors
            need = ctx.needs_input_grad
            return ctx.plan.norm_backward(held if len(held) == 2 else held[0], weight, mean, rstd,
                                          _whole(grad_y), need[0], need[1], need[2]) + (None, None, None)

    return _NormFn


def cgconv_norm(x, weight, bias, plan: SequencePlan, eps: float = 1e-5, checkpoint=None):
    """Differentiable layer norm by degree in x, weight and bias (weight and
    bias may be None).  checkpoint="int8": the input is kept for the backward
    pass in 8 bits, written by the forward kernel and read by the backward."""
    wanted = _want_checkpoint(checkpoint) and _grad_wanted(x, weight, bias)
    if "norm" not in _functions:
        _functions["norm"] = _norm_function()
    return _functions["norm"].apply(x, weight, bias, plan, eps, wanted)


def _conv_function():
    import torch
    from torch.autograd.function import once_differentiable

    class _ConvFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, lengths, plan, activation, packed):
            y, _ = plan.conv(x, weight, bias, lengths, activation=activation)
            keep(ctx, packed, (x,), (weight, bias, lengths))
            ctx.plan, ctx.activation = plan, activation
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_y):
            (x,), (weight, bias, lengths) = kept(ctx)
            need = ctx.needs_input_grad
            return ctx.plan.conv_backward(x, weight, bias, _whole(grad_y), lengths, ctx.activation, need[0],
                                          need[1], need[2]) + (None,) * 4

    return _ConvFn


def cgconv_short_conv(x, weight, bias, plan: SequencePlan, lengths=None, activation: bool = True, checkpoint=None):
    """Differentiable short causal convolution (:meth:`SequencePlan.conv`, from
    the zero state) in x, weight and bias (may be None).  checkpoint="int8": x
    is kept for the backward pass in 8 bits."""
    packed = _want_checkpoint(checkpoint) and _grad_wanted(x, weight, bias)
    if "conv" not in _functions:
        _functions["conv"] = _conv_function()
    return _functions["conv"].apply(x, weight, bias, lengths, plan, activation, packed)


def _scan_function():
    import torch
    from torch.autograd.function import once_differentiable

    class _ScanFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, delta, A, Bt, Ct, D, delta_bias, lengths, plan, packed):
            y, _ = plan.scan(x, delta, A, Bt, Ct, D, delta_bias, lengths)
            keep(ctx, packed, (x,), (delta, A, Bt, Ct, D, delta_bias, lengths))
            ctx.plan = plan
            return y

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_y):
            (x,), (delta, A, Bt, Ct, D, delta_bias, lengths) = kept(ctx)
            need = tuple(n and t is not None
                         for n, t in zip(ctx.needs_input_grad, (x, delta, A, Bt, Ct, D, delta_bias)))
            return ctx.plan.scan_backward(x, delta, A, Bt, Ct, D, _whole(grad_y), delta_bias, lengths,
                                          need) + (None,) * 3

    return _ScanFn


def cgconv_scan(x, delta, A, Bt, Ct, D, plan: SequencePlan, delta_bias=None, lengths=None, checkpoint=None):
    """Differentiable selective scan (:meth:`SequencePlan.scan`, from the zero
    state) in all its inputs; D and delta_bias may be None.  checkpoint="int8":
    x is kept for the backward pass in 8 bits (delta, Bt and Ct whole)."""
    packed = _want_checkpoint(checkpoint) and _grad_wanted(x, delta, A, Bt, Ct, D, delta_bias)
    if "scan" not in _functions:
        _functions["scan"] = _scan_function()
    return _functions["scan"].apply(x, delta, A, Bt, Ct, D, delta_bias, lengths, plan, packed)


def _rule_function():
    import torch
    from torch.autograd.function import once_differentiable

    class _RuleFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, decay, beta, state, lengths, plan, scale, normalize, packed):
            y, last = plan.delta_rule(q, k, v, decay, beta, scale, normalize, lengths, state)
            keep(ctx, packed, (v,), (q, k, decay, beta, state, lengths))
            ctx.plan, ctx.scale, ctx.normalize = plan, scale, normalize
            ctx.set_materialize_grads(False)
            return y, last

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_y, grad_state):
            (v,), (q, k, decay, beta, state, lengths) = kept(ctx)
            grad_y = torch.zeros_like(v) if grad_y is None else _whole(grad_y)
            grad_state = None if grad_state is None else _whole(grad_state)
            need = tuple(n and t is not None for n, t in zip(ctx.needs_input_grad, (q, k, v, decay, beta, state)))
            return ctx.plan.delta_rule_backward(q, k, v, decay, beta, grad_y, ctx.scale, ctx.normalize, lengths, state,
                                                grad_state, need) + (None,) * 5

    return _RuleFn


def cgconv_delta_rule(q, k, v, decay, beta, plan: SequencePlan, scale=None, normalize: bool = True, lengths=None,
                      state=None, return_state: bool = False, checkpoint=None):
    """Differentiable gated delta rule (:meth:`SequencePlan.delta_rule`) in q, k,
    v, decay, beta and state; returns y, or (y, the final state), which is then
    differentiable too.  checkpoint="int8": v is kept for the backward pass in 8
    bits (q, k, decay and beta whole)."""
    packed = _want_checkpoint(checkpoint) and _grad_wanted(q, k, v, decay, beta, state)
    if "rule" not in _functions:
        _functions["rule"] = _rule_function()
    y, last = _functions["rule"].apply(q, k, v, decay, beta, state, lengths, plan, scale, normalize, packed)
    return (y, last) if return_state else y


def _residual_function():
    import torch
    from torch.autograd.function import once_differentiable

    class _ResidualFn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, u, gate, post_weight, scale, weight, bias, plan, eps, packed):
            r, y, stats = plan.residual_norm(x, u, gate, post_weight, scale, weight, bias, eps)
            keep(ctx, packed, (x, u), (gate, post_weight, scale, weight, bias, stats))
            ctx.plan = plan
            ctx.set_materialize_grads(False)
            return r, y

        @staticmethod
        @once_differentiable
        def backward(ctx, grad_r, grad_y):
            (x, u), (gate, post_weight, scale, weight, bias, stats) = kept(ctx)
            grad_r = None if grad_r is None else _whole(grad_r)
            grad_y = torch.zeros_like(x) if grad_y is None else _whole(grad_y)
            need = tuple(n and t is not None
                         for n, t in zip(ctx.needs_input_grad, (x, u, gate, post_weight, scale, weight, bias)))
            return ctx.plan.residual_norm_backward(x, u, gate, post_weight, scale, weight, stats, grad_r, grad_y,
                                                   need) + (None,) * 3

    return _ResidualFn


def cgconv_residual_norm(x, u, gate, post_weight, scale, weight, bias, plan: SequencePlan, eps: float = 1e-5,
                         checkpoint=None):
    """Differentiable norms around a residual connection
    (:meth:`SequencePlan.residual_norm`): (r, y).  checkpoint="int8": x and u are
    kept for the backward pass in 8 bits."""
    packed = _want_checkpoint(checkpoint) and _grad_wanted(x, u, gate, post_weight, scale, weight, bias)
    if "residual" not in _functions:
        _functions["residual"] = _residual_function()
    return _functions["residual"].apply(x, u, gate, post_weight, scale, weight, bias, plan, eps, packed)
