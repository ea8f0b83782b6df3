"""Layer norm by degree, 8-bit checkpoints, the short causal convolution and
the selective scan in float64, with their gradients, for the oracle (test
infrastructure only).  Features are (B, N, K, C), K = (L+1)^2.

Norm (d, r, h per token; only the invariants l = 0 are shifted):

    d = x - [l = 0] mean_c x,  r_l = (mean_{m,c} d^2 + eps)^-1/2,  h = d r_l
    y = w[l,c] h + [l = 0] bias[c]

Short convolution, weights (W, L+1, C), tokens before the first from `state`
(the W-1 inputs before it, oldest first) or zero:

    z[t,k,c] = sum_j w[j,l(k),c] x[t-j,k,c] + [k = 0] bias[c]
    y_0 = z_0 sigmoid(z_0) (activation) or z_0,  y_k = z_k

Selective scan, A (C, S), B_t and C_t (B, N, S), state h (B, S, K, C):

    delta = log(1 + exp(raw + bias)),  h_t = exp(delta_t A) h_{t-1} + delta_t B_t x_t
    y_t = sum_s C_t[s] h_t[s] + D x_t

Tokens at and behind a sequence's length: outputs and gradients are zero, the
state is the one after the last token that is there.
"""

from __future__ import annotations

import numpy as np


def degrees(L: int) -> np.ndarray:
    return np.array([l for l in range(L + 1) for _ in range(2 * l + 1)])


def _f64(*arrays):
    return [None if a is None else np.asarray(a, dtype=np.float64) for a in arrays]


# ---- layer norm ------------------------------------------------------------------

def norm_parts(x, L: int, eps: float):
    """(h, mean (B, N), rstd (B, N, L+1))."""
    x, = _f64(x)
    d = x.copy()
    mean = x[:, :, 0].mean(-1)
    d[:, :, 0] -= mean[..., None]
    rstd = np.stack([1 / np.sqrt((d[:, :, l * l:(l + 1) ** 2] ** 2).mean((2, 3)) + eps) for l in range(L + 1)], -1)
    return d * rstd[:, :, degrees(L), None], mean, rstd


def norm(x, weight, bias, L: int, eps: float):
    weight, bias = _f64(weight, bias)
    y = norm_parts(x, L, eps)[0]
    if weight is not None:
        y = y * weight[degrees(L)]
    if bias is not None:
        y[:, :, 0] += bias
    return y


def norm_backward(x, weight, gy, L: int, eps: float, held=None):
    """(gx, gw, gb); held: the values that stand for x in h (a checkpoint),
    under x's own statistics."""
    weight, gy = _f64(weight, gy)
    h, mean, rstd = norm_parts(x, L, eps)
    deg = degrees(L)
    r = rstd[:, :, deg, None]
    if held is not None:
        h = np.asarray(held, dtype=np.float64).copy()
        h[:, :, 0] -= mean[..., None]
        h *= r
    g = gy if weight is None else gy * weight[deg]
    C = gy.shape[-1]
    gx, gw = np.empty_like(gy), np.zeros((L + 1, C))
    for l in range(L + 1):
        s = slice(l * l, (l + 1) ** 2)
        gx[:, :, s] = g[:, :, s] - h[:, :, s] * (g[:, :, s] * h[:, :, s]).mean((2, 3), keepdims=True)
        gw[l] = (gy[:, :, s] * h[:, :, s]).sum((0, 1, 2))
    gx[:, :, 0] -= g[:, :, 0].mean(-1, keepdims=True)
    return gx * r, gw, gy[:, :, 0].sum((0, 1))


# ---- 8-bit checkpoints --------------------------------------------------------------

def pack(x):
    """(codes int8, scale bytes uint8 (..., ceil(C / 32))) of finite x and of
    groups with an infinity or NaN (byte 255, codes 0)."""
    x, = _f64(x)
    C = x.shape[-1]
    codes = np.zeros(x.shape, dtype=np.int8)
    scales = np.zeros(x.shape[:-1] + (-(-C // 32),), dtype=np.uint8)
    for n, c in enumerate(range(0, C, 32)):
        v = x[..., c:c + 32]
        top = np.abs(v).max(-1)
        bad = ~np.isfinite(top)
        e = np.full(top.shape, -126)
        for k in range(-125, 123):  # the smallest that holds
            e = np.where(top > np.ldexp(127.0, k - 1), k, e)
        codes[..., c:c + 32] = np.where(bad[..., None], 0, np.rint(np.ldexp(np.where(bad[..., None], 0, v), -e[..., None])))
        scales[..., n] = np.where(bad, 255, e + 127)
    return codes, scales


def unpack(codes, scales):
    e = np.repeat(scales.astype(np.int64) - 127, 32, axis=-1)[..., :codes.shape[-1]]
    return np.where(e == 128, np.nan, np.ldexp(codes.astype(np.float64), e))


# ---- short causal convolution ---------------------------------------------------------

def _there(B, N, lengths):
    if lengths is None:
        return np.ones((B, N, 1, 1))
    return (np.arange(N)[None] < np.clip(np.asarray(lengths), 0, N)[:, None]).astype(np.float64)[:, :, None, None]


def _conv_sum(x, weight, bias, L, state):
    """z and the padded input (W - 1 rows in front)."""
    B, N, K, C = x.shape
    W = weight.shape[0]
    front = np.zeros((B, W - 1, K, C)) if state is None else state
    row = np.concatenate([front, x], 1)
    w = weight[:, degrees(L)]
    z = sum(w[j] * row[:, W - 1 - j:W - 1 - j + N] for j in range(W))
    if bias is not None:
        z[:, :, 0] += bias
    return z, row


def conv(x, weight, bias, L: int, lengths=None, state=None, activation: bool = True):
    """(y, the last W - 1 inputs of every sequence, oldest first)."""
    x, weight, bias, state = _f64(x, weight, bias, state)
    B, N = x.shape[:2]
    there = _there(B, N, lengths)
    x = x * there
    z, row = _conv_sum(x, weight, bias, L, state)
    if activation:
        z[:, :, 0] /= 1 + np.exp(-z[:, :, 0])
    ends = [N] * B if lengths is None else np.clip(np.asarray(lengths), 0, N)
    W = weight.shape[0]
    return z * there, np.stack([row[b, e:e + W - 1] for b, e in enumerate(ends)])


def conv_backward(x, weight, bias, gy, L: int, lengths=None, activation: bool = True):
    """(gx, gw, gb) from the zero state."""
    x, weight, bias, gy = _f64(x, weight, bias, gy)
    B, N = x.shape[:2]
    W = weight.shape[0]
    there = _there(B, N, lengths)
    x, gz = x * there, gy * there
    z, row = _conv_sum(x, weight, bias, L, None)
    if activation:
        s = 1 / (1 + np.exp(-z[:, :, 0]))
        gz[:, :, 0] *= s * (1 + z[:, :, 0] * (1 - s))
    w = weight[:, degrees(L)]
    behind = np.concatenate([gz, np.zeros((B, W - 1) + gz.shape[2:])], 1)
    gx = sum(w[j] * behind[:, j:j + N] for j in range(W))
    gw = np.zeros_like(weight)
    for j in range(W):
        per = (gz * row[:, W - 1 - j:W - 1 - j + N]).sum((0, 1))
        for l in range(L + 1):
            gw[j, l] = per[l * l:(l + 1) ** 2].sum(0)
    return gx * there, gw, gz[:, :, 0].sum((0, 1))


# ---- selective scan ----------------------------------------------------------------------

def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def scan(x, raw, A, Bt, Ct, D, bias=None, lengths=None, state=None, keep=False):
    """(y, the state after the last token that is there[, every h_t])."""
    x, raw, A, Bt, Ct, D, bias, state = _f64(x, raw, A, Bt, Ct, D, bias, state)
    B, N, K, C = x.shape
    S = A.shape[1]
    there = _there(B, N, lengths)
    delta = softplus(raw if bias is None else raw + bias) * there[..., 0]
    h = np.zeros((B, S, K, C)) if state is None else state.copy()
    y, states = np.zeros_like(x), [h]
    for t in range(N):
        a = np.exp(delta[:, t, None] * A.T)[:, :, None]
        xt = np.where(there[:, t] > 0, x[:, t], 0.0)
        h = a * h + Bt[:, t, :, None, None] * (delta[:, t, None] * xt)[:, None] * there[:, t, None]
        y[:, t] = ((Ct[:, t, :, None, None] * h).sum(1) + (0 if D is None else D * xt)) * there[:, t]
        if keep:
            states.append(h)
    return (y, h, states) if keep else (y, h)


def scan_backward(x, raw, A, Bt, Ct, D, gy, bias=None, lengths=None):
    """Gradients of (x, raw, A, Bt, Ct, D, bias) from the zero state."""
    _, _, states = scan(x, raw, A, Bt, Ct, D, bias, lengths, keep=True)
    x, raw, A, Bt, Ct, D, gy, bias = _f64(x, raw, A, Bt, Ct, D, gy, bias)
    B, N, K, C = x.shape
    there = _there(B, N, lengths)
    x, gy = x * there, gy * there
    v = raw if bias is None else raw + bias
    delta = softplus(v) * there[..., 0]
    gx, gd = np.zeros_like(x), np.zeros_like(raw)
    gA, gB, gC = np.zeros_like(A), np.zeros_like(Bt), np.zeros_like(Ct)
    r = np.zeros_like(states[0])
    for t in reversed(range(N)):
        on = there[:, t, 0, 0]
        d = delta[:, t]
        g = r + Ct[:, t, :, None, None] * gy[:, t, None]
        gC[:, t] = (states[t + 1] * gy[:, t, None]).sum((2, 3)) * on[:, None]
        gB[:, t] = (g * (d[:, None] * x[:, t])[:, None]).sum((2, 3)) * on[:, None]
        into = (Bt[:, t, :, None, None] * g).sum(1)
        gx[:, t] = d[:, None] * into
        r = np.exp(d[:, None] * A.T)[:, :, None] * g
        q = (r * states[t]).sum(2)  # (B, S, C)
        gA += (d[:, None] * q).sum(0).T
        gd[:, t] = ((A.T * q).sum(1) + (into * x[:, t]).sum(1)) * on[:, None]
    if D is not None:
        gx += D * gy
    graw = gd / (1 + np.exp(-v))
    return gx * there, graw, gA, gB, gC, (gy * x).sum((0, 1, 2)), graw.sum((0, 1))
