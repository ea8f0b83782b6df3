"""The gated delta rule, the norms around a residual connection and the clipping
by the global norm in float64, with their gradients, for the oracle (test
infrastructure only).  Features are (B, N, K, C), K = (L+1)^2.

Delta rule, head h of H: P = C / H channels of every component, key head
h Hk / H, state S (D, K P) per sequence and head, token by token:

    kn = k / sqrt(|k|^2 + 1e-6), qn alike (normalize), F = exp(decay) S
    u = beta (v - F^T kn),  S' = F + kn u^T,  y = scale S'^T qn

Residual connection (norms by degree without weights, see oracle/sequence.py):

    r = x + scale silu(gate) post_weight norm(u),  y = weight norm(r) + bias

Clipping: out = g min(1, max_norm / (norm + eps)), norm over all tensors.
"""

from __future__ import annotations

import numpy as np

from oracle.sequence import _f64, degrees, norm_backward, norm_parts

KEY_EPS = 1e-6


# ---- gated delta rule ---------------------------------------------------------------

def split_heads(t, H: int):
    """(..., K, C) as (..., H, K P)."""
    *lead, K, C = t.shape
    t = t.reshape(*lead, K, H, C // H)
    return np.moveaxis(t, -2, -3).reshape(*lead, H, K * (C // H))


def join_heads(t, K: int):
    *lead, H, V = t.shape
    t = t.reshape(*lead, H, K, V // K)
    return np.moveaxis(t, -3, -2).reshape(*lead, K, H * (V // K))


def unit(t, normalize: bool = True):
    """(t at norm 1, the factor)."""
    f = 1 / np.sqrt((t * t).sum(-1, keepdims=True) + KEY_EPS) if normalize else np.ones(t.shape[:-1] + (1,))
    return t * f, f


def _rule_inputs(q, k, v, decay, beta, normalize):
    q, k, v, decay, beta = _f64(q, k, v, decay, beta)
    H, each = decay.shape[-1], decay.shape[-1] // q.shape[-2]
    qn, kn = (np.repeat(unit(t, normalize)[0], each, -2) for t in (q, k))
    return qn, kn, split_heads(v, H), np.exp(decay), beta


def _ends(B, N, lengths):
    return np.full(B, N) if lengths is None else np.clip(np.asarray(lengths), 0, N)


def delta_rule(q, k, v, decay, beta, scale=None, normalize=True, lengths=None, state=None, every=None):
    """(y, the last state (B, D, K, C)).  q, k (B, N, Hk, D), decay and beta
    (B, N, H); every: a list that receives the states (B, H, D, V) before every
    token and the last."""
    qn, kn, vh, a, b = _rule_inputs(q, k, v, decay, beta, normalize)
    B, N, H, D = kn.shape
    K = v.shape[-2]
    scale = D ** -0.5 if scale is None else scale
    S = np.zeros((B, H, D, vh.shape[-1])) if state is None else np.moveaxis(split_heads(_f64(state)[0], H), 1, 2).copy()
    ends, y = _ends(B, N, lengths), np.zeros_like(vh)
    for t in range(N):
        on = np.flatnonzero(t < ends)
        if every is not None:
            every.append(S.copy())
        F = a[on, t][..., None, None] * S[on]
        u = b[on, t][..., None] * (vh[on, t] - (kn[on, t][..., None] * F).sum(-2))
        S[on] = F + kn[on, t][..., None] * u[..., None, :]
        y[on, t] = scale * (qn[on, t][..., None] * S[on]).sum(-2)
    if every is not None:
        every.append(S.copy())
    return join_heads(y, K), join_heads(np.moveaxis(S, 1, 2), K)


def delta_rule_backward(q, k, v, decay, beta, gy, scale=None, normalize=True, lengths=None, state=None, gstate=None):
    """Gradients of (q, k, v, decay, beta, state)."""
    states = []
    delta_rule(q, k, v, decay, beta, scale, normalize, lengths, state, states)
    qn, kn, vh, a, b = _rule_inputs(q, k, v, decay, beta, normalize)
    q, k, gy = _f64(q, k, gy)
    B, N, H, D = kn.shape
    K, Hk = v.shape[-2], q.shape[-2]
    scale = D ** -0.5 if scale is None else scale
    G = np.zeros_like(states[0]) if gstate is None else np.moveaxis(split_heads(_f64(gstate)[0], H), 1, 2).copy()
    g, ends = split_heads(gy, H), _ends(B, N, lengths)
    gq, gk, gv = np.zeros_like(qn), np.zeros_like(kn), np.zeros_like(vh)
    ga, gb = np.zeros_like(a), np.zeros_like(b)
    for t in reversed(range(N)):
        on = np.flatnonzero(t < ends)
        kt, bt, gt = kn[on, t][..., None], b[on, t][..., None], g[on, t][..., None, :]
        F = a[on, t][..., None, None] * states[t][on]
        left = vh[on, t] - (kt * F).sum(-2)
        u = bt * left
        gS = G[on] + scale * qn[on, t][..., None] * gt
        gq[on, t] = scale * (states[t + 1][on] * gt).sum(-1)
        gu = (gS * kt).sum(-2)
        gb[on, t] = (gu * left).sum(-1)
        gv[on, t] = bt * gu
        gk[on, t] = (gS * u[..., None, :]).sum(-1) - (F * gv[on, t][..., None, :]).sum(-1)
        gF = gS - kt * gv[on, t][..., None, :]
        ga[on, t] = (gF * F).sum((-1, -2))
        G[on] = a[on, t][..., None, None] * gF
    each = H // Hk
    out = []
    for x, gx in ((q, gq), (k, gk)):
        n, f = unit(x, normalize)
        gx = gx.reshape(B, N, Hk, each, D).sum(3)
        out.append(f * (gx - n * (n * gx).sum(-1, keepdims=True)) if normalize else gx)
    return out[0], out[1], join_heads(gv, K), ga, gb, join_heads(np.moveaxis(G, 1, 2), K)


# ---- norms around a residual connection -----------------------------------------------

def _silu(z):
    return z / (1 + np.exp(-z))


def residual(x, u, gate, post_weight, scale, weight, bias, L: int, eps: float):
    """(r, y)."""
    x, u, gate, post_weight, scale, weight, bias = _f64(x, u, gate, post_weight, scale, weight, bias)
    deg = degrees(L)
    p = norm_parts(u, L, eps)[0]
    p = p * (1 if post_weight is None else post_weight[deg]) * (1 if scale is None else scale)
    if gate is not None:
        p = p * _silu(gate)[:, :, None]
    r = x + p
    y = norm_parts(r, L, eps)[0] * (1 if weight is None else weight[deg])
    if bias is not None:
        y[:, :, 0] += bias
    return r, y


def residual_backward(x, u, gate, post_weight, scale, weight, bias, gr, gy, L: int, eps: float):
    """Gradients of (x, u, gate, post_weight, scale, weight, bias); of parameters
    that are None as if they were ones and zeros, of a gate that is None: None."""
    x, u, gate, post_weight, scale, weight, gr, gy = _f64(x, u, gate, post_weight, scale, weight, gr, gy)
    deg, C = degrees(L), x.shape[-1]
    po = np.ones((L + 1, C)) if post_weight is None else post_weight
    sc = np.ones(C) if scale is None else scale
    s = np.ones(x.shape[:2] + (C,)) if gate is None else _silu(gate)
    r, _ = residual(x, u, gate, po, sc, weight, None, L, eps)
    G, gw, gb = norm_backward(r, weight, gy, L, eps)
    G = G + (0 if gr is None else gr)
    h = norm_parts(u, L, eps)[0]
    inner = G * h
    Q = np.stack([(inner * s[:, :, None])[:, :, l * l:(l + 1) ** 2].sum((0, 1, 2)) for l in range(L + 1)])
    gu, _, _ = norm_backward(u, po, G * s[:, :, None] * sc, L, eps)
    ggate = None
    if gate is not None:
        sig = 1 / (1 + np.exp(-gate))
        ggate = sig * (1 + gate * (1 - sig)) * sc * (inner * po[deg]).sum(2)
    return G, gu, ggate, Q * sc, (Q * po).sum(0), gw, gb


# ---- clipping ----------------------------------------------------------------------------

def clip(grads, max_norm: float, eps: float):
    grads = _f64(*grads)
    norm = np.sqrt(sum((g * g).sum() for g in grads))
    factor = min(1.0, max_norm / (norm + eps))
    return norm, [g * factor for g in grads]
