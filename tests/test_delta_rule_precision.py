"""How exact the gated delta rule's products in fp32 are: outputs, states and gradients of
every chunk of 64 tokens of every head against float64, beside the same chunks formed in
plain 32-bit products.

The bar is four times the plain form's largest error of a chunk.  Both sum in 32 bits with
roundings of half a step u = 2^-24, in another order; the kernels leave out of every product
m l + l m + l l of two sums of three bfloat16 parts (below 2^-21 of it, 0.7 u on average and
always towards zero), in a chain of six to eight products between an input and a gradient:
at most 8 x 0.7 u = 3.4e-7 on top of the plain form's 1.5e-7 to 5e-7.  A part less, and the errors
are a hundred times the plain form's (the first test, on the CPU).

Errors are relative to the 2-norm of the chunk's values, but for the gradient of beta.  That is
one sum per token, gbeta = sum_c w_c d_c with w = gv / beta and d = v - e^g S^T kn, and if w and d
are off by a share e each and the sum by a share e, gbeta is off by up to 3 e sum_c |w_c d_c|:
of that magnitude, which is not bounded by |gbeta|.  (The last chunk of the second shape has two
tokens; in one of its heads the sums come to 1/239 of their terms' magnitudes, so that an error
of 5e-8 of the terms is 1.2e-5 of the sums.)
"""

import numpy as np
import pytest

from oracle import memory as M
from tests.seq_util import get, put, torch_gpu

CHUNK = 64
NAMES = ("y", "state", "q", "k", "v", "decay", "beta", "first state")
# (B, N, L, C, H, Hk, D): segments with a state, shared keys, partial chunks, widths of 1 to 4
# tiles, of one and two buffers of a chunk, no multiple of eight
SHAPES = [(1, 700, 0, 64, 2, 2, 64), (2, 130, 1, 16, 4, 2, 24), (1, 1100, 0, 144, 1, 1, 100), (1, 200, 0, 128, 1, 1, 128),
          (2, 1000, 0, 24, 2, 1, 20), (1, 90, 0, 100, 1, 1, 65)]
ID = lambda s: "B%dN%dL%dC%dH%dHk%dD%d" % s  # noqa: E731


def _inputs(shape, seed=1):
    B, N, L, C, H, Hk, D = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    f = lambda a: np.asarray(a, np.float32).astype(np.float64)  # noqa: E731
    t = [f(r.normal(size=(B, N, Hk, D))), f(r.normal(size=(B, N, Hk, D))), f(r.normal(size=(B, N, K, C))),
         f(-np.exp(r.normal(size=(B, N, H)) - 3)), f(1 / (1 + np.exp(-r.normal(size=(B, N, H)))))]
    return t, f(r.normal(size=(B, D, K, C))), f(r.normal(size=(B, N, K, C))), f(r.normal(size=(B, D, K, C)))


def _plain(q, k, v, decay, beta, state, product):
    """(y, the last state) by chunks in 32 bits on the CPU; decays are summed in 64."""
    import torch
    B, N, K, C = v.shape
    H, D = decay.shape[-1], q.shape[-1]

    def heads(t):
        t = t * torch.rsqrt((t * t).sum(-1, keepdim=True) + 1e-6)
        return t.repeat_interleave(H // t.shape[2], 2).transpose(1, 2)

    def columns(t):
        return t.reshape(*t.shape[:3], H, C // H).permute(0, 3, 1, 2, 4).reshape(B, H, t.shape[1], -1)

    def back(t):
        return t.reshape(B, H, t.shape[2], K, C // H).permute(0, 2, 3, 1, 4).reshape(B, t.shape[2], K, C)

    q, k, v, S = heads(q), heads(k), columns(v), columns(state)
    decay, beta, ys = decay.transpose(1, 2).double(), beta.transpose(1, 2)[..., None], []
    for c in range(0, N, CHUNK):
        i = slice(c, min(c + CHUNK, N))
        G, one = decay[:, :, i].cumsum(-1), torch.eye(i.stop - c)
        low = torch.ones_like(one).tril()
        f = (G[..., :, None] - G[..., None, :]).masked_fill(low == 0, 0.0).exp().float() * low
        A = beta[:, :, i] * f.tril(-1) * product(k[:, :, i], k[:, :, i].transpose(-1, -2))
        T = torch.linalg.solve_triangular(one + A, one.expand_as(A), upper=False, unitriangular=True)
        e, rest = G.exp().float()[..., None], (G[..., -1:] - G).exp().float()[..., None]
        u = product(T, beta[:, :, i] * (v[:, :, i] - e * product(k[:, :, i], S)))
        inside = f * product(q[:, :, i], k[:, :, i].transpose(-1, -2))
        ys.append(D ** -0.5 * (e * product(q[:, :, i], S) + product(inside, u)))
        S = e[..., -1:, :] * S + product((rest * k[:, :, i]).transpose(-1, -2), u)
    return back(torch.cat(ys, 2)), back(S)


def _magnitudes(t, s, gv):
    """The sums of the magnitudes of the terms of beta's gradient, (B, N, H)."""
    q, k, v, decay, beta = t
    H, states = beta.shape[-1], []
    M.delta_rule(*t, state=s, every=states)
    kn = np.repeat(M.unit(k)[0], H // k.shape[2], 2)
    F = np.exp(decay)[..., None, None] * np.stack(states[:-1], 1)
    d = M.split_heads(v, H) - (kn[..., None] * F).sum(-2)
    return np.abs(M.split_heads(gv, H) / beta[..., None] * d).sum(-1)


def _worst(name, got, ref, H, size=None):
    """The largest error in the 2-norm of a chunk of a head (a state: of a head), relative to
    that of ref or size."""
    size = ref if size is None else size
    got = np.asarray(got, np.float64)
    tokens = [slice(None)] if "state" in name else [slice(c, c + CHUNK) for c in range(0, ref.shape[1], CHUNK)]
    if name in ("q", "k", "decay", "beta"):
        heads = [(slice(None), h) for h in range(ref.shape[2])]
    else:
        P = ref.shape[-1] // H
        heads = [(slice(None), slice(None), slice(h * P, (h + 1) * P)) for h in range(H)]
    worst = 0.0
    for b in range(ref.shape[0]):
        for i in tokens:
            for h in heads:
                off = np.linalg.norm(got[b, i][h] - ref[b, i][h])
                worst = max(worst, float(off / np.linalg.norm(size[b, i][h])))
    return worst


def _bars(shape, t, s, gy, gs, ref, sizes):
    import torch
    leaves = [torch.tensor(x, dtype=torch.float32, requires_grad=True) for x in t + [s]]
    outs = _plain(*leaves, torch.matmul)
    grads = torch.autograd.grad(outs, leaves, [torch.tensor(x, dtype=torch.float32) for x in (gy, gs)])
    return [4 * _worst(n, x.detach().numpy(), r, shape[4], z) for n, x, r, z in
            zip(NAMES, outs + grads, ref, sizes)]


def _parts(x):
    import torch

    def top(y):
        return torch.from_numpy((y.numpy().view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32))
    x = x.contiguous()
    h = top(x)
    m = top(x - h)
    return h.double(), m.double(), (x - h - m).double()


@pytest.mark.parametrize("shape", SHAPES[:2] + SHAPES[3:4], ids=ID)
def test_what_the_parts_give(shape):
    """The six products of three parts are within the bar, the four of two parts far outside."""
    import torch
    t, s, gy, gs = _inputs(shape)
    ref = M.delta_rule(*t, state=s)
    args = [torch.tensor(x, dtype=torch.float32) for x in t + [s]]

    def four(a, b):
        (h, m, _), (H, R, _) = _parts(a), _parts(b)
        return (m @ R + (h @ R + m @ H) + h @ H).float()

    def six(a, b):
        (h, m, k), (H, R, L) = _parts(a), _parts(b)
        return ((h @ L + m @ R + k @ H) + (h @ R + m @ H) + h @ H).float()

    bars = [4 * _worst(n, x.numpy(), r, shape[4]) for n, x, r in zip(NAMES, _plain(*args, torch.matmul), ref)]
    for n, bar, x, z, r in zip(NAMES, bars, _plain(*args, six), _plain(*args, four), ref):
        assert _worst(n, x.numpy(), r, shape[4]) <= bar / 2, n
        assert _worst(n, z.numpy(), r, shape[4]) >= 10 * bar, n


def test_what_a_product_leaves_out():
    """The parts are exact; what is left out has the product's sign and is below 2^-21 of it."""
    import torch
    r = np.random.default_rng(2)
    x, y = (torch.from_numpy(r.normal(size=1 << 20).astype(np.float32)) for _ in range(2))
    x[0] = y[0] = 1 + 2.0 ** -7 - 2.0 ** -23
    a, b = _parts(x), _parts(y)
    assert torch.equal(a[0] + a[1] + a[2], x.double())
    kept = a[0] * b[2] + a[1] * b[1] + a[2] * b[0] + a[0] * b[1] + a[1] * b[0] + a[0] * b[0]
    left = (x.double() * y.double() - kept) / (x.double() * y.double())
    assert float(left.min()) >= 0 and 7.8 * 2.0 ** -24 <= float(left.max()) <= 2.0 ** -21
    assert 0.6 * 2.0 ** -24 <= float(left.mean()) <= 0.8 * 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=ID)
def test_outputs_states_and_gradients(shape):
    torch_gpu()
    import paper_2509_24093_amd as P
    print(f"[gpu] precision {shape}", flush=True)
    B, N, L, C, H, Hk, D = shape
    t, s, gy, gs = _inputs(shape)
    ref = M.delta_rule(*t, state=s) + M.delta_rule_backward(*t, gy, state=s, gstate=gs)
    sizes = [_magnitudes(t, s, ref[4]) if n == "beta" else None for n in NAMES]
    bars = _bars(shape, t, s, gy, gs, ref, sizes)
    plan = P.SequencePlan(B, N, L, C, heads=H, key_heads=Hk, key_dim=D)
    a, first, grad, last = [put(x)[0] for x in t], put(s)[0], put(gy)[0], put(gs)[0]
    got = plan.delta_rule(*a, state=first) + plan.delta_rule_backward(*a, grad, state=first, grad_state=last)
    plan.close()
    off = {n: (_worst(n, get(x), r, H, z), bar) for n, x, r, bar, z in zip(NAMES, got, ref, bars, sizes)}
    print({n: "%.1e of %.1e" % v for n, v in off.items()}, flush=True)
    for n, (e, bar) in off.items():
        assert e <= bar, (n, e, bar)
