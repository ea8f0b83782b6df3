"""Pins of oracle/sequence.py on the CPU: torch's layer norm and autograd of
independent float64 forms, central differences, brute force over the
definitions, equivariance, and the checkpoint format's properties."""

import numpy as np
import pytest

from oracle import sequence as S


def _rng(seed):
    return np.random.default_rng(seed)


def _directional(f, args, which, grad, seed, eps=1e-6):
    """Central difference of f along a random direction of args[which]."""
    d = _rng(seed).normal(size=args[which].shape)
    hi, lo = list(args), list(args)
    hi[which], lo[which] = args[which] + eps * d, args[which] - eps * d
    num = (f(*hi) - f(*lo)) / (2 * eps)
    assert abs(num - (grad * d).sum()) <= 1e-6 * max(1.0, abs(num))


def test_norm_of_scalars_is_torchs_layer_norm():
    import torch
    r = _rng(1)
    x, w, b = r.normal(size=(2, 5, 1, 7)) + 3, r.normal(size=(1, 7)), r.normal(size=7)
    xt, wt, bt = (torch.tensor(a, requires_grad=True) for a in (x, w, b))
    y = torch.nn.functional.layer_norm(xt, (7,), wt[0], bt, 1e-5)
    assert np.abs(S.norm(x, w, b, 0, 1e-5) - y.detach().numpy()).max() < 1e-12
    g = r.normal(size=x.shape)
    ref = torch.autograd.grad(y, (xt, wt, bt), torch.tensor(g))
    for a, c in zip(S.norm_backward(x, w, g, 0, 1e-5), ref):
        assert np.abs(a - c.numpy()).max() < 1e-12


@pytest.mark.parametrize("L", [0, 1, 3])
def test_norm_gradients_against_differences(L):
    r = _rng(10 + L)
    K = (L + 1) ** 2
    x, w, b, g = r.normal(size=(2, 3, K, 5)), r.normal(size=(L + 1, 5)), r.normal(size=5), r.normal(size=(2, 3, K, 5))
    grads = S.norm_backward(x, w, g, L, 1e-3)
    for i in range(3):
        _directional(lambda *a: (S.norm(*a, L, 1e-3) * g).sum(), [x, w, b], i, grads[i], 20 + i)


def test_norm_commutes_with_rotations():
    from oracle.sh import random_rotation, wigner_D_real
    L = 3
    r = _rng(3)
    x = r.normal(size=(1, 2, (L + 1) ** 2, 4))
    q = random_rotation(r)
    D = wigner_D_real(L, q, r)

    def turn(v):
        out = v.copy()
        for l in range(L + 1):
            s = slice(l * l, (l + 1) ** 2)
            out[:, :, s] = np.einsum("ab,tnbc->tnac", D[l], v[:, :, s])
        return out

    w, b = r.normal(size=(L + 1, 4)), r.normal(size=4)
    assert np.abs(S.norm(turn(x), w, b, L, 1e-5) - turn(S.norm(x, w, b, L, 1e-5))).max() < 1e-9


def test_pack_format():
    r = _rng(4)
    x = (r.normal(size=(6, 77)) * np.exp(r.normal(size=(6, 1)) * 20)).astype(np.float32)
    codes, scales = S.pack(x)
    back = S.unpack(codes, scales)
    for c in range(0, 77, 32):
        top = np.abs(x[:, c:c + 32].astype(np.float64)).max(-1)
        s = np.ldexp(1.0, scales[:, c // 32].astype(int) - 127)
        assert (top <= 127 * s).all() and (top > 127 * s / 2).all()
        assert (np.abs(back[:, c:c + 32] - x[:, c:c + 32]).max(-1) <= s / 2).all()
    again, sc2 = S.pack(back)
    assert (S.unpack(again, sc2) == back).all()  # what 8 bits hold is kept
    # borders: 127 keeps scale 1, the next float needs 2; zeros; the smallest scale
    v = np.array([[127.0], [np.nextafter(np.float32(127), np.float32(200))], [0.0], [1e-45], [3.4028235e38]])
    codes, scales = S.pack(v)
    assert scales[:, 0].tolist() == [127, 128, 1, 1, 127 + 122]
    assert codes[:, 0].tolist() == [127, 64, 0, 0, 64]
    codes, scales = S.pack(np.array([[1.0, np.inf], [np.nan, 0.0], [2.0, 3.0]]))
    assert scales[:, 0].tolist() == [255, 255, 127 - 5] and np.isnan(S.unpack(codes, scales)[:2]).all()


def _conv_brute(x, w, b, L, lengths, state, activation):
    B, N, K, C = x.shape
    W, deg = w.shape[0], S.degrees(L)
    y = np.zeros_like(x)
    for n in range(B):
        for t in range(min(N, lengths[n])):
            for k in range(K):
                z = np.zeros(C)
                for j in range(W):
                    if t - j >= 0:
                        z += w[j, deg[k]] * x[n, t - j, k]
                    elif state is not None:
                        z += w[j, deg[k]] * state[n, W - 1 + t - j, k]
                if k == 0:
                    z = z + b
                    if activation:
                        z = z / (1 + np.exp(-z))
                y[n, t, k] = z
    return y


@pytest.mark.parametrize("activation", [True, False])
def test_conv_against_brute_force_and_differences(activation):
    r = _rng(5)
    L, W, C, N = 1, 3, 2, 6
    lengths = [6, 1, 0]
    x, w, b = r.normal(size=(3, N, 4, C)), r.normal(size=(W, 2, C)), r.normal(size=C)
    state = r.normal(size=(3, W - 1, 4, C))
    y, last = S.conv(x, w, b, L, lengths, state, activation)
    assert np.abs(y - _conv_brute(x, w, b, L, lengths, state, activation)).max() < 1e-13
    assert (last[0] == x[0, 4:6]).all() and (last[2] == state[2]).all()
    assert (last[1][0] == state[1, 1]).all() and (last[1][1] == x[1, 0]).all()
    # a prompt in two pieces is the prompt
    y1, s1 = S.conv(x[:1, :2], w, b, L, None, state[:1], activation)
    y2, s2 = S.conv(x[:1, 2:], w, b, L, None, s1, activation)
    assert np.abs(np.concatenate([y1, y2], 1) - y[:1]).max() < 1e-13 and (s2 == last[:1]).all()
    g = r.normal(size=x.shape)
    grads = S.conv_backward(x, w, b, g, L, lengths, activation)
    for i in range(3):
        _directional(lambda *a: (S.conv(*a, L, lengths, None, activation)[0] * g).sum(), [x, w, b], i, grads[i], 30 + i)


def test_scan_against_its_closed_sum_and_differences():
    r = _rng(6)
    B, N, K, C, St = 3, 5, 4, 2, 3
    lengths = [5, 2, 0]
    x, raw, bias, D = r.normal(size=(B, N, K, C)), r.normal(size=(B, N, C)), r.normal(size=C), r.normal(size=C)
    A, Bt, Ct = -np.exp(r.normal(size=(C, St))), r.normal(size=(B, N, St)), r.normal(size=(B, N, St))
    h0 = r.normal(size=(B, St, K, C))
    y, last = S.scan(x, raw, A, Bt, Ct, D, bias, lengths, h0)
    delta = np.log(1 + np.exp(raw + bias))
    for b in range(B):
        for t in range(lengths[b]):
            ref = D * x[b, t]
            for s in range(St):
                h = np.exp(A[:, s] * delta[b, :t + 1].sum(0)) * h0[b, s]
                for i in range(t + 1):
                    h = h + np.exp(A[:, s] * delta[b, i + 1:t + 1].sum(0)) * delta[b, i] * Bt[b, i, s] * x[b, i]
                ref = ref + Ct[b, t, s] * h
                if t == lengths[b] - 1:
                    assert np.abs(last[b, s] - h).max() < 1e-12
            assert np.abs(y[b, t] - ref).max() < 1e-12
    assert (last[2] == h0[2]).all() and (y[1, 2:] == 0).all()
    g = r.normal(size=x.shape)
    grads = S.scan_backward(x, raw, A, Bt, Ct, D, g, bias, lengths)

    def f(x, raw, A, Bt, Ct, D, bias):
        return (S.scan(x, raw, A, Bt, Ct, D, bias, lengths)[0] * g).sum()

    args = [x, raw, A, Bt, Ct, D, bias]
    for i in range(7):
        _directional(f, args, i, grads[i], 40 + i)
