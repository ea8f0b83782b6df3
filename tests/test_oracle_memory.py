"""Pins of oracle/memory.py on the CPU: autograd of independent float64 forms,
central differences, the delta rule's own properties (what was written is read
back, rotations, shared key heads, pieces), the norms' from oracle/sequence.py."""

import numpy as np
import pytest

from oracle import memory as M
from oracle import sequence as S


def _rule(seed, B=2, N=7, L=1, H=4, Hk=2, P=3, D=5):
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    return (r.normal(size=(B, N, Hk, D)), r.normal(size=(B, N, Hk, D)), r.normal(size=(B, N, K, H * P)),
            -np.exp(r.normal(size=(B, N, H))), 1 / (1 + np.exp(-r.normal(size=(B, N, H))))), r


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("lengths", [None, [7, 3], [0, 5]])
def test_delta_rule_against_autograd(normalize, lengths):
    import torch
    args, r = _rule(1)
    B, N, Hk, D = args[0].shape
    H, K, C = args[3].shape[-1], args[2].shape[-2], args[2].shape[-1]
    s0, gy, gs = r.normal(size=(B, D, K, C)), r.normal(size=args[2].shape), r.normal(size=(B, D, K, C))
    leaves = [torch.tensor(a, requires_grad=True) for a in args + (s0,)]
    q, k, v, g, b, S0 = leaves
    if normalize:
        q, k = (t / (t.square().sum(-1, keepdim=True) + 1e-6).sqrt() for t in (q, k))
    ys, last = [], []
    for i in range(B):
        end = N if lengths is None else lengths[i]
        state = [S0[i, :, :, h * (C // H):(h + 1) * (C // H)] for h in range(H)]
        rows = []
        for t in range(N):
            if t >= end:
                rows.append(torch.zeros(K, C, dtype=torch.float64))
                continue
            heads = []
            for h in range(H):
                kt, qt = k[i, t, h * Hk // H], q[i, t, h * Hk // H]
                A = torch.exp(g[i, t, h]) * (torch.eye(D, dtype=torch.float64) - b[i, t, h] * torch.outer(kt, kt))
                new = torch.einsum("de,ekp->dkp", A, state[h]) + b[i, t, h] * torch.einsum(
                    "d,kp->dkp", kt, v[i, t, :, h * (C // H):(h + 1) * (C // H)])
                state[h] = new
                heads.append(torch.einsum("d,dkp->kp", qt, new) / D ** 0.5)
            rows.append(torch.cat(heads, -1))
        ys.append(torch.stack(rows))
        last.append(torch.cat(state, -1))
    y, st = torch.stack(ys), torch.stack(last)
    oy, os = M.delta_rule(*args, normalize=normalize, lengths=lengths, state=s0)
    assert np.abs(oy - y.detach().numpy()).max() < 1e-12 and np.abs(os - st.detach().numpy()).max() < 1e-12
    want = torch.autograd.grad((y, st), leaves, (torch.tensor(gy), torch.tensor(gs)))
    got = M.delta_rule_backward(*args, gy, normalize=normalize, lengths=lengths, state=s0, gstate=gs)
    for a, w in zip(got, want):
        assert np.abs(a - w.numpy()).max() < 1e-11


def test_delta_rule_against_differences():
    args, r = _rule(2)
    gy, d = r.normal(size=args[2].shape), [r.normal(size=a.shape) for a in args]
    along = sum((x * y).sum() for x, y in zip(M.delta_rule_backward(*args, gy), d))
    e = 1e-6
    hi, lo = ((M.delta_rule(*(a + s * e * x for a, x in zip(args, d)))[0] * gy).sum() for s in (1, -1))
    assert abs((hi - lo) / (2 * e) - along) <= 1e-7 * max(1, abs(along))


def test_what_a_key_wrote_is_read_back():
    (q, k, v, g, b), _ = _rule(3, N=1)
    y, s = M.delta_rule(k, k, v, 0 * g, np.ones_like(b), scale=1.0)
    assert np.abs(y - v).max() < 1e-5  # |kn|^2 = 1 but for the 1e-6 under the root
    y2, _ = M.delta_rule(k, k, 3 * v, 0 * g, np.ones_like(b), scale=1.0, state=s)  # written over, not added
    assert np.abs(y2 - 3 * v).max() < 1e-5


def test_delta_rule_in_pieces_and_rotated():
    args, r = _rule(4)
    y, s = M.delta_rule(*args)
    y1, s1 = M.delta_rule(*(a[:, :3] for a in args))
    y2, s2 = M.delta_rule(*(a[:, 3:] for a in args), state=s1)
    assert np.abs(np.concatenate([y1, y2], 1) - y).max() < 1e-13 and np.abs(s2 - s).max() < 1e-13
    R, _ = np.linalg.qr(r.normal(size=(3, 3)))
    turn = np.eye(4)
    turn[1:, 1:] = R
    rot = lambda t: np.einsum("km,bnmc->bnkc", turn, t)  # noqa: E731
    assert np.abs(M.delta_rule(args[0], args[1], rot(args[2]), *args[3:])[0] - rot(y)).max() < 1e-12


def _residual(seed, B=2, N=3, L=2, C=5):
    r = np.random.default_rng(seed)
    x = r.normal(size=(B, N, (L + 1) ** 2, C))
    return (x, r.normal(size=x.shape), r.normal(size=(B, N, C)), 1 + 0.3 * r.normal(size=(L + 1, C)), r.normal(size=C),
            1 + 0.3 * r.normal(size=(L + 1, C)), r.normal(size=C)), r.normal(size=x.shape), r.normal(size=x.shape)


@pytest.mark.parametrize("L", [0, 2])
@pytest.mark.parametrize("none", [(), (2,), (3, 4), (2, 3, 4, 5, 6)])
def test_residual_against_differences(L, none):
    args, gr, gy = _residual(5 + L, L=L)
    args = tuple(None if i in none else a for i, a in enumerate(args))
    grads = M.residual_backward(*args, gr, gy, L, 1e-5)
    r = np.random.default_rng(9)
    d = [None if a is None else r.normal(size=a.shape) for a in args]
    along = sum((g * x).sum() for g, x in zip(grads, d) if x is not None)
    loss = lambda s: sum((a * b).sum() for a, b in zip(M.residual(  # noqa: E731
        *(a if a is None else a + s * x for a, x in zip(args, d)), L, 1e-5), (gr, gy)))
    e = 1e-6
    assert abs((loss(e) - loss(-e)) / (2 * e) - along) <= 1e-6 * max(1, abs(along))


def test_residual_without_a_block_is_the_norm():
    args, _, _ = _residual(6)
    x, u, gate, po, sc, w, b = args
    r, y = M.residual(x, u, gate, po, 0 * sc, w, b, 2, 1e-5)
    assert (r == x).all() and np.abs(y - S.norm(x, w, b, 2, 1e-5)).max() < 1e-14
    r, _ = M.residual(0 * x, u, None, None, None, None, None, 2, 1e-5)
    assert np.abs(r - S.norm(u, None, None, 2, 1e-5)).max() < 1e-14


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, out = M.clip(g, 1.0, 0.0)
    assert norm == 5.0 and np.allclose(out[0], [0.6, 0]) and np.allclose(out[1], 0.8)
    assert all((a == b).all() for a, b in zip(M.clip(g, 6.0, 0.0)[1], g))
