"""GPU parity of the gated delta rule (whole sequences, single tokens, gradients)
against the float64 oracle.

Bounds, per column of the states in the 2-norm.  With keys of norm 1 and betas in 0..2 a
token shrinks an error of the state by its decay a; it adds its own.  A value u that a
token writes is a sum of up to 64 products of two triangles' entries, each a sum over up
to 64 tokens of sums over D: D + 232 roundings (3 x 64 for the triangles, 40 for norms,
decays and the rest) of magnitudes that the triangles amplify at most by k = |T| (1 +
|A|) in the row-sum norm, T = (1 + A)^-1 (_Bound):

    e_t = a_t (e_{t-1} + 64 u |S_{t-1}|) + (D + 232) u k beta_t (|v_t| + a_t |S_{t-1}|)
    error of y_t = scale |qn| (e_t + (D + 232) u |S_t|),    u = 2^-24

Gradients pass the same recursions backwards; there independent roundings add as their
root: relative to the tensor's 2-norm 4 k sqrt(N (D + 256)) u, four for the ratio of a
gradient's terms to their sum.  To it comes an output's own rounding.
"""

import numpy as np
import pytest

from oracle import memory as M
from tests.conftest import rel_l2
from tests.seq_util import HALF, U, get, put, torch_gpu

pytestmark = pytest.mark.gpu

# (B, N, L, C, H, Hk, D): one token, key and channel; key widths on both sides of every tile
# of 32 and no multiple of 8; chunks of 64 with partial last ones; heads that share keys;
# columns in one to several tiles and blocks, none a multiple; several components; segments
SHAPES = [(1, 1, 0, 1, 1, 1, 1), (2, 5, 0, 6, 3, 1, 4), (1, 64, 0, 16, 1, 1, 32), (1, 65, 0, 16, 1, 1, 33),
          (2, 63, 2, 6, 2, 2, 24), (3, 130, 1, 12, 4, 2, 7), (1, 200, 0, 160, 4, 2, 64), (1, 129, 0, 130, 1, 1, 128),
          (1, 100, 3, 4, 1, 1, 96), (2, 37, 0, 72, 9, 3, 65), (1, 70, 0, 300, 1, 1, 40), (1, 80, 4, 16, 2, 1, 16),
          (2, 1000, 0, 24, 2, 1, 20), (1, 700, 0, 144, 1, 1, 100), (1, 1100, 0, 144, 1, 1, 100), (1, 1030, 0, 40, 1, 1, 64),
          (2, 1090, 1, 24, 2, 1, 90), (1, 2100, 0, 16, 1, 1, 32)]


def _inputs(shape, dtype, seed, ragged=False):
    B, N, L, C, H, Hk, D = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    t = [put(r.normal(size=(B, N, Hk, D)), dtype), put(r.normal(size=(B, N, Hk, D)), dtype),
         put(r.normal(size=(B, N, K, C)), dtype), put(-np.exp(2 * r.normal(size=(B, N, H)) - 2)),
         put(1 / (1 + np.exp(-r.normal(size=(B, N, H)))))]
    state, gy, gs = put(r.normal(size=(B, D, K, C))), put(r.normal(size=(B, N, K, C)), dtype), put(r.normal(size=(B, D, K, C)))
    lengths = None
    if ragged:
        lengths = r.integers(0, N + 1, size=B)
        lengths[0] = N if B > 1 else max(1, N - 3)
        if B > 2:
            lengths[1] = 0
    return t, state, gy, gs, lengths


def _plan(P, shape, **kw):
    B, N, L, C, H, Hk, D = shape
    return P.SequencePlan(B, N, L, C, heads=H, key_heads=Hk, key_dim=D, **kw)


def _amplification(kn, decay, beta):
    """k of every chunk's tokens (B, N, H)."""
    B, N, H, _ = kn.shape
    out = np.ones((B, N, H))
    for b in range(B):
        for h in range(H):
            for c in range(0, N, 64):
                s = slice(c, min(c + 64, N))
                G = np.cumsum(np.maximum(decay[b, s, h], -1e3))
                A = np.tril(beta[b, s, h, None] * np.exp(np.minimum(G[:, None] - G[None], 0)) * (kn[b, s, h] @ kn[b, s, h].T), -1)
                T = np.linalg.inv(np.eye(len(A)) + A)
                out[b, s, h] = np.abs(T).sum(1).max() * (1 + np.abs(A).sum(1).max())
    return out


class _Bound:
    """Errors of y and of the last state, (B, N, K, C) and (B, D, K, C)."""

    def __init__(self, q, k, v, decay, beta, scale, state, normalize=True):
        B, N, K, C = v.shape
        H, D = decay.shape[-1], q.shape[-1]
        each = H // q.shape[-2]
        qn, kn = (np.repeat(M.unit(t, normalize)[0], each, -2) for t in (q, k))
        self.k = _amplification(kn, decay, beta)
        states = []
        M.delta_rule(q, k, v, decay, beta, scale, normalize, None, state, states)
        vh, a = np.abs(M.split_heads(v, H)), np.exp(decay)
        e = np.zeros((B, H, vh.shape[-1]))
        y = np.zeros(vh.shape)
        for t in range(N):
            f, at, bt = np.sqrt((states[t] ** 2).sum(-2)), a[:, t, :, None], np.abs(beta[:, t, :, None])
            e = at * (e + 64 * U * f) + (D + 232) * U * self.k[:, t, :, None] * bt * (vh[:, t] + at * f)
            g = np.sqrt((states[t + 1] ** 2).sum(-2))
            y[:, t] = scale * np.sqrt((qn[:, t] ** 2).sum(-1))[..., None] * (e + (D + 232) * U * g)
        self.y = M.join_heads(y, K)
        self.state = np.broadcast_to(M.join_heads(e[:, None], K), (B, D, K, C)) + U * np.abs(
            M.join_heads(np.moveaxis(states[-1], 1, 2), K))


def _near(name, got, ref, bound, dtype):
    got = get(got)
    assert np.isfinite(got).all(), name
    bound = bound + HALF[dtype] * (np.abs(ref) + bound) + 1e-30
    worst = float(np.max(np.abs(got - ref) / bound))
    assert worst <= 1.0, f"{name}: {worst:.3g} of the bound"


def _bar(shape, k, dtype):
    _, N, _, _, _, _, D = shape
    return 4 * float(k.max()) * np.sqrt(N * (D + 256)) * U + HALF[dtype]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%dN%dL%dC%dH%dHk%dD%d" % s)
def test_outputs_states_and_gradients(shape, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    print(f"[gpu] delta rule {shape} {dtype}", flush=True)
    t, (s, sv), (gy, gyv), (gs, gsv), _ = _inputs(shape, dtype, sum(shape))
    (a, av) = zip(*t)
    D = shape[-1]
    plan = _plan(P, shape)
    y, last = plan.delta_rule(*a)
    y2, last2 = plan.delta_rule(*a, state=s, scale=0.7)
    grads = plan.delta_rule_backward(*a, gy, state=s, grad_state=gs, scale=0.7)
    plain = plan.delta_rule_backward(*a, gy)
    again = plan.delta_rule_backward(*a, gy)
    only = plan.delta_rule_backward(*a, gy, need=(False, False, True, False, False, False))
    some = plan.delta_rule_backward(*a, gy, need=(True, False, False, False, True, False))
    torch.cuda.synchronize()
    plan.close()
    for yy, ll, scale, state in ((y, last, D ** -0.5, None), (y2, last2, 0.7, sv)):
        b = _Bound(*av, scale, state)
        ry, rs = M.delta_rule(*av, scale, state=state)
        _near("y", yy, ry, b.y, dtype)
        _near("state", ll, rs, b.state, "fp32")
    k = b.k
    names = ("q", "k", "v", "decay", "beta", "state")
    for got, ref in ((grads, M.delta_rule_backward(*av, gyv, 0.7, state=sv, gstate=gsv)),
                     (plain, M.delta_rule_backward(*av, gyv))):
        for n, x, r in zip(names, got, ref):
            if np.linalg.norm(r) == 0 or (D == 1 and n in "qk"):  # a key of one number at norm 1 has none to speak of
                assert np.abs(get(x) - r).max() <= 1e-4, n
                continue
            bar = _bar(shape, k, dtype if n in ("q", "k", "v") else "fp32")
            assert rel_l2(get(x), r) <= bar, (n, rel_l2(get(x), r), bar)
    assert all(torch.equal(x, z) for x, z in zip(plain, again))  # the order of the sums is fixed
    assert torch.equal(only[2], plain[2]) and only[0] is None and only[5] is None
    assert torch.equal(some[0], plain[0]) and torch.equal(some[4], plain[4]) and some[1] is None


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 130, 1, 12, 4, 2, 7), (4, 70, 0, 40, 2, 1, 64), (3, 900, 0, 32, 2, 2, 24)],
                         ids=lambda s: "B%dN%dL%dC%dH%dHk%dD%d" % s)
def test_lengths(shape, dtype):
    """What stands behind the lengths reaches nothing; outputs and gradients there are
    zero; the state is the one behind the last token."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    t, (s, sv), (gy, gyv), (gs, gsv), n = _inputs(shape, dtype, 7, ragged=True)
    (a, av) = zip(*t)
    plan = _plan(P, shape)
    lengths = torch.tensor(n, dtype=torch.int32, device="cuda")
    clean = plan.delta_rule(*a, lengths=lengths, state=s) + plan.delta_rule_backward(
        *a, gy, lengths=lengths, state=s, grad_state=gs)
    ref = M.delta_rule(*av, lengths=n, state=sv) + M.delta_rule_backward(*av, gyv, lengths=n, state=sv, gstate=gsv)
    k = _Bound(*av, 1.0, sv).k
    for x, r in zip(clean, ref):
        assert rel_l2(get(x), r) <= _bar(shape, k, dtype)
    for b, e in enumerate(n):
        for x in (clean[0],) + clean[2:7]:
            assert (x[b, e:] == 0).all()
        if e == 0:
            assert torch.equal(clean[1][b], s[b]) and torch.equal(clean[7][b], gs[b])
    for fill in (float("nan"), float("inf"), -float("inf")):
        bad = [x.clone() for x in a + (gy,)]
        for x in bad:
            for b, e in enumerate(n):
                x[b, e:] = fill
        got = plan.delta_rule(*bad[:5], lengths=lengths, state=s) + plan.delta_rule_backward(
            *bad, lengths=lengths, state=s, grad_state=gs)
        assert all(torch.equal(x, z) for x, z in zip(got, clean)), fill
    # lengths outside 0..N count as the nearest of them
    far = torch.tensor([2 ** 31 - 1, -5] + [-2 ** 31] * (shape[0] - 2), dtype=torch.int32, device="cuda")
    near = torch.tensor([shape[1], 0] + [0] * (shape[0] - 2), dtype=torch.int32, device="cuda")
    assert all(torch.equal(x, z) for x, z in zip(plan.delta_rule(*a, lengths=far), plan.delta_rule(*a, lengths=near)))
    plan.close()


def test_extreme_gates_and_keys():
    """Decays of minus infinity (a state forgotten), of zero, betas of 0, 1 and 2, keys of
    zero, the same key in every token, keys far from norm 1: finite where the oracle is."""
    torch_gpu()
    import paper_2509_24093_amd as P
    shape = (1, 150, 0, 32, 2, 2, 16)
    t, (s, sv), (gy, gyv), (gs, gsv), _ = _inputs(shape, "fp32", 3)
    (a, av) = map(list, zip(*t))
    plan = _plan(P, shape)

    def check(tag):
        for i in range(5):
            av[i] = get(a[i])
        with np.errstate(under="ignore"):
            ref = M.delta_rule(*av, state=sv) + M.delta_rule_backward(*av, gyv, state=sv, gstate=gsv)
        got = plan.delta_rule(*a, state=s) + plan.delta_rule_backward(*a, gy, state=s, grad_state=gs)
        b = _Bound(*av, 0.25, sv)
        _near(tag + " y", got[0], ref[0], b.y, "fp32")
        _near(tag + " state", got[1], ref[1], b.state, "fp32")
        for n, x, r in zip(("q", "k", "v", "decay", "beta", "state"), got[2:], ref[2:]):
            assert np.isfinite(get(x)).all(), (tag, n)
            # relative to the largest gradient of a token: a forgotten state leaves some at zero
            assert np.abs(get(x) - r).max() <= _bar(shape, b.k, "fp32") * np.abs(r).max() * 8 + 1e-30, (tag, n)

    check("ordinary")
    keep = [x.clone() for x in a]
    a[3][:, ::7] = -float("inf")
    a[3][:, 1::7] = -1e30
    a[3][:, 2::7] = -120.0
    check("forgotten")
    a[3].zero_()
    check("kept")
    a[3].copy_(keep[3])
    for beta in (0.0, 1.0, 2.0):
        a[4].fill_(beta)
        check(f"beta {beta}")
    a[4].copy_(keep[4])
    a[1][:, 3::5] = 0
    a[0][:, 4::5] = 0
    check("zero keys")
    a[0].copy_(keep[0] * 1e4)
    a[1].copy_(keep[1] * 1e4)
    check("large keys")
    a[0].copy_(keep[0])
    a[1].copy_(keep[1][:, :1].expand_as(a[1]))
    check("one key")
    plan.close()


def test_without_norm():
    torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 90, 1, 12, 4, 2, 24)
    t, (s, sv), (gy, gyv), (gs, gsv), _ = _inputs(shape, "fp32", 5)
    (a, av) = map(list, zip(*t))
    for i in (0, 1):  # keys within norm 1
        a[i] = (a[i] / (a[i].norm(dim=-1, keepdim=True) * 1.5)).contiguous()
        av[i] = get(a[i])
    plan = _plan(P, shape)
    y, last = plan.delta_rule(*a, normalize=False, state=s)
    grads = plan.delta_rule_backward(*a, gy, normalize=False, state=s, grad_state=gs)
    plan.close()
    b = _Bound(*av, 24 ** -0.5, sv, normalize=False)
    ry, rs = M.delta_rule(*av, normalize=False, state=sv)
    _near("y", y, ry, b.y, "fp32")
    _near("state", last, rs, b.state, "fp32")
    for x, r in zip(grads, M.delta_rule_backward(*av, gyv, normalize=False, state=sv, gstate=gsv)):
        assert rel_l2(get(x), r) <= _bar(shape, b.k, "fp32")


STEPS = [(1, 0, 1, 1, 1, 1), (3, 0, 6, 3, 1, 4), (2, 1, 12, 4, 2, 7), (5, 0, 128, 1, 1, 128), (64, 0, 256, 4, 2, 64),
         (2, 3, 20, 4, 4, 33), (1, 6, 24, 3, 1, 100), (130, 2, 8, 2, 2, 16), (7, 0, 2048, 16, 8, 128)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("step", STEPS, ids=lambda s: "B%dL%dC%dH%dHk%dD%d" % s)
def test_step(step, dtype):
    torch_gpu()
    import paper_2509_24093_amd as P
    B, L, C, H, Hk, D = step
    shape = (B, 1, L, C, H, Hk, D)
    t, (s, sv), _, _, _ = _inputs(shape, dtype, 11 + sum(step))
    (a, av) = zip(*t)
    for normalize, scale in ((True, None), (False, 0.5)):
        if not normalize:
            av = tuple(x / (3 * np.sqrt(D)) if i < 2 else x for i, x in enumerate(av))
            a = tuple(put(x, dtype)[0] if i < 2 else z for i, (x, z) in enumerate(zip(av, a)))
            av = tuple(get(z) if i < 2 else x for i, (x, z) in enumerate(zip(av, a)))
        plan = _plan(P, shape, backward=False)
        state = s.clone()
        y = plan.delta_rule_step(*(x[:, 0].contiguous() for x in a), state, scale=scale, normalize=normalize)
        plan.close()
        b = _Bound(*av, D ** -0.5 if scale is None else scale, sv, normalize)
        ry, rs = M.delta_rule(*av, scale, normalize, state=sv)
        _near("y", y, ry[:, 0], b.y[:, 0], dtype)
        _near("state", state, rs, b.state, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_prompt_pieces_and_tokens(dtype):
    """A padded batch of prompts in two pieces, then token by token: the whole."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 150, 1, 16, 4, 2, 32)
    t, _, _, _, _ = _inputs(shape, dtype, 13)
    (a, av) = zip(*t)
    whole, piece = _plan(P, shape), _plan(P, (2, 70) + shape[2:], backward=False)
    one = _plan(P, (2, 1) + shape[2:], backward=False)
    b = _Bound(*av, 32 ** -0.5, None)
    y, last = whole.delta_rule(*a)
    y1, s1 = piece.delta_rule(*(x[:, :70].contiguous() for x in a))
    n = torch.tensor([70, 41], dtype=torch.int32, device="cuda")
    y2, state = piece.delta_rule(*(x[:, 70:140].contiguous() for x in a), lengths=n, state=s1)
    ry, rs = M.delta_rule(*av)
    _near("first piece", y1, ry[:, :70], b.y[:, :70], dtype)
    for i, e in enumerate((70, 41)):
        _near("second piece", y2[i, :e], ry[i, 70:70 + e], b.y[i, 70:70 + e], dtype)
    at = torch.tensor([140, 111], device="cuda")
    rows = torch.arange(2, device="cuda")
    for i in range(10):
        yt = one.delta_rule_step(*(x[rows, at + i].clone() for x in a), state)
        for j in range(2):
            t_ = int(at[j]) + i
            _near("token", yt[j], ry[j, t_], b.y[j, t_], dtype)
    _near("state", state[:1], rs[:1], b.state[:1], "fp32")
    _near("whole", last, rs, b.state, "fp32")
    for p in (whole, piece, one):
        p.close()


def test_autograd_and_differences():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 80, 1, 12, 2, 1, 16)
    t, (s, _), (gy, _), (gs, _), _ = _inputs(shape, "fp32", 17)
    leaves = [x.requires_grad_(True) for x, _ in t] + [s.requires_grad_(True)]
    plan = _plan(P, shape)
    n = torch.tensor([80, 33], dtype=torch.int32, device="cuda")
    y, last = P.cgconv_delta_rule(*leaves[:5], plan, lengths=n, state=leaves[5], return_state=True)
    got = torch.autograd.grad((y, last), leaves, (gy.transpose(0, 1).contiguous().transpose(0, 1), gs))
    with torch.no_grad():
        want = plan.delta_rule_backward(*leaves[:5], gy, lengths=n, state=leaves[5], grad_state=gs)
    assert all(torch.equal(x, z) for x, z in zip(got, want))
    # the state's gradient alone, y's alone, and a leaf that needs none
    y, last = P.cgconv_delta_rule(*leaves[:5], plan, state=leaves[5], return_state=True)
    alone, = torch.autograd.grad(last, (leaves[1],), gs, retain_graph=True)
    with torch.no_grad():
        assert torch.equal(alone, plan.delta_rule_backward(*leaves[:5], torch.zeros_like(gy), state=leaves[5], grad_state=gs)[1])
        assert torch.equal(torch.autograd.grad(y, (leaves[2],), gy)[0],
                           plan.delta_rule_backward(*leaves[:5], gy, state=leaves[5])[2])
    # a central difference along a random direction of all inputs: its cubic term and the
    # rounding of the two losses (both about 1e-3 of it) stay below 1%
    gen = torch.Generator("cuda").manual_seed(1)
    d = [torch.randn(x.shape, generator=gen, device="cuda") * x.detach().abs().mean() for x in leaves]
    along = sum(float((x.double() * z.double()).sum()) for x, z in zip(got, d))
    e = 2e-3

    def loss(sign):
        with torch.no_grad():
            moved = [x + sign * e * z for x, z in zip(leaves, d)]
            yy, ll = plan.delta_rule(*moved[:5], lengths=n, state=moved[5])
            return float((yy.double() * gy).sum() + (ll.double() * gs).sum())
    assert abs((loss(1) - loss(-1)) / (2 * e) - along) <= 0.01 * abs(along) + 0.05
    with torch.no_grad():
        assert not P.cgconv_delta_rule(*leaves[:5], plan).requires_grad
    # v in 8 bits: the gradients of the values that the 8 bits hold
    y = P.cgconv_delta_rule(*leaves[:5], plan, checkpoint="int8")
    got = torch.autograd.grad(y, leaves[:5], gy)
    with torch.no_grad():
        held = P.checkpoint_unpack(*P.checkpoint_pack(leaves[2]))
        want = plan.delta_rule_backward(leaves[0], leaves[1], held, leaves[3], leaves[4], gy)
    assert all(torch.equal(x, z) for x, z in zip(got, want))
    with pytest.raises(ValueError, match="checkpoint"):
        P.cgconv_delta_rule(*leaves[:5], plan, checkpoint="int4")
    plan.close()


def test_shared_heads_and_the_same_leaf_twice():
    """A key that several heads share gets the sum of their gradients; the same tensor as
    key and query the sum of both."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (1, 75, 0, 24, 4, 2, 12)
    t, _, (gy, _), _, _ = _inputs(shape, "fp32", 19)
    q, k, v, g, b = (x for x, _ in t)
    plan, full = _plan(P, shape), _plan(P, shape[:5] + (4, 12))
    wide = [x.repeat_interleave(2, 2).contiguous() for x in (q, k)]
    y, s = plan.delta_rule(q, k, v, g, b)
    y4, s4 = full.delta_rule(*wide, v, g, b)
    assert torch.equal(y, y4) and torch.equal(s, s4)
    got, want = plan.delta_rule_backward(q, k, v, g, b, gy), full.delta_rule_backward(*wide, v, g, b, gy)
    for i in (0, 1):
        each = get(want[i]).reshape(1, 75, 2, 2, 12)
        # the sum of two rounded gradients against the rounded sum, and through the norm's derivative
        assert np.abs(get(got[i]) - each.sum(3)).max() <= 64 * U * np.abs(each).sum(3).max()
    assert all(torch.equal(x, z) for x, z in zip(got[2:5], want[2:5]))
    both = k.clone().requires_grad_(True)
    gboth, = torch.autograd.grad(P.cgconv_delta_rule(both, both, v, g, b, plan), both, gy)
    gq, gk = plan.delta_rule_backward(k, k, v, g, b, gy)[:2]
    assert torch.equal(gboth, gq + gk)
    plan.close()
    full.close()


def test_rotations():
    """Rotating the components of the values rotates the outputs."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (1, 100, 1, 16, 2, 2, 32)
    t, _, _, _, _ = _inputs(shape, "fp32", 23)
    (a, av) = map(list, zip(*t))
    R, _ = np.linalg.qr(np.random.default_rng(1).normal(size=(3, 3)))
    turn = torch.eye(4, device="cuda")
    turn[1:, 1:] = torch.tensor(R, device="cuda")
    plan = _plan(P, shape)
    y = torch.einsum("km,bnmc->bnkc", turn, plan.delta_rule(*a)[0])
    a[2] = torch.einsum("km,bnmc->bnkc", turn, a[2]).contiguous()
    assert rel_l2(get(plan.delta_rule(*a)[0]), get(y)) <= _bar(shape, _Bound(*av, 1.0, None).k, "fp32")
    plan.close()


def test_tensor_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 9, 1, 12, 4, 2, 8)
    t, (s, _), (gy, _), _, _ = _inputs(shape, "fp32", 29)
    a = [x for x, _ in t]
    plan = _plan(P, shape)
    for i, name in enumerate(("q", "k", "v", "decay", "beta")):
        for bad in (a[i].cpu(), a[i].half(), a[i][:1], a[i].transpose(0, 1).contiguous().transpose(0, 1)):
            with pytest.raises(ValueError, match=name):
                plan.delta_rule(*a[:i], bad, *a[i + 1:])
    with pytest.raises(ValueError, match="state"):
        plan.delta_rule(*a, state=s[:1])
    with pytest.raises(ValueError, match="lengths"):
        plan.delta_rule(*a, lengths=torch.tensor([9, 9], device="cuda"))
    with pytest.raises(P.CgconvError, match="overlap"):
        plan.delta_rule(*a, out=a[2])
    with pytest.raises(ValueError, match="grad_y"):
        plan.delta_rule_backward(*a, gy.to(torch.bfloat16))
    small = _plan(P, shape, backward=False)
    assert small.info() < plan.info()
    with pytest.raises(P.CgconvError, match="backward"):
        small.delta_rule_backward(*a, gy)
    none = P.SequencePlan(2, 9, 1, 12)
    with pytest.raises((P.CgconvError, ValueError)):
        none.delta_rule(*a)
    for p in (plan, small, none):
        p.close()
