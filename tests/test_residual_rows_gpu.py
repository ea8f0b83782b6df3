"""Rows that the norms around a residual connection find hard: constant ones and ones whose mean
is far above their deviation, in the block's output and in the stream, with gates that let them
through; and the gate's sigmoid over its whole range.

Bounds of the rows.  A mean is a sum of up to 40 roundings in a row (values of a thread, lanes,
waves), so it is off by up to 40 u |mean|, u = 2^-24, and the deviations, of size s, by a share
e = 40 u |mean| / s.  The variance then is off by a share e^2; outputs have the deviation once,
gradients up to three times, so to the roundings of the other tests (280 u of the 2-norm, in
tests/test_residual_gpu.py) come e and 3 e; a norm behind another has both rows' shares.
Squares added without their mean would be off by a share u (|mean| / s)^2, 10 to 100 times e.
"""

import numpy as np
import pytest

from oracle import memory as M
from tests.seq_util import U, get, put, torch_gpu

pytestmark = pytest.mark.gpu

EPS = 1e-5
BAR = 280 * U
# rows of 16 lanes, long rows of scalars, long rows of vectors
FORMS = {"rows": (1, 64), "wide": (0, 1000), "channels": (1, 320)}


def _run(form, u, x, gate, seed):
    """Outputs, stats and gradients, the oracle's, and the parameters' names."""
    torch_gpu()
    import paper_2509_24093_amd as P
    L, C = FORMS[form]
    r = np.random.default_rng(seed)
    B, N, K, _ = u.shape
    par = [put(1 + 0.2 * r.normal(size=(L + 1, C))), put(0.5 + 0.3 * r.random(C)), put(1 + 0.2 * r.normal(size=(L + 1, C))),
           put(0.2 * r.normal(size=C))]
    (x, xv), (u, uv) = put(x), put(u)
    gate, gv = put(gate) if gate is not None else (None, None)
    (gr, grv), (gy, gyv) = put(r.normal(size=u.shape)), put(r.normal(size=u.shape))
    plan = P.SequencePlan(B, N, L, C)
    a = [x, u, gate] + [p for p, _ in par]
    out = plan.residual_norm(*a, eps=EPS)
    grads = plan.residual_norm_backward(*a[:6], out[2], gr, gy, need=(True, True, gate is not None) + (True,) * 4)
    plan.close()
    av = [xv, uv, gv] + [p for _, p in par]
    return [get(o) for o in out], [None if g is None else get(g) for g in grads], M.residual(*av, L, EPS), \
        M.residual_backward(*av, grv, gyv, L, EPS), av


def _spread(C):
    return np.arange(C) % 64 / 64  # exact beside a mean of up to 2^17


@pytest.mark.parametrize("gated", [False, True], ids=["", "gate"])
@pytest.mark.parametrize("where", ["u", "x", "both"])
@pytest.mark.parametrize("mean", [100.0, 1000.0])
@pytest.mark.parametrize("form", FORMS)
def test_large_means(form, mean, where, gated):
    L, C = FORMS[form]
    r = np.random.default_rng(7)
    K, N = (L + 1) ** 2, 3
    u, x = 0.3 * r.normal(size=(1, N, K, C)), 0.3 * r.normal(size=(1, N, K, C))
    if where != "x":
        u[:, :, 0] = mean + _spread(C)
    if where != "u":
        x[:, :, 0] = -mean - _spread(C)[::-1]
    gate = 1 + 0.1 * r.normal(size=(1, N, C)) if gated else None
    (ro, y, stats), grads, (rr, ry), refs, av = _run(form, u, x, gate, 8)
    xv, uv = av[:2]
    su, sr = uv[:, :, 0].std(-1), rr[:, :, 0].std(-1)
    mu, mr = uv[:, :, 0].mean(-1), rr[:, :, 0].mean(-1)
    eu, er = 40 * U * np.abs(mu) / su, 40 * U * np.abs(mr) / sr
    assert eu.max() + er.max() < 0.05 and max(eu.max(), er.max()) > 40 * U * 100  # means of 100 deviations and more
    # the statistics: mean and factor of u, then of r, whose deviations carry u's share too
    for at, m, s, e in ((0, mu, su, eu), (L + 2, mr, sr, er)):
        assert (np.abs(stats[..., at] - m) <= 40 * U * np.abs(m) + (0 if at == 0 else (eu + BAR) * sr)).all()
        f = 1 / np.sqrt(s ** 2 + EPS)
        assert (np.abs(stats[..., at + 1] - f) <= (BAR + e ** 2 + (0 if at == 0 else eu)) * f).all()
    e = float((eu + er).max())

    def near(name, got, ref, share):
        off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert off <= BAR + share, (name, off, BAR + share)

    near("r", ro - xv, rr - xv, e + U * mean * np.sqrt(ro.size) / np.linalg.norm(rr - xv))  # r is rounded beside x
    near("y", y, ry, e)
    for n, g, ref in zip(("x", "u", "gate", "post", "scale", "weight", "bias"), grads, refs):
        if g is not None:
            near("g" + n, g, ref, 3 * e)


@pytest.mark.parametrize("form", FORMS)
def test_constant_rows(form):
    """A constant row of invariants has no deviation: it adds nothing, exactly; in the stream its
    output is the bias alone.  Gates of one let everything through."""
    L, C = FORMS[form]
    K = (L + 1) ** 2
    u, x = np.full((1, 4, K, C), 5.0), np.zeros((1, 4, K, C))
    u[:, 1] = -0.125
    u[:, 2:, 0] = 0.0
    x[:, 1] = 3.0
    x[:, 3, 0] = -1024.0
    (ro, y, stats), grads, (rr, ry), refs, av = _run(form, u, x, np.ones((1, 4, C)), 9)
    assert (ro[:, :, 0] == av[0][:, :, 0]).all() and (y[:, :, 0] == av[6]).all()
    for at, m in ((0, u[:, :, 0, 0]), (L + 2, x[:, :, 0, 0])):
        assert (stats[..., at] == m).all()
        assert (np.abs(stats[..., at + 1] - EPS ** -0.5) <= 4 * U * EPS ** -0.5).all()
    for n, got, ref in (("r", ro, rr), ("y", y, ry)) + tuple(zip(("gx", "gu", "ggate", "gpost", "gscale", "gweight", "gbias"),
                                                                grads, refs)):
        # the gradients of rows without a deviation are 316 times the others: eps alone is under their root
        assert np.isfinite(got).all() and np.linalg.norm(got - ref) <= BAR * np.linalg.norm(ref), n


def _ones(plan_tokens, torch):
    """u of norm +-1 exactly: (1, -1) has mean 0 and deviation 1."""
    u = torch.ones(1, plan_tokens, 1, 2, device="cuda")
    u[..., 1] = -1
    return u


def test_sigmoid_over_its_range():
    """r = +-silu(gate) and the gate's gradient +-silu'(gate) of one, where nothing but the gate's
    own arithmetic rounds.  With z log2(e) in two parts the power of 2 is off by the instruction's
    2 u and three roundings, 1 + e^-z by one more, the reciprocal with one Newton step by 2: 8 u of
    the sigmoid.  silu has one product more; its slope s (1 + z (1 - s)) the difference, the sum
    and two products, of terms up to s (1 + |z|).  Below -87 the sigmoid is under the smallest normal
    number, 2^-126, where the reciprocal may give zero, and never above it.

    eps = 1e-30: it is lost beside the deviation of one, which stays exact, and keeps the second
    norm finite, whose squares (silu^2, down to 1e-74 here) are below the smallest fp32 number;
    with eps = 0 its factor is 1 / 0, and 0 times it NaN."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    r = np.random.default_rng(3)
    z = np.concatenate([r.uniform(-87, 87, 120000), r.normal(size=60000), np.linspace(-20, 20, 60001),
                        np.exp(r.uniform(-80, 0, 20000)), -np.exp(r.uniform(-80, 0, 20000)), [0.0, -0.0],
                        np.exp(r.uniform(np.log(87), np.log(3e38), 5000)), -np.exp(r.uniform(np.log(87), np.log(3e38), 5000))])
    n = z.size
    gate, zv = put(np.repeat(z[None, :, None], 2, 2))
    zv = zv[0, :, 0]
    u = _ones(n, torch)
    x = torch.zeros_like(u)
    plan = P.SequencePlan(1, n, 0, 2)
    out, _, stats = plan.residual_norm(x, u, gate, eps=1e-30)
    grad = plan.residual_norm_backward(x, u, gate, None, None, None, stats, torch.ones_like(u), torch.zeros_like(u),
                                       need=(False, False, True) + (False,) * 4)[2]
    plan.close()
    assert (stats[..., 0] == 0).all() and (stats[..., 1] == 1).all()
    with np.errstate(over="ignore", under="ignore"):
        s = np.where(zv >= 0, 1 / (1 + np.exp(-np.abs(zv))), np.exp(-np.abs(zv)) / (1 + np.exp(-np.abs(zv))))
        other = np.where(zv >= 0, np.exp(-np.abs(zv)) / (1 + np.exp(-np.abs(zv))), 1 / (1 + np.exp(-np.abs(zv))))
    silu, slope = zv * s, s * (1 + zv * other)
    low = np.where(s < 2.0 ** -125, 2.0 ** -125, 0.0) * (1 + np.abs(zv))
    usual = zv > -87
    for sign, c in ((1, 0), (-1, 1)):
        got, got1 = sign * get(out)[0, :, 0, c], sign * get(grad)[0, :, c]
        assert np.isfinite(got).all() and np.isfinite(got1).all()
        assert (np.abs(got - silu) <= (8 + 1) * U * np.abs(silu) + low + 2.0 ** -149).all()
        assert (np.abs(got1 - slope) <= (2 * 8 + 4) * U * s * (1 + np.abs(zv)) + low).all()
    # two units of the last place, and silu's own rounding
    assert (np.abs(get(out)[0, usual, 0, 0] - silu[usual]) <= 5 * U * np.abs(silu[usual]) + 2.0 ** -149).all()
