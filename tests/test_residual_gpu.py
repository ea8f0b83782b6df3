"""GPU parity of the norms around a residual connection and their gradients against
the float64 oracle, in fp32 and bf16, in the three forms of the kernels.

Bounds.  An element passes at most 4 x 64 roundings in the sums of its token (two norms,
each forward and backward; 64 as in the norm's tests) and, in the parameters' gradients, 512
over the tokens: 768 half steps of the magnitudes at worst, independent ones as their root,
28.  The magnitudes are at most ten times the result's 2-norm here (deviations of order one,
parameters near one): 280 half steps of fp32, 1.7e-5, relative to the 2-norm, and the
rounding of the output's own type.
"""

import numpy as np
import pytest

from oracle import memory as M
from tests.conftest import rel_l2
from tests.seq_util import HALF, U, get, put, torch_gpu

pytestmark = pytest.mark.gpu

EPS = 1e-5
BAR = 280 * U

# (B, N, L, C): rows of 1 to 64 lanes, whole and partial vectors and tiles; wide rows of
# scalars, their forms by length; wide rows of vectors; one token, one channel
SHAPES = [(1, 1, 0, 1), (2, 3, 0, 5), (1, 300, 0, 8), (3, 7, 1, 12), (2, 64, 2, 4), (1, 33, 6, 32), (2, 5, 5, 20),
          (1, 9, 8, 3), (1, 4, 8, 64), (2, 3, 3, 130), (1, 70, 0, 64), (1, 5, 0, 257), (3, 2, 0, 1030), (1, 3, 2, 416),
          (1, 6, 0, 4096), (1, 7, 0, 4098), (1, 3, 0, 8200), (1, 2, 0, 16384), (1, 3, 0, 16383), (1, 2, 8, 960),
          (2, 2, 1, 1001), (2, 5, 1, 300), (1, 600, 3, 16)]
NAMES = ("x", "u", "gate", "post_weight", "scale", "weight", "bias")


def _inputs(shape, dtype, seed, grouped=True):
    B, N, L, C = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    f = lambda: r.normal(size=(B, N, K, C))  # noqa: E731
    t = [put(f() + 0.3 * r.normal(size=C), dtype), put(0.5 * f(), dtype), put(r.normal(size=(B, N, C)), dtype),
         put(1 + 0.2 * r.normal(size=(L + 1, C))), put(0.5 + 0.3 * r.random(C)), put(1 + 0.2 * r.normal(size=(L + 1, C))),
         put(0.2 * r.normal(size=C))]
    return t, put(f(), dtype), put(f(), dtype)


def _check(name, got, ref, dtype, C):
    # a row of few channels has a deviation far from one now and then: sums of its few values cancel
    bar = BAR * (10 if C < 8 else 1) + HALF[dtype]
    assert np.isfinite(get(got)).all(), name
    scale = np.linalg.norm(ref)
    off = np.linalg.norm(get(got) - ref)
    assert off <= bar * scale + 1e-6 * np.sqrt(ref.size) * (scale < 1e-3), (name, off / max(scale, 1e-30), bar)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%dN%dL%dC%d" % s)
def test_outputs_and_gradients(shape, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C = shape
    print(f"[gpu] residual {shape} {dtype}", flush=True)
    t, (gr, grv), (gy, gyv) = _inputs(shape, dtype, 200 + C + N)
    a, av = (list(x) for x in zip(*t))
    plan = P.SequencePlan(B, N, L, C)
    r, y, stats = plan.residual_norm(*a, eps=EPS)
    grads = plan.residual_norm_backward(*a[:6], stats, gr, gy)
    again = plan.residual_norm_backward(*a[:6], stats, gr, gy)
    no_r = plan.residual_norm_backward(*a[:6], stats, None, gy)
    only = [plan.residual_norm_backward(*a[:6], stats, gr, gy, need=tuple(i == j for j in range(7))) for i in range(7)]
    bare = plan.residual_norm(a[0], a[1], eps=EPS)
    gbare = plan.residual_norm_backward(a[0], a[1], None, None, None, None, bare[2], gr, gy,
                                        need=(True, True, False, True, True, True, True))
    torch.cuda.synchronize()
    plan.close()
    for n, x, z in zip("ry", (r, y), M.residual(*av, L, EPS)):
        _check(n, x, z, dtype, C)
    for n, x, z in zip("ry", bare, M.residual(av[0], av[1], *(None,) * 5, L, EPS)):
        _check("bare " + n, x, z, dtype, C)
    sets = ((grads, av, grv), (no_r, av, None), (gbare, av[:2] + [None] * 5, grv))
    for got, args, g in sets:
        for i, (n, x, z) in enumerate(zip(NAMES, got, M.residual_backward(*args, g, gyv, L, EPS))):
            if x is not None:
                _check(n, x, z, dtype if i < 3 else "fp32", C)
    assert all(torch.equal(x, z) for x, z in zip(grads, again))
    for i, one in enumerate(only):
        assert torch.equal(one[i], grads[i]) and all(x is None for j, x in enumerate(one) if j != i)


def test_many_tokens_fill_every_block():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    for L, C, N, dtype in ((0, 16, 100003, "bf16"), (2, 20, 20011, "fp32"), (0, 1032, 5003, "bf16"), (1, 520, 1201, "bf16")):
        t, (gr, grv), (gy, gyv) = _inputs((1, N, L, C), dtype, 5)
        a, av = (list(x) for x in zip(*t))
        plan = P.SequencePlan(1, N, L, C)
        stats = plan.residual_norm(*a, eps=EPS)[2]
        grads = plan.residual_norm_backward(*a[:6], stats, gr, gy)
        again = plan.residual_norm_backward(*a[:6], stats, gr, gy)
        plan.close()
        for i, (n, x, z) in enumerate(zip(NAMES, grads, M.residual_backward(*av, grv, gyv, L, EPS))):
            # sums of up to 1e5 tokens: their root is 300 half steps, of magnitudes up to 20 times the sum's norm
            bar = (6000 * U if i >= 3 else BAR) + HALF[dtype if i < 3 else "fp32"]
            assert rel_l2(get(x), z) <= bar, (L, C, n)
        assert all(torch.equal(x, z) for x, z in zip(grads, again))


def test_it_is_the_two_norms_and_the_sum():
    """Against the package's own norm, rounded between: fp32, a few roundings apart."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 40, 2, 24)
    t, _, _ = _inputs(shape, "fp32", 31)
    x, u, gate, po, sc, w, b = (v for v, _ in t)
    plan = P.SequencePlan(*shape)
    r, y, _ = plan.residual_norm(x, u, gate, po, sc, w, b, eps=EPS)
    want = x + plan.norm(u, po, eps=EPS)[0] * (sc * torch.nn.functional.silu(gate))[:, :, None]
    assert torch.allclose(r, want, rtol=0, atol=16 * U * float(want.abs().max()))
    assert torch.allclose(y, plan.norm(r, w, b, EPS)[0], rtol=0, atol=64 * U * float(y.abs().max()))
    plan.close()


def test_constant_rows_large_means_and_gates():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(1, 6, 1, 64)
    x, u = torch.zeros(1, 6, 4, 64, device="cuda"), torch.zeros(1, 6, 4, 64, device="cuda")
    gate = torch.zeros(1, 6, 64, device="cuda")
    u[0, 1] = 5.0
    u[0, 2, 0] = 1e4 + torch.arange(64, device="cuda") / 64
    u[0, 3:] = torch.randn(3, 4, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    gate[0, 3], gate[0, 4], gate[0, 5] = 200.0, -200.0, -1e4  # silu: the gate itself, zero, zero
    r, y, stats = plan.residual_norm(x, u, gate, eps=EPS)
    g = plan.residual_norm_backward(x, u, gate, None, None, None, stats, torch.ones_like(x), torch.ones_like(x),
                                    need=(True, True, True, True, True, True, True))
    assert all(torch.isfinite(v).all() for v in (r, y, stats) + g)
    assert (r[0, 4:] == 0).all() and (y[0, 4:] == 0).all() and (r[0, :2, 0] == 0).all()
    h = M.norm_parts(get(u), 1, EPS)[0]
    assert rel_l2(get(r[0, 3]), 200 * h[0, 3]) <= BAR
    plan.close()


def test_nan_stays_in_its_degree():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    for C, dtype in ((40, "fp32"), (600, "bf16")):
        shape = (2, 3, 1, C)
        t, _, _ = _inputs(shape, dtype, 37)
        a = [v for v, _ in t]
        plan = P.SequencePlan(*shape)
        r, y, _ = plan.residual_norm(*a, eps=EPS)
        bad = a[1].clone()
        bad[0, 1, 2, 7] = float("nan")
        bad[1, 0, 0, 3] = float("inf")
        r2, y2, _ = plan.residual_norm(a[0], bad, *a[2:], eps=EPS)
        hit = torch.zeros(shape[:2] + (4, C), dtype=torch.bool, device="cuda")
        hit[0, 1, 1:] = True
        hit[1, 0, 0] = True
        assert torch.equal(r[~hit], r2[~hit]) and torch.equal(y[~hit], y2[~hit])
        assert torch.isnan(r2[hit]).all() and torch.isnan(y2[hit]).all()
        plan.close()


def test_autograd_and_differences():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 9, 2, 24)
    t, (gr, _), (gy, _) = _inputs(shape, "fp32", 41)
    leaves = [v.requires_grad_(True) for v, _ in t]
    plan = P.SequencePlan(*shape)
    r, y = P.cgconv_residual_norm(*leaves, plan, eps=EPS)
    got = torch.autograd.grad((r, y), leaves, (gr.transpose(0, 1).contiguous().transpose(0, 1), gy), retain_graph=True)
    with torch.no_grad():
        stats = plan.residual_norm(*leaves, eps=EPS)[2]
        want = plan.residual_norm_backward(*leaves[:6], stats, gr, gy)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        # one output alone
        assert torch.equal(torch.autograd.grad(y, leaves[1], gy, retain_graph=True)[0],
                           plan.residual_norm_backward(*leaves[:6], stats, None, gy)[1])
        assert torch.equal(torch.autograd.grad(r, leaves[1], gr)[0],
                           plan.residual_norm_backward(*leaves[:6], stats, gr, torch.zeros_like(gy))[1])
    # a central difference along a random direction of all inputs: its cubic term and the
    # rounding of the losses stay below 1%
    gen = torch.Generator("cuda").manual_seed(3)
    d = [torch.randn(v.shape, generator=gen, device="cuda") * v.detach().abs().mean() for v in leaves]
    along = sum(float((a.double() * b.double()).sum()) for a, b in zip(got, d))

    def loss(step):
        with torch.no_grad():
            rr, yy, _ = plan.residual_norm(*(v + step * z for v, z in zip(leaves, d)), eps=EPS)
            return float((rr.double() * gr).sum() + (yy.double() * gy).sum())
    assert abs((loss(2e-3) - loss(-2e-3)) / 4e-3 - along) <= 0.01 * abs(along) + 0.05
    # x and u in 8 bits: the gradients at the values that the 8 bits hold
    r, y = P.cgconv_residual_norm(*leaves, plan, eps=EPS, checkpoint="int8")
    got = torch.autograd.grad((r, y), leaves, (gr, gy))
    with torch.no_grad():
        held = [P.checkpoint_unpack(*P.checkpoint_pack(v)) for v in leaves[:2]]
        want = plan.residual_norm_backward(*held, *leaves[2:6], stats, gr, gy)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert not P.cgconv_residual_norm(*leaves, plan)[0].requires_grad
    # the same tensor as stream and block
    x = leaves[0]
    both, = torch.autograd.grad(P.cgconv_residual_norm(x, x, None, None, None, None, None, plan)[1], x, gy)
    with torch.no_grad():
        st = plan.residual_norm(x, x)[2]
        gx, gu = plan.residual_norm_backward(x, x, None, None, None, None, st, None, gy,
                                             need=(True, True) + (False,) * 5)[:2]
    assert torch.equal(both, gx + gu)
    plan.close()


def test_tensor_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 4, 1, 16)
    t, (gr, _), (gy, _) = _inputs(shape, "fp32", 43)
    a = [v for v, _ in t]
    plan = P.SequencePlan(*shape)
    for i, name in enumerate(NAMES):
        for bad in (a[i].cpu(), a[i].half(), a[i][..., :8]):
            with pytest.raises(ValueError, match="dtype|float32 or bfloat16|" + name):
                plan.residual_norm(*a[:i], bad, *a[i + 1:])
    with pytest.raises(P.CgconvError, match="overlap"):
        plan.residual_norm(*a, out_r=a[0])
    with pytest.raises(P.CgconvError, match="overlap"):
        plan.residual_norm(*a, out_r=a[0].clone(), out_y=a[1])
    with pytest.raises(P.CgconvError, match="eps"):
        plan.residual_norm(*a, eps=float("nan"))
    stats = plan.residual_norm(*a)[2]
    with pytest.raises(ValueError, match="stats"):
        plan.residual_norm_backward(*a[:6], stats[:1], gr, gy)
    with pytest.raises(P.CgconvError, match="gate"):
        plan.residual_norm_backward(a[0], a[1], None, *a[3:6], stats, gr, gy)
    plan.close()
