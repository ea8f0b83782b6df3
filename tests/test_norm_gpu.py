"""GPU parity of layer norm by degree and its gradients against the float64
oracle, in fp32 and bf16, from rows of one channel to the widest, in both forms
of the kernels, with the input whole or as its 8-bit checkpoint.

Bounds per element.  A sum of n values by lanes and rows passes each value
through at most ROUND = 64 roundings (V R <= 32 in a thread, 6 lane steps, 17
rows or 16 waves, a division), so mean, variance and rstd are within ROUND half
steps of sums of magnitudes; y and the gradients combine a few of them.  gw and
gb add tokens in a thread (at most 2 tiles of the sizes here, 8 rows), over a
block's rows and over blocks: TOKENS = 512 roundings cover every size below.
"""

import numpy as np
import pytest

from oracle import sequence as S
from tests.seq_util import check, put, torch_gpu

pytestmark = pytest.mark.gpu

ROUND, TOKENS = 64, 512
EPS = 1e-5

# (B, N, L, C): the row form from 1 to 64 lanes a row (C a multiple of 1, 2, 4,
# 8; C = 1; whole and partial last tiles), the wide form (more than 64 vectors a
# row) for odd and even C, the longest segment, one token
SHAPES = [(1, 1, 0, 1), (2, 3, 0, 5), (1, 300, 0, 8), (3, 7, 1, 12), (2, 64, 2, 4), (1, 33, 6, 32), (2, 5, 5, 20),
          (1, 9, 8, 3), (1, 4, 8, 64), (2, 3, 3, 130), (1, 70, 0, 64), (1, 5, 0, 257), (3, 2, 0, 1030), (1, 3, 2, 416),
          (1, 6, 0, 4096), (1, 2, 0, 16384), (1, 3, 0, 16383), (1, 2, 8, 960), (2, 2, 1, 1001)]


def _inputs(shape, dtype, seed):
    B, N, L, C = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    x = r.normal(size=(B, N, K, C)) * np.exp(r.normal(size=(B, N, 1, 1))) + r.normal(size=C)
    return put(x, dtype), put(1 + 0.2 * r.normal(size=(L + 1, C))), put(r.normal(size=C)), put(r.normal(size=x.shape), dtype)


def _magnitudes(x, w, L, eps):
    """Bounds of |h| and of what rounding in the statistics can move it by."""
    h, mean, rstd = S.norm_parts(x, L, eps)
    r = rstd[:, :, S.degrees(L), None]
    m = np.abs(h) + np.abs(x) * r
    m[:, :, 0] += np.abs(x[:, :, 0]).mean(-1, keepdims=True) * r[:, :, 0]
    # rstd carries the mean's error too: relative, times h
    m += np.abs(h) * (np.abs(x[:, :, :1]).mean((2, 3), keepdims=True) * r[:, :, :1])
    return h, r, m


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%dN%dL%dC%d" % s)
def test_norm_and_gradients(shape, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C = shape
    print(f"[gpu] norm {shape} {dtype}", flush=True)
    (x, xv), (w, wv), (b, bv), (g, gv) = _inputs(shape, dtype, 100 + C + N)
    plan = P.SequencePlan(B, N, L, C)
    y, mean, rstd, codes, scales = plan.norm(x, w, b, EPS, checkpoint=True)
    gx, gw, gb = plan.norm_backward(x, w, mean, rstd, g)
    qx, qw, qb = plan.norm_backward((codes, scales), w, mean, rstd, g)
    only_x = plan.norm_backward(x, w, mean, rstd, g, need_weight=False, need_bias=False)
    only_b = plan.norm_backward(x, w, mean, rstd, g, need_x=False, need_weight=False)
    y1, mean1, rstd1 = plan.norm(x, None, None, EPS)
    px, pw, pb = plan.norm_backward(x, None, mean1, rstd1, g)
    torch.cuda.synchronize()
    plan.close()
    deg = S.degrees(L)
    h, r, mag = _magnitudes(xv, wv, L, EPS)
    check("y", y, S.norm(xv, wv, bv, L, EPS), mag * np.abs(wv)[deg] + np.abs(bv), 2 * ROUND, dtype)
    check("y plain", y1, h, mag, 2 * ROUND, dtype)
    # the checkpoint is exact
    ref_codes, ref_scales = S.pack(xv)
    assert (codes.cpu().numpy() == ref_codes).all() and (scales.cpu().numpy() == ref_scales).all()
    held = S.unpack(ref_codes, ref_scales)
    for tag, res, weight, hv in (("whole", (gx, gw, gb), wv, None), ("codes", (qx, qw, qb), wv, held),
                                 ("plain", (px, pw, pb), np.ones_like(wv), None)):
        rx, rw, rb = S.norm_backward(xv, weight, gv, L, EPS, held=hv)
        hm = mag if hv is None else mag + np.abs(hv) * r + np.abs(xv[:, :, :1]).mean(-1, keepdims=True) * r * (deg == 0)[:, None]
        hq = np.abs(h) if hv is None else hm
        gm = np.abs(gv) * np.abs(weight)[deg]
        m = gm.copy()
        for l in range(L + 1):
            s = slice(l * l, (l + 1) ** 2)
            dot, err = (gm[:, :, s] * hq[:, :, s]).mean((2, 3), keepdims=True), (gm[:, :, s] * hm[:, :, s]).mean((2, 3), keepdims=True)
            m[:, :, s] += hm[:, :, s] * dot + hq[:, :, s] * err + dot * hq[:, :, s]
        m[:, :, 0] += gm[:, :, 0].mean(-1, keepdims=True)
        relr = 1 + np.abs(xv[:, :, :1]).mean((2, 3), keepdims=True) * r[:, :, :1]
        check(tag + " gx", res[0], rx, m * r * relr, 4 * ROUND, dtype)
        gwm = np.stack([(np.abs(gv) * (hm + np.abs(h)))[:, :, l * l:(l + 1) ** 2].sum((0, 1, 2)) for l in range(L + 1)])
        check(tag + " gw", res[1], rw, gwm, TOKENS + 2 * ROUND)
        check(tag + " gb", res[2], rb, np.abs(gv[:, :, 0]).sum((0, 1)), TOKENS)
    assert torch.equal(only_x[0], gx) and only_x[1] is None and only_x[2] is None
    assert only_b[0] is None and torch.equal(only_b[2], gb)


def test_many_tokens_fill_every_block():
    # more tiles than blocks of the backward: the sums go round a second time
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    for L, C, N, dtype in ((0, 16, 200003, "bf16"), (2, 300, 1501, "fp32")):
        r = np.random.default_rng(7)
        (x, xv), (w, wv) = put(r.normal(size=(1, N, (L + 1) ** 2, C)), dtype), put(1 + 0.1 * r.normal(size=(L + 1, C)))
        g, gv = put(r.normal(size=xv.shape), dtype)
        plan = P.SequencePlan(1, N, L, C)
        y, mean, rstd = plan.norm(x, w, None, EPS)
        gx, gw, gb = plan.norm_backward(x, w, mean, rstd, g)
        again = plan.norm_backward(x, w, mean, rstd, g)
        plan.close()
        rx, rw, rb = S.norm_backward(xv, wv, gv, L, EPS)
        h = S.norm_parts(xv, L, EPS)[0]
        # a thread's share of the tokens, its block's rows and the blocks: below 4096 roundings
        check("gw", gw, rw, np.stack([np.abs(gv * h)[:, :, l * l:(l + 1) ** 2].sum((0, 1, 2)) for l in range(L + 1)]), 4096)
        check("gb", gb, rb, np.abs(gv[:, :, 0]).sum((0, 1)), 4096)
        assert all(torch.equal(a, b) for a, b in zip((gx, gw, gb), again))  # the order of the sums is fixed


def test_constant_rows_and_large_means():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(1, 4, 1, 64)
    x = torch.zeros(1, 4, 4, 64, device="cuda")
    x[0, 1] = 5.0
    x[0, 2, 0] = 1e4 + torch.arange(64, device="cuda") / 64
    y, mean, rstd = plan.norm(x, None, None, EPS)
    gx, _, _ = plan.norm_backward(x, None, mean, rstd, torch.ones_like(x))
    assert torch.isfinite(y).all() and torch.isfinite(gx).all()
    assert (y[0, 0] == 0).all() and (y[0, 1, 0] == 0).all()
    # the variance comes from centred values: a mean 3e4 times the deviation costs
    # at most |mean| rstd half steps of fp32 in y, a few per value
    h = S.norm_parts(x.cpu().numpy(), 1, EPS)
    assert np.abs(y[0, 2, 0].cpu().numpy() - h[0][0, 2, 0]).max() <= 66 * 2.0 ** -24 * 1e4 * h[2][0, 2, 0]
    plan.close()


def test_nan_and_infinity_stay_in_their_token():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(2, 3, 1, 40)
    x = torch.randn(2, 3, 4, 40, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    clean = plan.norm(x)[0]
    bad = x.clone()
    bad[0, 1, 2, 7] = float("nan")
    bad[1, 0, 0, 3] = float("inf")
    y, _, _, codes, scales = plan.norm(bad, checkpoint=True)
    # degree 1 of one token, degree 0 of another
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[0, 1, 1:] = True
    hit[1, 0, 0] = True
    assert torch.equal(y[~hit], clean[~hit]) and torch.isnan(y[hit]).all()
    back = P.checkpoint_unpack(codes, scales)
    assert torch.isnan(back[0, 1, 2, :32]).all() and torch.isfinite(back[0, 1, 2, 32:]).all()
    assert int(torch.isnan(back).sum()) == 64
    plan.close()


@pytest.mark.parametrize("checkpoint", [None, "int8"])
def test_autograd(checkpoint):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(2, 9, 2, 24)
    (x, _), (w, _), (b, _), (g, _) = _inputs((2, 9, 2, 24), "fp32", 5)
    leaves = [t.requires_grad_(True) for t in (x, w, b)]
    y = P.cgconv_norm(x, w, b, plan, eps=EPS, checkpoint=checkpoint)
    got = torch.autograd.grad(y, leaves, g.transpose(0, 1).contiguous().transpose(0, 1))  # a strided gradient
    with torch.no_grad():
        y0, mean, rstd, codes, scales = plan.norm(x, w, b, EPS, checkpoint=True)
        ref = plan.norm_backward((codes, scales) if checkpoint else x, w, mean, rstd, g)
    assert torch.equal(y, y0) and all(torch.equal(a, c) for a, c in zip(got, ref))
    # only the weight, and inference
    y = P.cgconv_norm(x.detach(), w, None, plan, checkpoint=checkpoint)
    gw, = torch.autograd.grad(y, (w,), g)
    assert gw.shape == w.shape
    with torch.no_grad():
        assert not P.cgconv_norm(x, w, b, plan, checkpoint=checkpoint).requires_grad
    with pytest.raises(ValueError, match="checkpoint"):
        P.cgconv_norm(x, w, b, plan, checkpoint="int4")
    plan.close()


def test_tensor_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(2, 4, 1, 16)
    x = torch.zeros(2, 4, 4, 16, device="cuda")
    w = torch.ones(2, 16, device="cuda")
    for bad in (x.cpu(), x.half(), x.transpose(0, 1).contiguous().transpose(0, 1), x[:1], x[..., :8]):
        with pytest.raises(ValueError):
            plan.norm(bad, w)
    for bad in (w[:1], w.to(torch.bfloat16), w.T.contiguous().T):
        with pytest.raises(ValueError, match="weight"):
            plan.norm(x, bad)
    y, mean, rstd = plan.norm(x, w)
    with pytest.raises(ValueError, match="x must"):
        plan.norm_backward(x.to(torch.bfloat16), w, mean, rstd, x)
    with pytest.raises(ValueError, match="mean"):
        plan.norm_backward(x, w, mean[:1], rstd, x)
    with pytest.raises(P.CgconvError, match="overlap"):
        plan.norm(x, w, out=x)
    with pytest.raises(P.CgconvError, match="eps"):
        plan.norm(x, w, eps=-1.0)
    plan.close()
