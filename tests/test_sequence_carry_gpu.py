"""The scan where its states, their gradients and the chunks' sums pass 2^31
elements (2^20 + 3 tokens of 2048 columns, 16 states, chunks of 16 tokens in the
backward), with decays slow enough for what the carry hands from chunk to chunk to
count: the last tokens against the float64 oracle on a copy of the last 128.  Of
what lies before the copy nothing is left 104 tokens later, exp(-104), while the
states that the last tokens' own chunks start with decide their values.  The sums
over all tokens, in float64 torch: gradients of D, and of the norm's and the
convolution's weights.
"""

import numpy as np
import pytest

import tests.test_scan_gpu as scan_tests
from oracle import sequence as S
from tests.seq_util import HALF, U, get, torch_gpu

pytestmark = pytest.mark.gpu

N, COLUMNS, STATES = (1 << 20) + 3, 2048, 16
COPY, LAST = 128, 24
CHUNKS = (N + 15) // 16
assert CHUNKS * STATES * COLUMNS > 2 ** 31 and N * COLUMNS > 2 ** 31


@pytest.fixture(scope="module")
def arrays():
    torch = torch_gpu()
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.empty(1, N, 1, COLUMNS, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    g = torch.empty_like(x).normal_(generator=gen)
    yield torch, x, g, gen
    del x, g
    torch.cuda.empty_cache()


def _last(a):
    return a[:, -LAST:]


def _slices(torch, x, g):
    """x and g in float64, 2^14 tokens at a time."""
    for t in range(0, N, 1 << 14):
        yield t, x[0, t:t + (1 << 14)].double(), g[0, t:t + (1 << 14)].double()


def _check(name, got, ref, magnitude, roundings):
    bound = (roundings * U + HALF["fp32"]) * magnitude
    worst = float(((got.double() - ref).abs() / bound).max())
    assert worst <= 1, f"{name}: {worst:.3g} of the bound"


@pytest.mark.parametrize("L", [0, 1])
def test_scan(arrays, L):
    torch, x, g, gen = arrays
    import paper_2509_24093_amd as P
    K, C = (L + 1) ** 2, COLUMNS // (L + 1) ** 2
    x, g = x.view(1, N, K, C), g.view(1, N, K, C)
    new = lambda *s: torch.empty(*s, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)  # noqa: E731
    # steps of at least softplus(1.5) = 1.70, times A below -1/1.7: decays of at most exp(-1)
    delta = (2 + 0.5 * torch.rand(1, N, C, device="cuda", generator=gen)).to(torch.bfloat16)
    bias = torch.rand(C, device="cuda", generator=gen) * 0.5 - 0.5
    A = -(1 + torch.rand(C, STATES, device="cuda", generator=gen)) / 1.7
    Bt, Ct, D = new(1, N, STATES), new(1, N, STATES), torch.randn(C, device="cuda", generator=gen)
    plan = P.SequencePlan(1, N, L, C, states=STATES)
    order = (x, delta, A, Bt, Ct, D, bias)
    cut = [get(t if t.ndim < 3 else t[:, -COPY:]) for t in order]
    gc = get(g[:, -COPY:])
    b = scan_tests._Bounds(*cut)
    ry, rh = S.scan(*cut)
    y, state = plan.scan(x, delta, A, Bt, Ct, D, bias)
    scan_tests.close("y", _last(y), _last(ry), _last(b.ye), "bf16")
    scan_tests.close("state", state, rh, b.he[-1])
    del y
    got = plan.scan_backward(x, delta, A, Bt, Ct, D, g, bias, need=(True, True, False, True, True, True, False))
    ref, bounds = S.scan_backward(*cut[:-1], gc, cut[-1]), b.backward(gc)
    for i, name in ((0, "x"), (1, "delta"), (3, "Bt"), (4, "Ct")):
        scan_tests.close("grad " + name, _last(got[i]), _last(ref[i]), _last(bounds[name]), "bf16")
    plan.close()
    # 16 tokens in a thread, the components (or none), 1025 chunks in a slice, 6 steps
    # between the slices
    want, size = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2))
    for _, xs, gs in _slices(torch, x, g):
        want += (xs * gs).sum((0, 1))
        size += (xs * gs).abs().sum((0, 1))
    _check("grad D", got[5], want, size, 16 + K * 1025 + 6)


def test_norm_and_convolution_weights(arrays):
    """Roundings.  Norm: 512 tokens in a thread, 2048 blocks in 16 slices, 16 more,
    and 64 half steps each for h's mean and deviation; convolution: 64 tokens in a
    thread, 4 chunks in a block, 4097 blocks in 64 slices, 6 steps: 139."""
    torch, x, g, gen = arrays
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(1, N, 0, COLUMNS)
    w = 1 + 0.1 * torch.randn(1, COLUMNS, device="cuda", generator=gen)
    y, mean, rstd = plan.norm(x, w)
    del y
    _, gw, gb = plan.norm_backward(x, w, mean, rstd, g, need_x=False)
    want, size, sum_g, abs_g = (torch.zeros(COLUMNS, dtype=torch.float64, device="cuda") for _ in range(4))
    for t, xs, gs in _slices(torch, x, g):
        xs, gs = xs[:, 0], gs[:, 0]
        d = xs - xs.mean(-1, keepdim=True)
        r = ((d * d).mean(-1, keepdim=True) + 1e-5).rsqrt()
        want += (gs * d * r).sum(0)
        # h carries the mean's error (of sums of |x|) and the deviation's (relative)
        size += (gs.abs() * (2 * d.abs() + xs.abs() + xs.abs().mean(-1, keepdim=True)) * r).sum(0)
        sum_g += gs.sum(0)
        abs_g += gs.abs().sum(0)
    _check("norm gw", gw[0], want, size, 512 + 128 + 16 + 128)
    _check("norm gb", gb, sum_g, abs_g, 512 + 128 + 16)
    W = 3
    cw = torch.randn(W, 1, COLUMNS, device="cuda", generator=gen)
    _, gw, gb = plan.conv_backward(x, cw, None, g, activation=False, need_x=False)
    want, size = (torch.zeros(W, COLUMNS, dtype=torch.float64, device="cuda") for _ in range(2))
    for t, xs, gs in _slices(torch, x, g):
        xs, gs = xs[:, 0], gs[:, 0]
        if t:
            xs = torch.cat([x[0, t - W + 1:t, 0].double(), xs])
        else:
            xs = torch.cat([torch.zeros(W - 1, COLUMNS, dtype=torch.float64, device="cuda"), xs])
        for j in range(W):
            p = gs * xs[W - 1 - j:W - 1 - j + len(gs)]
            want[j] += p.sum(0)
            size[j] += p.abs().sum(0)
    _check("conv gw", gw[:, 0], want, size, 139)
    _check("conv gb", gb, sum_g, abs_g, 139)
    plan.close()
    assert np.isfinite(get(gw)).all()
