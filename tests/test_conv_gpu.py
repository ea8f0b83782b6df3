"""GPU parity of the short causal convolution (whole sequences, single tokens,
gradients) against the float64 oracle.

Bounds: z is at most W + 1 products and sums, so within 2 W half steps of M =
sum |w||x| + |b|; z sigmoid(z) and its derivative have slopes below 1.1 and add
up to 8 + 3 |z| half steps of the value (the exponential's argument is rounded
once): 32 half steps of M (1 + M) cover both.  gx adds W such products more (64);
gw and gb add up to 64 tokens in a thread, 64 chunks in a block and the blocks in
16 slices: 512 for the sizes here.
"""

import numpy as np
import pytest

from oracle import sequence as S
from tests.seq_util import check, get, put, torch_gpu

pytestmark = pytest.mark.gpu

# (B, N, L, C, W): one token, shorter than the filter, odd columns, several
# chunks with a partial last one, more than 64 column vectors, every vector width
SHAPES = [(1, 1, 0, 1, 2), (2, 2, 0, 4, 8), (1, 9, 1, 3, 4), (3, 70, 2, 20, 4), (2, 65, 0, 300, 3), (1, 130, 6, 32, 4),
          (2, 33, 3, 7, 5), (1, 200, 0, 1030, 6), (4, 19, 1, 6, 8), (1, 1000, 0, 2, 7)]


def _inputs(shape, dtype, seed, ragged):
    B, N, L, C, W = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    x, w, b = put(r.normal(size=(B, N, K, C)), dtype), put(r.normal(size=(W, L + 1, C))), put(r.normal(size=C))
    g = put(r.normal(size=(B, N, K, C)), dtype)
    state = put(r.normal(size=(B, W - 1, K, C)), dtype)
    lengths = r.integers(0, N + 1, size=B) if ragged else None
    if ragged:
        lengths[0] = N
        if B > 2:
            lengths[1] = 0
    return x, w, b, g, state, lengths


def _dev(torch, lengths):
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")


def _magnitude(x, w, b, L, lengths, state):
    return S.conv(np.abs(x), np.abs(w), np.abs(b), L, lengths, None if state is None else np.abs(state), False)[0]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("activation", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%dN%dL%dC%dW%d" % s)
def test_forward_and_gradients(shape, activation, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, W = shape
    print(f"[gpu] conv {shape} {activation} {dtype}", flush=True)
    plan = P.SequencePlan(B, N, L, C)
    for ragged in (False, True):
        (x, xv), (w, wv), (b, bv), (g, gv), (st, sv), lengths = _inputs(shape, dtype, 50 + N + W, ragged)
        n = _dev(torch, lengths)
        for state, value in ((None, None), (st, sv)):
            y, last = plan.conv(x, w, b, n, state, activation)
            ref, end = S.conv(xv, wv, bv, L, lengths, value, activation)
            m = _magnitude(xv, wv, bv, L, lengths, value)
            check("y", y, ref, m * (1 + m), 32, dtype)
            assert last.dtype == x.dtype and (get(last) == end).all()
        gx, gw, gb = plan.conv_backward(x, w, b, g, n, activation)
        rx, rw, rb = S.conv_backward(xv, wv, bv, gv, L, lengths, activation)
        m = _magnitude(xv, wv, bv, L, lengths, None)
        gm = np.abs(gv) * (1 + m)
        ax, aw, ab = S.conv_backward(np.abs(xv), np.abs(wv), np.zeros(C), gm, L, lengths, False)
        check("gx", gx, rx, 1.1 * ax, 64, dtype)
        check("gw", gw, rw, 1.1 * aw, 512)
        check("gb", gb, rb, 1.1 * ab, 512)
        only = plan.conv_backward(x, w, b, g, n, activation, need_weight=False, need_bias=False)
        assert torch.equal(only[0], gx) and only[1] is None
        only = plan.conv_backward(x, w, b, g, n, activation, need_x=False, need_bias=False)
        assert torch.equal(only[1], gw) and only[0] is None
    nobias = plan.conv(x, w, None, n, None, activation)[0]
    zero = plan.conv(x, w, torch.zeros_like(b), n, None, activation)[0]
    assert torch.equal(nobias, zero)
    plan.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4, 5, 8])
def test_steps_and_pieces_are_the_prompt(W, dtype):
    """A prompt, the same in two pieces, and token by token: the same bits (one
    order of the sums)."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C = 2, 11, 1, 12
    (x, _), (w, _), (b, _), _, _, _ = _inputs((B, N, L, C, W), dtype, 3, False)
    plan = P.SequencePlan(B, N, L, C)
    y, last = plan.conv(x, w, b)
    state, rows = plan.conv_state(W, x.dtype), []
    for t in range(N):
        rows.append(plan.conv_step(x[:, t].clone(memory_format=torch.contiguous_format), w, b, state))
    assert torch.equal(torch.stack(rows, 1), y) and torch.equal(state, last)
    for cut in (1, 4, N - 1):
        first, second = P.SequencePlan(B, cut, L, C), P.SequencePlan(B, N - cut, L, C)
        y1, s1 = first.conv(x[:, :cut].contiguous(), w, b)
        y2, s2 = second.conv(x[:, cut:].contiguous(), w, b, state=s1)
        assert torch.equal(torch.cat([y1, y2], 1), y) and torch.equal(s2, last)
        first.close()
        second.close()
    plan.close()


def test_nothing_behind_a_length_is_read():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, W = 3, 40, 1, 8, 4
    (x, _), (w, _), (b, _), (g, _), _, _ = _inputs((B, N, L, C, W), "fp32", 4, False)
    lengths = torch.tensor([40, 17, 0], dtype=torch.int32, device="cuda")
    plan = P.SequencePlan(B, N, L, C)
    clean = plan.conv(x, w, b, lengths), plan.conv_backward(x, w, b, g, lengths)
    xb, gb = x.clone(), g.clone()
    for t in (xb, gb):
        t[1, 17:] = float("nan")
        t[2] = float("inf")
    bad = plan.conv(xb, w, b, lengths), plan.conv_backward(xb, w, b, gb, lengths)
    for a, c in zip(clean[0] + clean[1], bad[0] + bad[1]):
        assert torch.equal(a, c)
    assert (clean[0][0][1, 17:] == 0).all() and (clean[1][0][2] == 0).all()
    # lengths out of range count as the nearest bound
    wild = torch.tensor([1000, 17, -5], dtype=torch.int32, device="cuda")
    assert torch.equal(plan.conv(x, w, b, wild)[0], clean[0][0])
    # a NaN reaches only the W outputs that read it
    xb = x.clone()
    xb[0, 10, 2, 3] = float("nan")
    diff = ~(plan.conv(xb, w, b, lengths)[0] == clean[0][0])
    hit = torch.zeros_like(diff)
    hit[0, 10:10 + W, 2, 3] = True
    assert torch.equal(diff, hit)
    plan.close()


@pytest.mark.parametrize("checkpoint", [None, "int8"])
def test_autograd(checkpoint):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    (x, _), (w, _), (b, _), (g, _), _, lengths = _inputs((2, 21, 2, 40, 4), "fp32", 8, True)
    n = _dev(torch, lengths)
    plan = P.SequencePlan(2, 21, 2, 40)
    leaves = [t.requires_grad_(True) for t in (x, w, b)]
    y = P.cgconv_short_conv(x, w, b, plan, lengths=n, checkpoint=checkpoint)
    got = torch.autograd.grad(y, leaves, g)
    with torch.no_grad():
        held = P.checkpoint_unpack(*P.checkpoint_pack(x)) if checkpoint else x
        assert torch.equal(y, plan.conv(x, w, b, n)[0])
        want = plan.conv_backward(held, w, b, g, n)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    plan.close()


def test_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    plan = P.SequencePlan(2, 5, 1, 8)
    x, w = torch.zeros(2, 5, 4, 8, device="cuda"), torch.zeros(4, 2, 8, device="cuda")
    for bad in (torch.zeros(1, 2, 8, device="cuda"), torch.zeros(9, 2, 8, device="cuda")):
        with pytest.raises(P.CgconvError, match="width"):
            plan.conv(x, bad)
    with pytest.raises(ValueError, match="weight"):
        plan.conv(x, w[:, :1])
    with pytest.raises(ValueError, match="lengths"):
        plan.conv(x, w, lengths=torch.tensor([5, 5], device="cuda"))  # int64
    with pytest.raises(ValueError, match="state"):
        plan.conv(x, w, state=torch.zeros(2, 2, 4, 8, device="cuda"))
    with pytest.raises(ValueError, match="state"):
        plan.conv_step(x[:, 0].contiguous(), w, None, torch.zeros(2, 3, 4, 8, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="x must"):
        plan.conv_step(x, w, None, plan.conv_state(4))
    plan.close()
