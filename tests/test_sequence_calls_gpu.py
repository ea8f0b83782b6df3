"""Calls of the sequence operators that the documentation allows beside the usual
ones: results into the caller's tensors, 8-bit inputs of a padded batch, training
steps captured through autograd, inputs changed after a checkpointed forward, two
plans at work on two streams, the same leaf twice."""

import pytest

from tests.seq_util import put, torch_gpu
from tests.test_sequence_block_gpu import B, C, K, L, N, NAMES, ST, W, _block, _parameters

pytestmark = pytest.mark.gpu


def test_results_into_the_callers_tensors():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, _ = _parameters(21)
    t = {k: put(v)[0] for k, v in p.items()}
    seq, one = P.SequencePlan(B, N, L, C, states=ST), P.SequencePlan(B, 1, L, C, states=ST)
    scan = [t[k] for k in ("x", "delta", "A", "Bt", "Ct", "D", "db")]
    out = torch.full_like(t["x"], 9)
    for call in (lambda **o: seq.norm(t["x"], t["w1"], t["b1"], **o), lambda **o: seq.conv(t["x"], t["cw"], t["cb"], **o),
                 lambda **o: seq.scan(*scan, **o)):
        want = call()
        got = call(out=out)
        assert got[0] is out and all(torch.equal(a, b) for a, b in zip(got, want))
        with pytest.raises(ValueError, match="out"):
            call(out=out.to(torch.bfloat16))
        with pytest.raises(P.CgconvError, match="overlap"):
            call(out=t["x"])
    xt, dt, bt, ct = (v[:, 0].clone() for v in (t["x"], t["delta"], t["Bt"], t["Ct"]))
    out = torch.full_like(xt, 9)
    for state, call in ((one.conv_state(W), lambda s, **o: one.conv_step(xt, t["cw"], t["cb"], s, **o)),
                        (one.scan_state(), lambda s, **o: one.scan_step(xt, dt, t["A"], bt, ct, t["D"], s, t["db"], **o))):
        mine = state.clone()
        want = call(state)
        assert call(mine, out=out) is out and torch.equal(out, want) and torch.equal(mine, state)
        with pytest.raises(P.CgconvError, match="overlap"):
            call(mine, out=xt)
    codes, scales = P.checkpoint_pack(t["x"])
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full(t["x"].shape, 9, dtype=dtype, device="cuda")
        assert P.checkpoint_unpack(codes, scales, out=out) is out
        assert torch.equal(out, P.checkpoint_unpack(codes, scales, dtype=dtype))
    seq.close()
    one.close()


@pytest.mark.parametrize("name", ["conv", "scan"])
def test_checkpoints_of_a_padded_batch(name):
    """What stands behind the lengths, NaN and infinities, is kept in 8 bits like the
    rest and reaches no gradient."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, g = _parameters(22)
    seq, gt = P.SequencePlan(B, N, L, C, states=ST), put(g)[0]
    n = torch.tensor([N - 9, 0], dtype=torch.int32, device="cuda")

    def grads(fill):
        t = {k: put(v)[0] for k, v in p.items()}
        for k in ("x", "delta", "Bt", "Ct"):
            t[k][0, N - 9:], t[k][1] = fill, -fill
        bad = gt.clone()
        bad[0, N - 9:], bad[1] = fill, fill
        leaves = [v.requires_grad_() for k, v in t.items() if k in {
            "conv": ("x", "cw", "cb"), "scan": ("x", "delta", "A", "Bt", "Ct", "D", "db")}[name]]
        if name == "conv":
            y = P.cgconv_short_conv(t["x"], t["cw"], t["cb"], seq, lengths=n, checkpoint="int8")
        else:
            y = P.cgconv_scan(t["x"], t["delta"], t["A"], t["Bt"], t["Ct"], t["D"], seq, delta_bias=t["db"], lengths=n,
                              checkpoint="int8")
        return (y.detach(),) + torch.autograd.grad(y, leaves, bad)

    clean = grads(0.0)
    for fill in (float("nan"), float("inf"), torch.finfo(torch.float32).max):
        assert all(torch.equal(a, b) for a, b in zip(grads(fill), clean))
    seq.close()


@pytest.mark.parametrize("checkpoint", [None, "int8"])
def test_captured_training_step(checkpoint):
    """Forward and backward of the block through autograd in one graph, replayed on
    other inputs with eager steps of the same plans between: the eager gradients."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    seq, plan = P.SequencePlan(B, N, L, C, states=ST), P.Plan(B, N, L, C, boundary="linear")

    def step(t, g):
        y = _block(P, t, seq, plan, checkpoint)
        return (y.detach(),) + torch.autograd.grad(y, [t[n] for n in NAMES], g)

    sets = []
    for seed in (23, 24):
        p, g = _parameters(seed)
        sets.append(({k: put(v)[0].requires_grad_() for k, v in p.items()}, put(g)[0]))
    eager = [step(*s) for s in sets]
    static = {k: v.detach().clone().requires_grad_() for k, v in sets[0][0].items()}
    sg = sets[0][1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(static, sg)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(static, sg)
    for i in (0, 1, 0, 1):
        with torch.no_grad():
            for k, v in sets[i][0].items():
                static[k].copy_(v)
        sg.copy_(sets[i][1])
        graph.replay()
        got = [o.clone() for o in outs]
        again = step(*sets[1 - i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[i]))
        assert all(torch.equal(a, b) for a, b in zip(again, eager[1 - i]))
    seq.close()
    plan.close()


def test_input_changed_after_a_checkpointed_forward():
    """The 8 bits are the input's own copy: it may be overwritten before the backward."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, g = _parameters(25)
    t, gt = {k: put(v)[0] for k, v in p.items()}, put(g)[0]
    seq = P.SequencePlan(B, N, L, C, states=ST)
    for leaf, op in ((t["w1"].requires_grad_(), lambda x: P.cgconv_norm(x, t["w1"], None, seq, checkpoint="int8")),
                     (t["cw"].requires_grad_(), lambda x: P.cgconv_short_conv(x, t["cw"], None, seq, checkpoint="int8"))):
        want, = torch.autograd.grad(op(t["x"].clone()), leaf, gt)
        x = t["x"].clone()
        y = op(x)
        x.fill_(float("nan"))
        got, = torch.autograd.grad(y, leaf, gt)
        assert torch.equal(got, want)
    # kept whole, a change is an error
    x = t["x"].clone()
    y = P.cgconv_norm(x, t["w1"], None, seq)
    x.fill_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, t["w1"], gt)
    seq.close()


def test_two_plans_on_two_streams():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    n, c = 4096, 64
    gen = torch.Generator("cuda").manual_seed(26)
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    sets = []
    for _ in range(2):
        sets.append([f(1, n, 4, c), f(1, n, c), -f(c, ST).abs(), f(1, n, ST), f(1, n, ST), f(c)])
    plans = [P.SequencePlan(1, n, 1, c, states=ST) for _ in sets]
    g = f(1, n, 4, c)
    call = lambda plan, s: plan.scan(*s) + plan.scan_backward(*s, g) + plan.conv_backward(s[0], s[0][0, :4, :2].contiguous(), None, g)  # noqa: E731
    want = [call(p, s) for p, s in zip(plans, sets)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(call(plans[i], sets[i]))
    torch.cuda.synchronize()
    for i, results in enumerate(got):
        for r in results:
            assert all(torch.equal(a, b) for a, b in zip(r, want[i]))
    for p in plans:
        p.close()


def test_the_same_leaf_twice():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, g = _parameters(27)
    gt = put(g)[0]
    plan = P.Plan(B, N, L, C, boundary="linear")
    q = put(p["x"])[0].requires_grad_()
    for checkpoint in (None, "int8"):
        both, = torch.autograd.grad(P.cgconv(q, q, plan, checkpoint=checkpoint), q, gt)
        held = P.checkpoint_unpack(*P.checkpoint_pack(q.detach())) if checkpoint else q.detach()
        gq, gk = plan.backward(held, held, gt)
        assert torch.equal(both, gq + gk)
    plan.close()
    assert K == (L + 1) ** 2
