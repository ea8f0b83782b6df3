"""The delta rule, the norms around the residual connection and the clipping together
with the operators they stand beside, as a causal block uses them: a training step
against the composed float64 oracle, prompts and tokens, HIP graphs, streams, results
into the caller's tensors, padded batches in 8 bits."""

import numpy as np
import pytest

from oracle import memory as M
from oracle import sequence as S
from tests.conftest import rel_l2
from tests.seq_util import get, put, torch_gpu

pytestmark = pytest.mark.gpu

B, N, L, C, H, HK, D, W = 2, 150, 1, 16, 4, 2, 24, 4
K = (L + 1) ** 2
EPS = 1e-5
NAMES = ("x", "w1", "b1", "cw", "cb", "q", "k", "decay", "beta", "gate", "po", "sc", "w2", "b2")


def _parameters(seed):
    r = np.random.default_rng(seed)
    f = lambda *s: r.normal(size=s)  # noqa: E731
    p = {"x": f(B, N, K, C), "w1": 1 + 0.1 * f(L + 1, C), "b1": 0.1 * f(C), "cw": f(W, L + 1, C) / 2, "cb": 0.1 * f(C),
         "q": f(B, N, HK, D), "k": f(B, N, HK, D), "decay": -np.exp(f(B, N, H) - 2), "beta": 1 / (1 + np.exp(-f(B, N, H))),
         "gate": f(B, N, C), "po": 1 + 0.1 * f(L + 1, C), "sc": 0.5 + 0.1 * f(C), "w2": 1 + 0.1 * f(L + 1, C), "b2": 0.1 * f(C)}
    return {n: np.asarray(v, dtype=np.float32) for n, v in p.items()}, [np.asarray(f(B, N, K, C), dtype=np.float32) for _ in "ry"]


def _oracle(p, gr, gy):
    """h = norm(x), c = conv(h), m = delta(q, k, c), (r, y) = residual(x, m, gate); all gradients."""
    p = {n: v.astype(np.float64) for n, v in p.items()}
    h = S.norm(p["x"], p["w1"], p["b1"], L, EPS)
    c, _ = S.conv(h, p["cw"], p["cb"], L)
    rule = (p["q"], p["k"], c, p["decay"], p["beta"])
    m, _ = M.delta_rule(*rule)
    res = (p["x"], m, p["gate"], p["po"], p["sc"], p["w2"], p["b2"])
    r, y = M.residual(*res, L, EPS)
    gx, gm, gg, gpo, gsc, gw2, gb2 = M.residual_backward(*res, gr, gy, L, EPS)
    gq, gk, gc, gd, gb, _ = M.delta_rule_backward(*rule, gm)
    gh, gcw, gcb = S.conv_backward(h, p["cw"], p["cb"], gc, L)
    gx1, gw1, gb1 = S.norm_backward(p["x"], p["w1"], gh, L, EPS)
    return (r, y), (gx + gx1, gw1, gb1, gcw, gcb, gq, gk, gd, gb, gg, gpo, gsc, gw2, gb2)


def _block(P, t, seq, checkpoint=None):
    h = P.cgconv_norm(t["x"], t["w1"], t["b1"], seq, EPS, checkpoint=checkpoint)
    c = P.cgconv_short_conv(h, t["cw"], t["cb"], seq, checkpoint=checkpoint)
    m = P.cgconv_delta_rule(t["q"], t["k"], c, t["decay"], t["beta"], seq, checkpoint=checkpoint)
    return P.cgconv_residual_norm(t["x"], m, t["gate"], t["po"], t["sc"], t["w2"], t["b2"], seq, EPS, checkpoint=checkpoint)


def _plan(P, n=N, **kw):
    return P.SequencePlan(B, n, L, C, heads=H, key_heads=HK, key_dim=D, **kw)


def _step(P, t, seq, gr, gy, checkpoint=None):
    """Outputs, clipped gradients and their norm."""
    import torch
    r, y = _block(P, t, seq, checkpoint)
    grads = torch.autograd.grad((r, y), [t[n] for n in NAMES], (gr, gy))
    norm = P.clip_gradients(grads, 1.0)
    return (r.detach(), y.detach(), norm) + grads


def test_training_step_of_a_block():
    """Bar: the library's 1e-4 relative L2 in fp32 (a chain of four operators, each within
    a few 1e-6).  With 8-bit checkpoints a kept value moves by at most 1/127 of its group's
    largest: 0.7% of the norm; the gradients are made of five such inputs."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, g = _parameters(1)
    outs, grads = _oracle(p, *(x.astype(np.float64) for x in g))
    norm, grads = M.clip(grads, 1.0, 1e-6)
    seq = _plan(P)
    gr, gy = (put(x)[0] for x in g)
    for checkpoint, bar in ((None, 1e-4), ("int8", 0.06)):
        t = {n: put(v)[0].requires_grad_(True) for n, v in p.items()}
        got = _step(P, t, seq, gr, gy, checkpoint)
        assert all(rel_l2(get(a), o) <= 1e-4 for a, o in zip(got, outs))
        assert abs(float(got[2]) - norm) <= bar * norm
        for n, a, o in zip(NAMES, got[3:], grads):
            assert rel_l2(get(a), o) <= bar, (checkpoint, n, rel_l2(get(a), o))
    seq.close()


@pytest.mark.parametrize("checkpoint", [None, "int8"])
def test_captured_training_step(checkpoint):
    """Forward, backward through autograd and clipping in one graph, replayed on other
    inputs with eager steps of the same plan between: the eager results."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    seq = _plan(P)
    sets = []
    for seed in (2, 3):
        p, g = _parameters(seed)
        sets.append(({n: put(v)[0].requires_grad_() for n, v in p.items()}, [put(x)[0] for x in g]))
    eager = [[x.clone() for x in _step(P, t, seq, *g, checkpoint)] for t, g in sets]
    static = {n: v.detach().clone().requires_grad_() for n, v in sets[0][0].items()}
    sg = [x.clone() for x in sets[0][1]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(P, static, seq, *sg, checkpoint)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _step(P, static, seq, *sg, checkpoint)
    for i in (0, 1, 0, 1):
        with torch.no_grad():
            for n, v in sets[i][0].items():
                static[n].copy_(v)
        for s, x in zip(sg, sets[i][1]):
            s.copy_(x)
        graph.replay()
        got = [o.clone() for o in outs]
        again = _step(P, sets[1 - i][0], seq, *sets[1 - i][1], checkpoint)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[i]))
        assert all(torch.equal(a, b) for a, b in zip(again, eager[1 - i]))
    seq.close()


def test_captured_tokens():
    """A token's step through the block in a graph: the states move on with every replay,
    and the tokens are those of the whole sequence (1e-5 of the largest: the same sums in
    another order)."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, _ = _parameters(4)
    t = {n: put(v)[0] for n, v in p.items()}
    seq, one = _plan(P), _plan(P, 1, backward=False)
    with torch.no_grad():
        want = _block(P, t, seq)
    cur = {n: t[n][:, 0].clone() for n in ("x", "q", "k", "decay", "beta", "gate")}

    def step(cs, ms):
        h = one.norm(cur["x"][:, None], t["w1"], t["b1"], EPS)[0]
        c = one.conv_step(h[:, 0], t["cw"], t["cb"], cs)
        m = one.delta_rule_step(cur["q"], cur["k"], c, cur["decay"], cur["beta"], ms)
        return one.residual_norm(cur["x"][:, None], m[:, None], cur["gate"][:, None], t["po"], t["sc"], t["w2"], t["b2"], EPS)[:2]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(one.conv_state(W), one.delta_rule_state())
    torch.cuda.synchronize()
    cs, ms = one.conv_state(W), one.delta_rule_state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cs, ms)
    cs.zero_()
    ms.zero_()
    for i in range(20):
        for n in cur:
            cur[n].copy_(t[n][:, i])
        graph.replay()
        torch.cuda.synchronize()
        for a, w in zip(out, want):
            assert float((a[:, 0] - w[:, i]).abs().max()) <= 1e-5 * float(w.abs().max())
    seq.close()
    one.close()


def test_streams_and_plans():
    """Two plans at work on two streams, behind other work there: the results of each alone."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    sets, plans = [], [_plan(P) for _ in range(2)]
    for seed in (5, 6):
        p, g = _parameters(seed)
        sets.append(({n: put(v)[0].requires_grad_() for n, v in p.items()}, [put(x)[0] for x in g]))
    want = [[x.clone() for x in _step(P, t, plan, *g)] for plan, (t, g) in zip(plans, sets)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in plans], [[], []]
    late = [None, None]
    for i, st in enumerate(streams):
        with torch.cuda.stream(st):
            a = torch.randn(2048, 2048, device="cuda")
            for _ in range(4):
                a = a @ a * 1e-4
            late[i] = {n: (v.detach() + 0 * a[0, 0].nan_to_num()).requires_grad_() for n, v in sets[i][0].items()}
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(_step(P, late[i], plans[i], *sets[i][1]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r, want[i]))
    for p in plans:
        p.close()


def test_long_sequences_on_two_streams():
    """Sequences in segments, whose workspaces are the plans' own."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    n, h, d = 2048, 2, 32
    gen = torch.Generator("cuda").manual_seed(7)
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    sets = [[f(1, n, h, d), f(1, n, h, d), f(1, n, 1, 64), -f(1, n, h).abs() / 8, torch.sigmoid(f(1, n, h))] for _ in range(2)]
    gy = f(1, n, 1, 64)
    plans = [P.SequencePlan(1, n, 0, 64, heads=h, key_dim=d) for _ in sets]
    call = lambda plan, s: plan.delta_rule(*s) + plan.delta_rule_backward(*s, gy, need=(True,) * 5 + (False,))[:5]  # noqa: E731
    want = [[x.clone() for x in call(p, s)] for p, s in zip(plans, sets)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(call(plans[i], sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for r in got[i] for a, b in zip(r, want[i]))
    for p in plans:
        p.close()


def test_results_into_the_callers_tensors():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, _ = _parameters(8)
    t = {n: put(v)[0] for n, v in p.items()}
    seq, one = _plan(P, backward=False), _plan(P, 1, backward=False)
    rule = [t[n] for n in ("q", "k", "x", "decay", "beta")]
    out = torch.full_like(t["x"], 9)
    want, got = seq.delta_rule(*rule), seq.delta_rule(*rule, out=out)
    assert got[0] is out and all(torch.equal(a, b) for a, b in zip(got, want))
    res = [t[n] for n in ("x", "x", "gate", "po", "sc", "w2", "b2")]
    other = torch.full_like(out, 9)
    want, got = seq.residual_norm(*res), seq.residual_norm(*res, out_r=out, out_y=other)
    assert got[0] is out and got[1] is other and all(torch.equal(a, b) for a, b in zip(got, want))
    tok = [v[:, 0].clone() for v in rule]
    s1, s2 = seq.delta_rule_state() + 1, seq.delta_rule_state() + 1
    mine = torch.full_like(tok[2], 9)
    want = one.delta_rule_step(*tok, s1)
    assert one.delta_rule_step(*tok, s2, out=mine) is mine and torch.equal(mine, want) and torch.equal(s1, s2)
    with pytest.raises(P.CgconvError, match="overlap"):
        one.delta_rule_step(*tok, s2, out=tok[2])
    for bad in (out.to(torch.bfloat16), out[:1]):
        with pytest.raises(ValueError, match="out"):
            seq.delta_rule(*rule, out=bad)
    seq.close()
    one.close()


def test_checkpoint_of_a_padded_batch():
    """What stands behind the lengths, NaN and infinities, is kept in 8 bits like the rest
    and reaches no gradient."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    p, g = _parameters(9)
    seq, gy = _plan(P), put(g[1])[0]
    n = torch.tensor([N - 9, 0], dtype=torch.int32, device="cuda")

    def grads(fill):
        t = [put(p[k])[0] for k in ("q", "k", "x", "decay", "beta")]
        bad = gy.clone()
        for v in t + [bad]:
            v[0, N - 9:], v[1] = fill, -fill
        leaves = [v.requires_grad_() for v in t]
        y = P.cgconv_delta_rule(*leaves, seq, lengths=n, checkpoint="int8")
        return (y.detach(),) + torch.autograd.grad(y, leaves, bad)

    clean = grads(0.0)
    for fill in (float("nan"), float("inf"), torch.finfo(torch.float32).max):
        assert all(torch.equal(a, b) for a, b in zip(grads(fill), clean))
    seq.close()


def test_gradient_that_starts_off_a_vector():
    """A part of a concatenation sends a gradient that starts anywhere."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    n, c, h, d = 7, 5, 1, 3
    seq = P.SequencePlan(1, n, 0, c, heads=h, key_dim=d)
    gen = torch.Generator(device="cuda").manual_seed(4)
    f = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").requires_grad_()  # noqa: E731
    q, k, x, decay, beta = f(1, n, h, d), f(1, n, h, d), f(1, n, 1, c), f(1, n, h), f(1, n, h)
    head = f(1, 1, 1, c)
    for op in (lambda: P.cgconv_delta_rule(q, k, x, -decay.detach().abs(), beta, seq),
               lambda: P.cgconv_residual_norm(x, x, None, None, None, None, None, seq)[1]):
        g = torch.randn(1, n + 1, 1, c, generator=gen, device="cuda")
        assert g[:, 1:].data_ptr() % 16
        want, = torch.autograd.grad(op(), x, g[:, 1:].clone())
        got, = torch.autograd.grad(torch.cat((head, op()), 1), x, g)
        assert torch.equal(got, want)
    seq.close()
