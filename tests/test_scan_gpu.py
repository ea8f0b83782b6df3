"""GPU parity of the selective scan (whole sequences, single tokens, gradients)
against the float64 oracle.

The bound of every element is the recurrence itself run on magnitudes, with the
error that fp32 adds at each step (_Bounds): u = 2^-24 is half a step.
  step     softplus: the exponential's argument is rounded once and scaled once,
           the series and the reciprocal take a few more: (2|v| + 12) u relative
  decay    exp(step A): the product and the step's own error times |step A|, the
           hardware exponential: (8 + |step A| (2|v| + 12)) u; the sums of up to
           64 steps over a chunk add at most 64 u |step A| more
  sums     one u per addition on the longest way to an element
"""

import numpy as np
import pytest

from oracle import sequence as S
from tests.seq_util import HALF, U, get, put, torch_gpu

pytestmark = pytest.mark.gpu

# (B, N, L, C, S): one token and state, every padded state count exact and not,
# several pieces and chunks with partial last ones, components in groups of 1, 3
# and 4 with and without a rest, columns in one and several blocks
SHAPES = [(1, 1, 0, 1, 1), (2, 5, 0, 3, 4), (1, 8, 1, 2, 8), (3, 33, 0, 70, 16), (2, 64, 2, 5, 16), (1, 300, 0, 64, 16),
          (2, 37, 1, 33, 32), (1, 40, 3, 40, 12), (2, 65, 0, 257, 16), (1, 100, 0, 130, 20), (1, 17, 6, 12, 24),
          (2, 96, 4, 3, 7), (1, 31, 5, 9, 32)]


def _inputs(shape, dtype, seed, ragged):
    B, N, L, C, St = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    t = {"x": put(r.normal(size=(B, N, K, C)), dtype), "delta": put(r.normal(size=(B, N, C)) * 1.5, dtype),
         "A": put(-np.exp(r.normal(size=(C, St)))), "Bt": put(r.normal(size=(B, N, St)), dtype),
         "Ct": put(r.normal(size=(B, N, St)), dtype), "D": put(r.normal(size=C)), "bias": put(r.normal(size=C) - 1.5)}
    g, state = put(r.normal(size=(B, N, K, C)), dtype), put(r.normal(size=(B, St, K, C)))
    lengths = r.integers(0, N + 1, size=B) if ragged else None
    if ragged:
        lengths[0] = N
        if B > 2:
            lengths[1] = 0
    return t, g, state, lengths


class _Bounds:
    """Magnitudes and errors (multiples of 1) of the recurrence on |inputs|."""

    def __init__(self, x, delta, A, Bt, Ct, D, bias, lengths=None, state=None):
        B, N, K, C = x.shape
        self.there = S._there(B, N, lengths)
        x = np.abs(np.where(self.there > 0, x, 0))
        v = delta + (0 if bias is None else bias)
        self.v, self.x, self.Bt, self.Ct, self.A = v, x, np.abs(Bt), np.abs(Ct), np.abs(A)
        self.D = np.zeros(C) if D is None else np.abs(D)
        self.d = S.softplus(v) * self.there[..., 0]
        self.ed = (2 * np.abs(v) + 12) * U
        h = np.zeros((B, A.shape[1], K, C)) if state is None else np.abs(state)
        he = np.zeros_like(h)
        self.h, self.he = [h], [he]
        self.y, self.ye = np.zeros_like(x), np.zeros_like(x)
        self.a, self.ea = [], []
        for t in range(N):
            on = self.there[:, t, None]
            z = self.d[:, t, None] * self.A.T
            a = np.exp(-z)[:, :, None]
            ea = ((8 + z * (2 * np.abs(v[:, t, None]) + 80)) * U)[:, :, None]
            add = self.Bt[:, t, :, None, None] * (self.d[:, t, None] * x[:, t])[:, None] * on
            he = a * (he + ea * h) + (self.ed[:, t, None, None] + 3 * U) * add
            h = a * h + add
            he = he + 2 * U * h
            self.a.append(a), self.ea.append(ea), self.h.append(h), self.he.append(he)
            cs = self.Ct[:, t, :, None, None]
            self.y[:, t] = ((cs * h).sum(1) + self.D * x[:, t]) * self.there[:, t]
            self.ye[:, t] = ((cs * he).sum(1) + (A.shape[1] + 4) * U * self.y[:, t]) * self.there[:, t]

    def backward(self, gy):
        B, N, K, C = self.x.shape
        St = self.A.shape[1]
        gy = np.abs(np.where(self.there > 0, gy, 0))
        sums = (96 + K * C / 64) * U  # lanes, waves, column blocks
        r, re = np.zeros_like(self.h[0]), np.zeros_like(self.h[0])
        out = {n: np.zeros(s) for n, s in (("x", self.x.shape), ("delta", self.v.shape), ("A", self.A.shape),
                                           ("Bt", self.Bt.shape), ("Ct", self.Ct.shape))}
        mA = np.zeros_like(self.A)
        raw = np.zeros(self.v.shape)
        for t in reversed(range(N)):
            on = self.there[:, t, 0]  # (B, 1)
            x, d, ed, gt = self.x[:, t], self.d[:, t], self.ed[:, t], gy[:, t]
            g = r + self.Ct[:, t, :, None, None] * gt[:, None]
            ge = re + 2 * U * g
            h, he = self.h[t + 1], self.he[t + 1]
            out["Ct"][:, t] = (gt[:, None] * (he + sums * h)).sum((2, 3)) * on
            dx = (d[:, None] * x)[:, None]
            out["Bt"][:, t] = (dx * (ge + g * (ed[:, None, None] + sums))).sum((2, 3)) * on
            into = (self.Bt[:, t, :, None, None] * g).sum(1)
            intoe = (self.Bt[:, t, :, None, None] * ge).sum(1) + (St + 2) * U * into
            dk, ek = d[:, None], ed[:, None]
            out["x"][:, t] = (dk * (intoe + into * ek) + 4 * U * (dk * into + self.D * gt)) * on[:, None]
            a, ea = self.a[t], self.ea[t]
            re = a * (ge + ea * g) + 2 * U * a * g
            r = a * g
            q, qe = r * self.h[t], re * self.h[t] + r * self.he[t] + 2 * U * r * self.h[t]
            q, qe = q.sum(2), (qe + (K + 4) * U * q).sum(2)  # (B, S, C)
            out["A"] += (d[:, None] * (qe + ed[:, None] * q)).sum(0).T
            mA += (d[:, None] * q).sum(0).T
            gd = (self.A.T * q).sum(1) + (into * x).sum(1)
            gde = (self.A.T * qe).sum(1) + (intoe * x).sum(1) + (St + K + 8) * U * gd
            sig = 1 / (1 + np.exp(-self.v[:, t]))
            out["delta"][:, t] = sig * (gde + gd * (12 + 3 * np.abs(self.v[:, t])) * U) * on
            raw[:, t] = sig * gd * on
        out["A"] += 256 * U * mA
        out["bias"] = out["delta"].sum((0, 1)) + 512 * U * raw.sum((0, 1))
        out["D"] = 512 * U * (gy * self.x).sum((0, 1, 2))
        return out


def close(name, got, ref, bound, dtype="fp32"):
    got = get(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    bound = bound + HALF[dtype] * (np.abs(ref) + bound) + 1e-37
    worst = np.max(np.abs(got - ref) / bound)
    assert worst <= 1, f"{name}: {worst:.3g} of the bound"


ORDER = ("x", "delta", "A", "Bt", "Ct", "D", "bias")


def _dev(torch, lengths):
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%dN%dL%dC%dS%d" % s)
def test_forward_and_gradients(shape, ragged, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, St = shape
    print(f"[gpu] scan {shape} {ragged} {dtype}", flush=True)
    t, (g, gv), (h0, h0v), lengths = _inputs(shape, dtype, 70 + N + C, ragged)
    dev, val = {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}
    n = _dev(torch, lengths)
    plan = P.SequencePlan(B, N, L, C, states=St)
    for state, sv in ((None, None), (h0, h0v)):
        y, last = plan.scan(dev["x"], dev["delta"], dev["A"], dev["Bt"], dev["Ct"], dev["D"], dev["bias"], n, state)
        ry, rh = S.scan(val["x"], val["delta"], val["A"], val["Bt"], val["Ct"], val["D"], val["bias"], lengths, sv)
        b = _Bounds(*(val[k] for k in ORDER), lengths, sv)
        close("y", y, ry, b.ye, dtype)
        close("state", last, rh, b.he[-1])
    grads = plan.scan_backward(*(dev[k] for k in ORDER[:-1]), g, dev["bias"], n)
    refs = S.scan_backward(*(val[k] for k in ORDER[:-1]), gv, val["bias"], lengths)
    bounds = _Bounds(*(val[k] for k in ORDER), lengths).backward(gv)
    for k, a, r in zip(ORDER, grads, refs):
        close("grad " + k, a, r, bounds[k], dtype if a.dtype == torch.bfloat16 else "fp32")
    again = plan.scan_backward(*(dev[k] for k in ORDER[:-1]), g, dev["bias"], n)
    assert all(torch.equal(a, c) for a, c in zip(grads, again))  # fixed orders
    for i in range(7):
        need = [j == i for j in range(7)]
        one = plan.scan_backward(*(dev[k] for k in ORDER[:-1]), g, dev["bias"], n, need=need)
        assert torch.equal(one[i], grads[i]) and all(o is None for j, o in enumerate(one) if j != i)
    # no D, no bias
    y, _ = plan.scan(dev["x"], dev["delta"], dev["A"], dev["Bt"], dev["Ct"], lengths=n)
    ry, _ = S.scan(val["x"], val["delta"], val["A"], val["Bt"], val["Ct"], None, None, lengths)
    close("plain y", y, ry, _Bounds(*(val[k] for k in ORDER[:5]), None, None, lengths).ye, dtype)
    plan.close()


@pytest.mark.parametrize("N", [64, 65, 256, 257, 1024, 1025, 4096, 4097, 8225])
def test_chunk_counts(N):
    """Both sides of every number of chunks at which the carry takes another form
    (chunks of 16 tokens backward, of 32 forward), with lengths."""
    test_forward_and_gradients((2, N, 0, 3, 4), True, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 6, 0, 1, 3), (3, 6, 1, 10, 16), (2, 6, 2, 33, 32), (1, 6, 0, 260, 16)], ids=str)
def test_steps(shape, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, St = shape
    t, _, (h0, h0v), _ = _inputs(shape, dtype, 20 + C, False)
    dev, val = {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}
    plan = P.SequencePlan(B, N, L, C, states=St)
    state = h0.clone()
    ry, rh = S.scan(*(val[k] for k in ORDER), None, h0v)
    b = _Bounds(*(val[k] for k in ORDER), None, h0v)
    whole = torch.contiguous_format
    ys = []
    for i in range(N):
        x, delta, Bt, Ct = (dev[k][:, i].clone(memory_format=whole) for k in ("x", "delta", "Bt", "Ct"))
        ys.append(plan.scan_step(x, delta, dev["A"], Bt, Ct, dev["D"], state, dev["bias"]))
    close("y", torch.stack(ys, 1), ry, b.ye, dtype)
    close("state", state, rh, b.he[-1])
    plan.close()


def test_pieces_are_the_prompt():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, St = 2, 90, 1, 24, 16
    t, _, (h0, h0v), _ = _inputs((B, N, L, C, St), "fp32", 5, False)
    dev, val = {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}
    cut = 41
    ys, state = [], h0
    for lo, hi in ((0, cut), (cut, N)):
        plan = P.SequencePlan(B, hi - lo, L, C, states=St)
        part = {k: dev[k][:, lo:hi].clone(memory_format=torch.contiguous_format) for k in ("x", "delta", "Bt", "Ct")}
        y, state = plan.scan(part["x"], part["delta"], dev["A"], part["Bt"], part["Ct"], dev["D"], dev["bias"], state=state)
        ys.append(y)
        torch.cuda.synchronize()
        plan.close()
    ry, rh = S.scan(*(val[k] for k in ORDER), None, h0v)
    b = _Bounds(*(val[k] for k in ORDER), None, h0v)
    close("y", torch.cat(ys, 1), ry, b.ye)
    close("state", state, rh, b.he[-1])


def test_long_rows():
    """Many chunks in both directions, slow and fast decays."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (1, 3001, 0, 40, 8)
    t, (g, gv), _, _ = _inputs(shape, "fp32", 6, False)
    A = -np.exp(np.random.default_rng(1).uniform(-9, 4, size=(40, 8)))
    t["A"] = put(A)
    dev, val = {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}
    plan = P.SequencePlan(1, 3001, 0, 40, states=8)
    y, last = plan.scan(dev["x"], dev["delta"], dev["A"], dev["Bt"], dev["Ct"], dev["D"], dev["bias"])
    ry, rh = S.scan(*(val[k] for k in ORDER))
    b = _Bounds(*(val[k] for k in ORDER))
    close("y", y, ry, b.ye)
    close("state", last, rh, b.he[-1])
    grads = plan.scan_backward(*(dev[k] for k in ORDER[:-1]), g, dev["bias"])
    refs = S.scan_backward(*(val[k] for k in ORDER[:-1]), gv, val["bias"])
    bounds = b.backward(gv)
    for k, a, r in zip(ORDER, grads, refs):
        close("grad " + k, a, r, bounds[k])
    plan.close()


def test_nothing_behind_a_length_is_read():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, St = 3, 80, 1, 20, 16
    t, (g, _), _, _ = _inputs((B, N, L, C, St), "fp32", 7, False)
    dev = {k: v[0] for k, v in t.items()}
    lengths = torch.tensor([80, 33, 0], dtype=torch.int32, device="cuda")
    plan = P.SequencePlan(B, N, L, C, states=St)

    def call(d, g):
        y, h = plan.scan(d["x"], d["delta"], d["A"], d["Bt"], d["Ct"], d["D"], d["bias"], lengths)
        return (y, h) + plan.scan_backward(*(d[k] for k in ORDER[:-1]), g, d["bias"], lengths)

    clean = call(dev, g)
    bad, gb = {k: v.clone() for k, v in dev.items()}, g.clone()
    for v in (bad["x"], bad["delta"], bad["Bt"], bad["Ct"], gb):
        v[1, 33:] = float("nan")
        v[2] = float("inf")
    for a, c in zip(clean, call(bad, gb)):
        assert torch.equal(a, c)
    assert (clean[0][1, 33:] == 0).all() and (clean[1][2] == 0).all()
    for i in (2, 3, 5, 6):  # gradients of x, delta, Bt, Ct behind a length
        assert (clean[i][1, 33:] == 0).all() and (clean[i][2] == 0).all()
    plan.close()


def test_masked_steps_and_vanishing_decays():
    """A step input of minus infinity, or of the lowest number, is a step of zero: the
    state passes by, y reads it, the step's gradient is zero.  Decays that vanish
    leave the token's own term; a step that is large keeps finite."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 45, 1, 12, 16)
    t, (g, gv), (h0, h0v), _ = _inputs(shape, "fp32", 31, False)
    raw = t["delta"][1].copy()
    raw[0, 3] = raw[1, 20:40] = -np.inf
    raw[0, 7] = np.finfo(np.float32).min
    raw[0, :, 5] = -np.inf  # a channel without any step
    raw[1, 2] = 60.0
    A = t["A"][1].copy()
    A[2, 4] = -1e30
    A[3, 1] = -0.0
    t["delta"], t["A"] = put(raw), put(A)
    dev, val = {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}
    seen = dict(val, delta=np.maximum(val["delta"], -200.0), A=np.maximum(val["A"], -1e4))  # for the bounds only
    plan = P.SequencePlan(*shape[:4], states=16)
    with np.errstate(over="ignore"):
        y, last = plan.scan(*(dev[k] for k in ORDER), state=h0)
        ry, rh = S.scan(*(val[k] for k in ORDER), None, h0v)
        b = _Bounds(*(seen[k] for k in ORDER), None, h0v)
        close("y", y, ry, b.ye)
        close("state", last, rh, b.he[-1])
        grads = plan.scan_backward(*(dev[k] for k in ORDER[:-1]), g, dev["bias"])
        refs = S.scan_backward(*(val[k] for k in ORDER[:-1]), gv, val["bias"])
        bounds = _Bounds(*(seen[k] for k in ORDER)).backward(gv)
    for k, a, r in zip(ORDER, grads, refs):
        close("grad " + k, a, r, bounds[k])
    assert (grads[1][1, 20:40] == 0).all() and (grads[1][0, :, 5] == 0).all()
    plan.close()


@pytest.mark.parametrize("checkpoint", [None, "int8"])
def test_autograd(checkpoint):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, St = 2, 40, 1, 36, 16
    t, (g, _), _, lengths = _inputs((B, N, L, C, St), "fp32", 9, True)
    dev = {k: v[0].requires_grad_(True) for k, v in t.items()}
    n = _dev(torch, lengths)
    plan = P.SequencePlan(B, N, L, C, states=St)
    y = P.cgconv_scan(*(dev[k] for k in ORDER[:-1]), plan, delta_bias=dev["bias"], lengths=n, checkpoint=checkpoint)
    got = torch.autograd.grad(y, [dev[k] for k in ORDER], g)
    with torch.no_grad():
        held = P.checkpoint_unpack(*P.checkpoint_pack(dev["x"])) if checkpoint else dev["x"]
        want = plan.scan_backward(held, *(dev[k] for k in ORDER[1:-1]), g, dev["bias"], n)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    # without D and bias, one leaf
    y = P.cgconv_scan(*(dev[k].detach() for k in ORDER[:2]), dev["A"], dev["Bt"].detach(), dev["Ct"].detach(), None, plan)
    gA, = torch.autograd.grad(y, (dev["A"],), g)
    assert gA.shape == dev["A"].shape
    plan.close()


def test_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    t, (g, _), _, _ = _inputs((2, 5, 1, 8, 4), "fp32", 9, False)
    d = {k: v[0] for k, v in t.items()}
    none = P.SequencePlan(2, 5, 1, 8)
    with pytest.raises(ValueError):  # A of [C, 0]
        none.scan(d["x"], d["delta"], d["A"], d["Bt"], d["Ct"])
    plan = P.SequencePlan(2, 5, 1, 8, states=4)
    for k, bad in (("x", d["x"][:1]), ("delta", d["delta"].to(torch.bfloat16)), ("A", d["A"].T), ("Bt", d["Bt"][..., :2]),
                   ("Ct", d["Ct"].cpu()), ("D", d["D"][:3])):
        with pytest.raises(ValueError, match=k):
            plan.scan(*(bad if n == k else d[n] for n in ORDER[:-1]))
    with pytest.raises(ValueError, match="state"):
        plan.scan(*(d[k] for k in ORDER[:-1]), state=torch.zeros(2, 4, 4, 7, device="cuda"))
    with pytest.raises(P.CgconvError, match="overlap"):
        plan.scan(*(d[k] for k in ORDER[:-1]), out=d["x"])
    plan.close()
    none.close()
