"""What is not finite in the gated delta rule, and how far it reaches.  A token's inputs
reach its own output and those of later tokens, an output's gradient the gradients of its
own and earlier tokens, so nothing before (behind) the token of a NaN or an infinity
changes by a bit: neither in its chunk of 64 tokens nor in another, nor in another column
of the values, head or sequence, unless the formula takes it there.

Checked bit by bit against the same call with a number in that place: where the formula
has no path from the place to an element, the products that stand for it are with zeros.
"""

import math

import numpy as np
import pytest

from tests.seq_util import put, torch_gpu

pytestmark = pytest.mark.gpu

# (B, N, L, C, H, D): one chunk, several, in segments; widths of one and more tiles of keys, of
# one and several blocks of columns, of several components
SHAPES = [(2, 64, 0, 12, 2, 16), (2, 150, 1, 16, 2, 40), (1, 200, 0, 272, 2, 128), (1, 1100, 0, 144, 1, 100),
          (2, 700, 0, 24, 2, 20)]
TOKENS = {64: (0, 1, 15, 16, 37, 62, 63), 150: (31, 64, 149), 200: (47, 100), 1100: (33, 600, 1090), 700: (350, 640)}
TYPES = ["fp32", "bf16"]
ID = lambda s: "B%dN%dL%dC%dH%dD%d" % s  # noqa: E731


def _inputs(shape, dtype, seed):
    B, N, L, C, H, D = shape
    r = np.random.default_rng(seed)
    K = (L + 1) ** 2
    a = [put(r.normal(size=(B, N, H, D)), dtype)[0], put(r.normal(size=(B, N, H, D)), dtype)[0],
         put(r.normal(size=(B, N, K, C)), dtype)[0], put(-np.exp(r.normal(size=(B, N, H)) - 3))[0],
         put(1 / (1 + np.exp(-r.normal(size=(B, N, H)))))[0]]
    return a, put(r.normal(size=(B, D, K, C)))[0], put(r.normal(size=(B, N, K, C)), dtype)[0], put(r.normal(size=(B, D, K, C)))[0]


def _plan(P, shape, **kw):
    B, N, L, C, H, D = shape
    return P.SequencePlan(B, N, L, C, heads=H, key_heads=H, key_dim=D, **kw)


def _head(C, H, h):
    return slice(h * (C // H), (h + 1) * (C // H))


def _same(torch, name, got, want, where):
    """got is want where `where` is true."""
    assert torch.equal(got[where], want[where]), (name, int((got != want)[where].sum()), "of", int(where.sum()))


def _odd(torch, name, got, where):
    """got is not finite where `where` is true."""
    assert not torch.isfinite(got[where]).any(), (name, int(torch.isfinite(got[where]).sum()), "of", int(where.sum()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=ID)
def test_outputs(shape, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, H, D = shape
    print(f"[gpu] not finite {shape} {dtype}", flush=True)
    a, s, _, _ = _inputs(shape, dtype, 1)
    plan = _plan(P, shape, backward=False)
    y, last = plan.delta_rule(*a, state=s)
    assert torch.isfinite(y).all() and torch.isfinite(last).all()
    b, h = B - 1, H - 1
    head = _head(C, H, h)
    places = {"q": (0, (h, D // 2)), "k": (1, (h, D - 1)), "v": (2, (0, head.start + 1)), "decay": (3, (h,)), "beta": (4, (h,))}
    for t in TOKENS[N]:
        for name, (i, at) in places.items():
            for value in (math.nan, math.inf) + ((-math.inf,) if i != 3 else ()):
                bad = [x.clone() for x in a]
                bad[i][(b, t) + at] = value
                got, state = plan.delta_rule(*bad, state=s)
                hit = torch.zeros(y.shape, dtype=torch.bool, device="cuda")
                lost = torch.zeros(last.shape, dtype=torch.bool, device="cuda")
                if name == "v":
                    hit[b, t:, 0, at[1]] = True
                    lost[b, :, 0, at[1]] = True
                else:
                    hit[b, t:t + 1 if name == "q" else N, :, head] = True
                    lost[b, :, :, head] = name != "q"
                _same(torch, (name, t, value, "y"), got, y, ~hit)
                _same(torch, (name, t, value, "state"), state, last, ~lost)
                _odd(torch, (name, t, value, "y"), got, hit)
                _odd(torch, (name, t, value, "state"), state, lost)
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=ID)
def test_gradients(shape, dtype):
    """A value reaches the gradients of its own token's and later keys, queries and betas and
    of later decays, but no value's and not the first state's; an output's gradient those of its
    own token's query, and of its own and earlier keys, values, decays and betas; a column of
    the first state no value's gradient, a column of the last state's gradient no query's."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, H, D = shape
    a, s, gy, gs = _inputs(shape, dtype, 2)
    plan = _plan(P, shape)
    want = plan.delta_rule_backward(*a, gy, state=s, grad_state=gs)
    names = ("q", "k", "v", "decay", "beta", "state")
    assert all(torch.isfinite(x).all() for x in want)
    b, h = B - 1, H - 1
    head = _head(C, H, h)
    col = head.start + 1

    def reached(**rows):
        """Masks: the tokens of `rows` in head h (of the values and the state: in the column)."""
        out = [torch.zeros(x.shape, dtype=torch.bool, device="cuda") for x in want]
        for n, r in rows.items():
            m = out[names.index(n)]
            if n == "state":
                m[b, :, 0, col] = True
            elif n == "v":
                m[b, r, 0, col] = True
            else:
                m[b, r, h] = True
        return out

    def check(tag, got, hit):
        for n, x, w, m in zip(names, got, want, hit):
            _same(torch, tag + (n,), x, w, ~m)
            _odd(torch, tag + (n,), x, m)

    def replaced(x, place, value):
        x = x.clone()
        x[place] = value
        return x

    for value in (math.nan, math.inf):
        for t in TOKENS[N]:
            place, on, to = (b, t, 0, col), slice(t, N), slice(0, t + 1)
            got = plan.delta_rule_backward(*a[:2], replaced(a[2], place, value), *a[3:], gy, state=s, grad_state=gs)
            check(("v", t, value), got, reached(q=on, k=on, decay=slice(t + 1, N), beta=on))
            got = plan.delta_rule_backward(*a, replaced(gy, place, value), state=s, grad_state=gs)
            check(("gy", t, value), got, reached(q=slice(t, t + 1), k=to, v=to, decay=to, beta=to, state=0))
        every = slice(0, N)
        got = plan.delta_rule_backward(*a, gy, state=replaced(s, (b, 0, 0, col), value), grad_state=gs)
        check(("state", value), got, reached(q=every, k=every, decay=every, beta=every))
        got = plan.delta_rule_backward(*a, gy, state=s, grad_state=replaced(gs, (b, 0, 0, col), value))
        check(("gstate", value), got, reached(k=every, v=every, decay=every, beta=every, state=0))
    # a key, query, decay or beta: at most its head's, of its sequence
    for i in (0, 1, 3, 4):
        bad = list(a)
        bad[i] = replaced(a[i], (b, TOKENS[N][-1], h) + ((D // 2,) if i < 2 else ()), math.nan)
        got = plan.delta_rule_backward(*bad, gy, state=s, grad_state=gs)
        for n, x, w in zip(names, got, want):
            mask = torch.ones(w.shape, dtype=torch.bool, device="cuda")
            if n in ("v", "state"):
                mask[b, :, :, head] = False
            else:
                mask[b, :, h] = False
            _same(torch, (i, n), x, w, mask)
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_the_last_token_of_a_partial_chunk(dtype):
    """Lengths: a NaN in the last token changes nothing before it, and what is behind stays zero."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (2, 100, 0, 16, 2, 24)
    a, s, gy, gs = _inputs(shape, dtype, 3)
    plan = _plan(P, shape)
    n = torch.tensor([70, 41], dtype=torch.int32, device="cuda")
    y, last = plan.delta_rule(*a, lengths=n, state=s)
    for b, e in ((0, 70), (1, 41)):
        bad = a[2].clone()
        bad[b, e - 1] = math.nan
        got, state = plan.delta_rule(*a[:2], bad, *a[3:], lengths=n, state=s)
        assert torch.equal(got[1 - b], y[1 - b]) and torch.equal(got[b, :e - 1], y[b, :e - 1])
        assert torch.isnan(got[b, e - 1]).all() and (got[b, e:] == 0).all()
        assert torch.equal(state[1 - b], last[1 - b]) and torch.isnan(state[b]).all()
        grads = plan.delta_rule_backward(*a[:2], bad, *a[3:], gy, lengths=n, state=s, grad_state=gs)
        for x in grads[:5]:
            assert torch.isfinite(x[1 - b]).all() and torch.isfinite(x[b, :e - 1]).all() and (x[b, e:] == 0).all()
        assert torch.isfinite(grads[2]).all() and torch.isfinite(grads[5]).all()
        late = gy.clone()
        late[b, e - 1] = math.nan
        grads = plan.delta_rule_backward(*a, late, lengths=n, state=s, grad_state=gs)
        for x in grads[:5]:
            assert torch.isfinite(x[1 - b]).all() and (x[b, e:] == 0).all()
        assert torch.isfinite(grads[0][b, :e - 1]).all() and torch.isnan(grads[2][b, :e]).all()
    plan.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_one_by_one_agree(dtype):
    """The same numbers are finite as where the tokens come one by one."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    shape = (1, 70, 0, 8, 2, 16)
    a, s, _, _ = _inputs(shape, dtype, 4)
    whole, one = _plan(P, shape, backward=False), _plan(P, (1, 1) + shape[2:], backward=False)
    for i, place in ((0, (0, 40, 1, 3)), (1, (0, 40, 1, 3)), (2, (0, 40, 0, 5)), (3, (0, 40, 1)), (4, (0, 40, 1))):
        bad = [x.clone() for x in a]
        bad[i][place] = math.nan
        y, last = whole.delta_rule(*bad, state=s)
        state = s.clone()
        each = [one.delta_rule_step(*(x[:, t].clone() for x in bad), state) for t in range(70)]
        assert torch.equal(torch.isfinite(torch.stack(each, 1)), torch.isfinite(y)), i
        assert torch.equal(torch.isfinite(state), torch.isfinite(last)), i
    whole.close()
    one.close()
