"""The delta rule, the norms around a residual connection and the clipping where offsets pass
32 bits: more than 2^31 elements of one array, and the widest rows of keys."""

import math

import pytest

from tests.seq_util import HALF, U, torch_gpu

pytestmark = pytest.mark.gpu

LAST = 24


def _normal(torch, gen, *shape, dtype=None):
    return torch.empty(*shape, device="cuda", dtype=dtype or torch.bfloat16).normal_(generator=gen)


# long rows of scalars; short rows, many tokens; long rows of vectors
@pytest.mark.parametrize("L, C, N", [(0, 2048, (1 << 20) + 3), (0, 32, (1 << 26) + 5), (1, 520, (1 << 20) + 3)],
                         ids=["wide", "rows", "channels"])
def test_residual_norm(L, C, N):
    """The last tokens of a long call are those of a short one on a copy of them, bit by bit."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    K = (L + 1) ** 2
    assert N * K * C > 2 ** 31
    print(f"[gpu] residual beyond 2^31: L={L} C={C}", flush=True)
    gen = torch.Generator("cuda").manual_seed(1)
    x, u, gate = (_normal(torch, gen, 1, N, k, C) for k in (K, K, 1))
    gate = gate[:, :, 0]
    par = [1 + 0.1 * torch.randn(L + 1, C, device="cuda", generator=gen), torch.rand(C, device="cuda", generator=gen),
           1 + 0.1 * torch.randn(L + 1, C, device="cuda", generator=gen)]
    bias = torch.randn(C, device="cuda", generator=gen)
    tail = lambda t: t[:, -LAST:].clone()  # noqa: E731
    plan, small = P.SequencePlan(1, N, L, C), P.SequencePlan(1, LAST, L, C)
    r, y, stats = plan.residual_norm(x, u, gate, *par, bias)
    sr, sy, sstats = small.residual_norm(tail(x), tail(u), tail(gate), *par, bias)
    for a, b in ((r, sr), (y, sy), (stats, sstats)):
        assert torch.equal(a[:, -LAST:], b)
    # the outputs' places serve as the incoming gradients
    need = (True, True, True) + (False,) * 4
    g = plan.residual_norm_backward(x, u, gate, *par, stats, r, y, need=need)
    sg = small.residual_norm_backward(tail(x), tail(u), tail(gate), *par, sstats, sr, sy, need=need)
    for a, b in zip(g[:3], sg[:3]):
        assert torch.equal(a[:, -LAST:], b)
    plan.close()
    small.close()


def test_delta_rule():
    """Every token forgets the state, exp(-1000) of it being zero, and sees itself alone:
    y = scale beta (qn.kn) v, gv = scale beta (qn.kn) gy, the last state kn beta v; one product
    of D terms, a few factors and the rounding to bf16."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    N, C, H, D = (1 << 20) + 3, 2048, 16, 8
    print("[gpu] delta rule beyond 2^31", flush=True)
    gen = torch.Generator("cuda").manual_seed(2)
    v, gy = _normal(torch, gen, 1, N, 1, C), _normal(torch, gen, 1, N, 1, C)
    assert v.numel() > 2 ** 31
    q, k = _normal(torch, gen, 1, N, H, D), _normal(torch, gen, 1, N, H, D)
    beta = torch.rand(1, N, H, device="cuda", generator=gen)
    decay = torch.full_like(beta, -1000.0)
    unit = lambda t: t.double() / (t.double().square().sum(-1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
    factor = lambda at: (D ** -0.5 * beta[:, at].double() *  # noqa: E731
                         (unit(q[:, at]) * unit(k[:, at])).sum(-1))[..., None]
    places = [slice(0, LAST), slice(N // 2, N // 2 + 70), slice(N - 70, N)]
    rows = lambda t, at: t[:, at].double().reshape(1, -1, H, C // H)  # noqa: E731

    def near(name, got, want, size):
        assert ((got - want).abs() <= (HALF["bf16"] + 4 * (D + 232) * U) * size + 1e-30).all(), name

    plan = P.SequencePlan(1, N, 0, C, heads=H, key_dim=D)
    y, state = plan.delta_rule(q, k, v, decay, beta)
    for at in places:
        size = (D ** -0.5 * beta[:, at].double())[..., None] * rows(v, at).abs()  # of terms that may cancel in qn.kn
        near(("y", at), rows(y, at), factor(at) * rows(v, at), size)
    want = unit(k[:, -1])[0, :, :, None] * (beta[0, -1].double()[:, None] * rows(v, slice(N - 1, N))[0, 0])[:, None]
    near("state", state[0, :, 0].double().reshape(D, H, -1).transpose(0, 1), want, want.abs())
    del y
    gv = plan.delta_rule_backward(q, k, v, decay, beta, gy, need=(False, False, True, False, False, False))[2]
    for at in places:
        size = (D ** -0.5 * beta[:, at].double())[..., None] * rows(gy, at).abs()
        near(("gv", at), rows(gv, at), factor(at) * rows(gy, at), size)
    del gv
    # the gradients of beta, sums over a head's columns: scale (qn.kn) gy.v
    gb = plan.delta_rule_backward(q, k, v, decay, beta, gy, need=(False, False, False, False, True, False))[4]
    for at in places:
        f = factor(at)[..., 0] / beta[:, at].double()
        terms = rows(gy, at) * rows(v, at)
        want, size = f * terms.sum(-1), D ** -0.5 * terms.abs().sum(-1)
        assert ((gb[:, at].double() - want).abs() <= 4 * (D + 232 + C // H) * U * size).all(), at
    plan.close()


def test_the_widest_rows_of_keys():
    """16384 key heads of 128 in fp32, 8 MiB a token and 2^29 bytes a chunk: the last heads are
    those of a call of their own, bit by bit."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    N, H, D, few = 130, 16384, 128, 4
    print("[gpu] delta rule, widest keys", flush=True)
    gen = torch.Generator("cuda").manual_seed(3)
    q, k = (_normal(torch, gen, 1, N, H, D, dtype=torch.float32) for _ in range(2))
    v, gy = (_normal(torch, gen, 1, N, 1, H, dtype=torch.float32) for _ in range(2))
    decay, beta = -torch.rand(1, N, H, device="cuda", generator=gen), torch.rand(1, N, H, device="cuda", generator=gen)
    plan, small = P.SequencePlan(1, N, 0, H, heads=H, key_dim=D), P.SequencePlan(1, N, 0, few, heads=few, key_dim=D)
    part = [t[..., -few:, :].clone() for t in (q, k)] + [t[..., -few:].clone() for t in (v, decay, beta)]
    y, state = plan.delta_rule(q, k, v, decay, beta)
    sy, sstate = small.delta_rule(*part)
    assert torch.equal(y[..., -few:], sy) and torch.equal(state[..., -few:], sstate)
    g = plan.delta_rule_backward(q, k, v, decay, beta, gy)
    sg = small.delta_rule_backward(*part, gy[..., -few:].clone())
    for i, (a, b) in enumerate(zip(g[:5], sg)):
        assert torch.equal(a[..., -few:, :] if i < 2 else a[..., -few:], b), i
    plan.close()
    small.close()


def test_clipping_of_one_tensor():
    """2^31 + 9 ones: the norm is the root of their number, every one is scaled."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    n = 2 ** 31 + 9
    print("[gpu] clip beyond 2^31", flush=True)
    g = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    out = torch.zeros_like(g)
    norm = float(P.clip_gradients([g], 2.0 ** 10, eps=0.0, out=[out]))
    assert abs(norm - math.sqrt(n)) <= 2 * U * norm
    want = torch.tensor(2.0 ** 10 / math.sqrt(n), dtype=torch.float64).to(torch.bfloat16).item()
    for part in out.split(1 << 28):
        assert float(part.min()) == want and float(part.max()) == want
    P.clip_gradients([g], 2.0 ** 10, eps=0.0)
    assert torch.equal(g, out)
