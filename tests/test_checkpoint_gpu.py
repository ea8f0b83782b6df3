"""GPU parity of the 8-bit checkpoints (exact: codes and scales equal the
oracle's) and of the autograd functions that keep their inputs in 8 bits."""

import numpy as np
import pytest

import workloads as W
from oracle import sequence as S
from tests.conftest import rel_l2
from tests.seq_util import get, put, torch_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1,), (5, 1), (3, 31), (2, 4, 32), (7, 33), (3, 5, 20), (2, 66), (4, 100), (1, 4096),
                                   (1000, 24)], ids=str)
def test_codes_are_exact(shape, dtype):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    print(f"[gpu] pack {shape} {dtype}", flush=True)
    r = np.random.default_rng(sum(shape))
    # magnitudes over the whole exponent range, values on ties, zeros
    x = r.normal(size=shape) * np.exp2(r.integers(-140, 120, size=shape[:-1] + (1,)))
    x = np.where(r.random(shape) < 0.1, 0, x)
    x = np.where(r.random(shape) < 0.2, np.round(x * 2) / 2, x)
    t, v = put(x, dtype)
    codes, scales = P.checkpoint_pack(t)
    rc, rs = S.pack(v)
    assert (codes.cpu().numpy() == rc).all() and (scales.cpu().numpy() == rs).all()
    back = P.checkpoint_unpack(codes, scales, dtype=t.dtype)
    assert back.dtype == t.dtype and (get(back) == S.unpack(rc, rs)).all()  # no rounding, in bf16 either


def test_not_finite_groups():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    x = torch.ones(3, 70, device="cuda")
    x[0, 40], x[1, 69], x[2, 0] = float("inf"), float("nan"), float("-inf")
    back = P.checkpoint_unpack(*P.checkpoint_pack(x))
    lost = torch.zeros(3, 70, dtype=torch.bool, device="cuda")
    lost[0, 32:64] = lost[1, 64:] = lost[2, :32] = True
    assert torch.isnan(back[lost]).all() and (back[~lost] == 1).all()


def test_empty_and_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    codes, scales = P.checkpoint_pack(torch.zeros(0, 8, device="cuda"))
    assert P.checkpoint_unpack(codes, scales).shape == (0, 8)
    with pytest.raises(ValueError):
        P.checkpoint_pack(torch.zeros(4, 8))
    with pytest.raises(ValueError):
        P.checkpoint_pack(torch.zeros(4, 8, device="cuda").T)
    with pytest.raises(ValueError):
        P.checkpoint_pack(torch.zeros(4, 8, device="cuda", dtype=torch.float16))
    codes, scales = P.checkpoint_pack(torch.ones(4, 40, device="cuda"))
    with pytest.raises(ValueError, match="scales"):
        P.checkpoint_unpack(codes, scales[:, :1])
    with pytest.raises(ValueError, match="codes"):
        P.checkpoint_unpack(codes.float(), scales)


def _held(t):
    return S.unpack(*S.pack(t.detach().cpu().numpy()))


def test_convolution_and_gate_keep_their_inputs_in_8_bits():
    """The gradients are those of the backward at the values the 8 bits hold,
    bit for bit, and close to the whole inputs' gradients: a value moves by at
    most 1/127 of its group's largest, 0.5% of the norm for normal inputs, and
    each gradient is linear in the other operand (the convolution)."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C = 2, 64, 2, 40
    q, k = (torch.from_numpy(a).cuda().requires_grad_(True) for a in W.iid(B, N, L, C, seed=3))
    g = torch.from_numpy(np.random.default_rng(4).normal(size=q.shape).astype(np.float32)).cuda()
    plan = P.Plan(B, N, L, C)
    hq, hk = (torch.from_numpy(_held(t).astype(np.float32)).cuda() for t in (q, k))
    for f, backward in ((P.cgconv, plan.backward), (P.cgconv_gate, plan.gate_value_backward)):
        whole = f(q, k, plan)
        out = f(q, k, plan, checkpoint="int8")
        assert torch.equal(whole, out)
        got = torch.autograd.grad(out, (q, k), g)
        want = backward(hq, hk, g)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        if f is P.cgconv:
            ref = torch.autograd.grad(whole, (q, k), g)
            for a, c in zip(got, ref):
                assert rel_l2(get(a), get(c)) <= 0.02
    # one gradient only, none
    only, = torch.autograd.grad(P.cgconv(q, k.detach(), plan, checkpoint="int8"), (q,), g)
    assert torch.equal(only, plan.backward(hq, hk, g)[0])
    with torch.no_grad():
        assert torch.equal(P.cgconv(q, k, plan, checkpoint="int8"), plan(q, k))
    with pytest.raises(ValueError, match="checkpoint"):
        P.cgconv(q, k, plan, checkpoint="fp8")
    plan.close()


def test_graph_convolution_keeps_its_inputs_in_8_bits():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C = 2, 30, 1, 8
    r = np.random.default_rng(9)
    U = torch.from_numpy(np.stack([np.linalg.qr(r.normal(size=(N, N)))[0] for _ in range(B)]).astype(np.float32)).cuda()
    q, k = (torch.from_numpy(a).cuda().requires_grad_(True) for a in W.iid(B, N, L, C, seed=5))
    g = torch.randn(q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    plan = P.GraphPlan(B, N, L, C)
    got = torch.autograd.grad(P.cgconv_graph(U, q, k, plan, checkpoint="int8"), (q, k), g)
    hq, hk = (torch.from_numpy(_held(t).astype(np.float32)).cuda() for t in (q, k))
    want = plan.backward(U, hq, hk, g)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    plan.close()


def test_memory_of_a_kept_input():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C = 2, 1024, 4, 32
    plan = P.Plan(B, N, L, C)
    q, k = (torch.randn(B, N, (L + 1) ** 2, C, device="cuda").requires_grad_(True) for _ in range(2))

    def held(checkpoint):
        a, b = q * 1.0, k * 1.0  # activations: nobody else keeps them
        torch.cuda.synchronize()
        out = P.cgconv(a, b, plan, checkpoint=checkpoint)
        del a, b
        n = torch.cuda.memory_allocated()
        del out
        return n - torch.cuda.memory_allocated()

    whole, packed = held(None), held("int8")
    n = q.numel()
    # out, and q and k; torch's allocator leaves up to 1 MiB unsplit in a block above
    # 1 MiB (out and both codes) and counts it as allocated
    assert whole >= 3 * 4 * n and packed <= 4 * n + 2 * (n + n // 32) + 3 * 2 ** 20
    plan.close()
