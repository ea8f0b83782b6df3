"""Incoming gradients that are contiguous but start off a 16-byte boundary, as a
part of a concatenation sends them at one sequence, through the convolution's
autograd functions: the same gradients as from one at its own address."""

import pytest

from tests.seq_util import torch_gpu

pytestmark = pytest.mark.gpu

N, C = 8, 5


@pytest.mark.parametrize("checkpoint", [None, "int8"])
@pytest.mark.parametrize("name", ["cgconv", "cgconv_gate", "cgconv_graph"])
def test_gradient_that_starts_off_a_vector(name, checkpoint):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    gen = torch.Generator(device="cuda").manual_seed(6)
    f = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").requires_grad_()  # noqa: E731
    q, k, head = f(1, N, 1, C), f(1, N, 1, C), f(1, 1, 1, C)
    if name == "cgconv_graph":
        plan = P.GraphPlan(1, N, 0, C)
        U = torch.linalg.qr(torch.randn(1, N, N, generator=gen, device="cuda"))[0].contiguous()
        op = lambda: P.cgconv_graph(U, q, k, plan, checkpoint=checkpoint)  # noqa: E731
    else:
        plan = P.Plan(1, N, 0, C)
        op = lambda: getattr(P, name)(q, k, plan, checkpoint=checkpoint)  # noqa: E731
    g = torch.randn(1, N + 1, 1, C, generator=gen, device="cuda")
    part = g[:, 1:]
    assert part.is_contiguous() and part.data_ptr() % 16
    want = torch.autograd.grad(op(), (q, k), part.clone())
    for got in (torch.autograd.grad(torch.cat((head, op()), 1), (q, k), g), torch.autograd.grad(op(), (q, k), part)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    plan.close()
