"""Clipping where its launches change: 2048 pieces, whose sums every block adds itself, and one
more, which a launch between brings to one; and lists so long (over 16384 x 8192 values) that the
pieces grow beyond 8192 values, with tensors that begin and end anywhere in them.

Bounds as in tests/test_clip_gpu.py: the squares are added in 64 bits, so the norm is the rounded
one; a value passes the factor's rounding, the product's and the output's."""

import math

import pytest

from tests.seq_util import HALF, U, torch_gpu

pytestmark = pytest.mark.gpu


def _check(torch, P, grads, max_norm, inplace):
    held = [g.clone() for g in grads]
    norm = math.sqrt(sum(float(p.double().square().sum()) for g in grads for p in g.split(1 << 24) if len(p)))
    out = None if inplace else [torch.full_like(g, 7) for g in grads]
    got = float(P.clip_gradients(grads, max_norm, eps=0.0, out=out))
    assert abs(got - norm) <= 2 * U * norm
    factor = min(1.0, max_norm / norm)
    for h, o in zip(held, grads if inplace else out):
        half = HALF["bf16" if h.dtype == torch.bfloat16 else "fp32"]
        for a, b in zip(h.split(1 << 24), o.split(1 << 24)):
            want = a.double() * factor
            assert ((b.double() - want).abs() <= (3 * U + half) * (1 + half) * want.abs()).all()
    if not inplace:
        assert all(torch.equal(g, h) for g, h in zip(grads, held))


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("pieces", [2047, 2048, 2049, 4097])
def test_number_of_pieces(pieces, inplace):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    print(f"[gpu] clip {pieces} pieces", flush=True)
    gen = torch.Generator("cuda").manual_seed(pieces)
    # many small tensors, one of three pieces and a value in the fourth
    grads = [torch.randn(5, device="cuda", generator=gen) for _ in range(pieces - 4)]
    grads.insert(3, torch.randn(3 * 8192 + 1, device="cuda", generator=gen).bfloat16())
    _check(torch, P, grads, 1.0, inplace)


@pytest.mark.parametrize("inplace", [False, True])
def test_long_pieces(inplace):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    sizes = [50000017, 8191, 60000003, 1, 30000001, 8193, 8551, 8552, 8553]
    total = sum(sizes)
    assert total > 16384 * 8192
    print(f"[gpu] clip {total} values", flush=True)
    gen = torch.Generator("cuda").manual_seed(1)
    grads = [torch.empty(n, device="cuda", dtype=torch.float32 if i % 3 == 1 else torch.bfloat16).normal_(generator=gen)
             for i, n in enumerate(sizes)]
    # a tensor that starts anywhere
    flat = torch.empty(7000003, device="cuda").normal_(generator=gen)
    grads.append(flat[1:7000000])
    first, last = float(flat[0]), flat[7000000:].clone()
    for max_norm in (100.0, 1e9):
        _check(torch, P, grads, max_norm, inplace)
    assert float(flat[0]) == first and torch.equal(flat[7000000:], last)
