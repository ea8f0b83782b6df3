"""The sequence operators beyond 2^31 elements of one array (bf16, 2^20 + 3 tokens
of 2048 channels): the last tokens, whose offsets pass 32 bits, equal those of a
short call on a copy of them."""

import pytest

from tests.seq_util import torch_gpu

pytestmark = pytest.mark.gpu

N, C, LAST = (1 << 20) + 3, 2048, 24


@pytest.fixture(scope="module")
def arrays():
    torch = torch_gpu()
    gen = torch.Generator("cuda").manual_seed(1)
    x = torch.empty(1, N, 1, C, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    g = torch.empty_like(x).normal_(generator=gen)
    assert x.numel() > 2 ** 31
    yield torch, x, g, gen
    del x, g
    torch.cuda.empty_cache()


def _tail(t):
    return t[:, -LAST:].clone()


def test_norm_and_pack(arrays):
    torch, x, g, gen = arrays
    import paper_2509_24093_amd as P
    w = 1 + 0.1 * torch.randn(1, C, device="cuda", generator=gen)
    plan, small = P.SequencePlan(1, N, 0, C), P.SequencePlan(1, LAST, 0, C)
    y, mean, rstd, codes, scales = plan.norm(x, w, None, checkpoint=True)
    sy, smean, srstd, scodes, sscales = small.norm(_tail(x), w, None, checkpoint=True)
    for a, b in ((y, sy), (mean, smean), (rstd, srstd), (codes, scodes), (scales, sscales)):
        assert torch.equal(a[:, -LAST:], b)
    del y
    gx, _, _ = plan.norm_backward((codes, scales), w, mean, rstd, g, need_weight=False, need_bias=False)
    assert torch.equal(gx[:, -LAST:], small.norm_backward((scodes, sscales), w, smean, srstd, _tail(g))[0])
    del gx
    again, ascales = P.checkpoint_pack(x)
    assert torch.equal(again[:, -LAST:], scodes) and torch.equal(ascales[:, -LAST:], sscales)
    back = P.checkpoint_unpack(again, ascales, dtype=torch.bfloat16)
    assert torch.equal(back[:, -LAST:], P.checkpoint_unpack(scodes, sscales, dtype=torch.bfloat16))
    plan.close()
    small.close()


def test_short_convolution(arrays):
    torch, x, g, gen = arrays
    import paper_2509_24093_amd as P
    W = 4
    w, b = torch.randn(W, 1, C, device="cuda", generator=gen), torch.randn(C, device="cuda", generator=gen)
    plan, small = P.SequencePlan(1, N, 0, C), P.SequencePlan(1, LAST, 0, C)
    y, state = plan.conv(x, w, b)
    before = x[:, -LAST - W + 1:-LAST].clone()
    sy, sstate = small.conv(_tail(x), w, b, state=before)
    assert torch.equal(y[:, -LAST:], sy) and torch.equal(state, sstate)
    del y
    gx, _, _ = plan.conv_backward(x, w, b, g, need_weight=False, need_bias=False)
    sgx, _, _ = small.conv_backward(_tail(x), w, b, _tail(g), need_weight=False, need_bias=False)
    assert torch.equal(gx[:, -LAST + W:], sgx[:, W:])  # (the first tokens of the copy see other inputs)
    plan.close()
    small.close()


def test_scan(arrays):
    """Decays of exp(-100) per token: a token sees itself and nothing else that
    counts (exp(-100) of the largest values is below 2^-100), so the copy agrees up
    to fp32 rounding: one bf16 step at most."""
    torch, x, g, gen = arrays
    import paper_2509_24093_amd as P
    S = 4
    delta = torch.full((1, N, C), 1.0, device="cuda", dtype=torch.bfloat16)
    A = torch.full((C, S), -100 / 1.3132616, device="cuda")
    Bt, Ct = (torch.empty(1, N, S, device="cuda", dtype=torch.bfloat16).normal_(generator=gen) for _ in range(2))
    D = torch.randn(C, device="cuda", generator=gen)
    plan, small = P.SequencePlan(1, N, 0, C, states=S), P.SequencePlan(1, LAST, 0, C, states=S)
    cut = [_tail(t) for t in (x, delta)] + [A] + [_tail(t) for t in (Bt, Ct)] + [D]
    y, state = plan.scan(x, delta, A, Bt, Ct, D)
    sy, sstate = small.scan(*cut)

    def close(a, b, steps=1):
        a, b = a.float(), b.float()
        assert float(((a - b).abs() - steps * 2.0 ** -7 * b.abs()).max()) <= 1e-30

    close(y[:, -LAST + 1:], sy[:, 1:])
    assert torch.allclose(state, sstate, rtol=1e-6, atol=1e-30)
    del y
    need = (True, True, False, False, False, False, False)
    gx, gd = plan.scan_backward(x, delta, A, Bt, Ct, D, g, need=need)[:2]
    sgx, sgd = small.scan_backward(*cut, _tail(g), need=need)[:2]
    close(gx[:, -LAST + 1:], sgx[:, 1:])
    close(gd[:, -LAST + 1:], sgd[:, 1:])
    plan.close()
    small.close()
