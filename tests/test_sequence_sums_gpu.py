"""Sums over many tokens of the sequence operators: sizes at which every block
goes through its loops more than once, the last sums read more than one block
each, and the highest degrees.

The references are the float64 oracle's, and for the convolution's large sizes the
same formulas in float64 torch.  Bounds: those of the operators' own tests, whose
counts of roundings hold here too, as stated at each test.
"""

import pytest

import tests.test_conv_gpu as conv_tests
import tests.test_norm_gpu as norm_tests
import tests.test_scan_gpu as scan_tests
from oracle import sequence as S
from tests.seq_util import HALF, U, put, tdtype, torch_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype", [((1, 4500, 0, 1024), "bf16"), ((1, 4500, 0, 1030), "bf16"),
                                         ((1, 600, 0, 16384), "bf16"), ((1, 600, 0, 16383), "fp32"),
                                         ((2, 1100, 1, 520), "bf16")], ids=str)
def test_norm_gradients_of_many_tokens(shape, dtype):
    """The wide form with several tokens a block: loaded a token ahead (bf16, up to
    256 threads), with a row's last vector in part, with blocks of 1024 threads; x
    whole and as its checkpoint.  gw and gb: at most 3 tokens in a thread, 2048
    blocks in 16 slices of 128 and 16 more, or 1024 blocks of three components: 211
    of the 512 roundings allowed."""
    norm_tests.test_norm_and_gradients(shape, dtype)


def _conv_backward(torch, x, w, b, g, L, there):
    """(gx, gw, gb) in float64 (a mask of the tokens that are there)."""
    deg = torch.tensor([l for l in range(L + 1) for _ in range(2 * l + 1)], device=x.device)
    x, gz, wk = x.double() * there, g.double() * there, w.double()[:, deg]
    N, W = x.shape[1], len(w)

    def earlier(v, j):
        return v if j == 0 else torch.cat([torch.zeros_like(v[:, :j]), v[:, :-j]], 1)

    def later(v, j):
        return v if j == 0 else torch.cat([v[:, j:], torch.zeros_like(v[:, :j])], 1)

    if b is not None:
        z = sum(w.double()[j, 0] * earlier(x[:, :, 0], j) for j in range(W)) + b.double()
        s = torch.sigmoid(z)
        gz[:, :, 0] *= s * (1 + z * (1 - s))
    gx = sum(wk[j] * later(gz, j) for j in range(W)) * there
    gw = torch.zeros(W, L + 1, x.shape[-1], dtype=torch.float64, device=x.device)
    for j in range(W):
        per = (gz * earlier(x, j)).sum((0, 1))
        for l in range(L + 1):
            gw[j, l] = per[l * l:(l + 1) ** 2].sum(0)
    return gx, gw, gz[:, :, 0].sum((0, 1))


# (B, N, L, C, W), tokens per chunk, blocks whose sums are added: at least 2^18
# columns of chunks are in flight (csrc/conv.hip), so these take chunks of every length
@pytest.mark.parametrize("shape,dtype", [((1, 16400, 0, 1024, 4), "bf16"),  # 64, 65
                                         ((2, 4100, 0, 1026, 6), "bf16"),  # 32, 65
                                         ((2, 4100, 2, 60, 4), "fp32"),  # 16, 129
                                         ((2, 4100, 1, 66, 7), "fp32"),  # 8, 257
                                         ((3, 4099, 6, 33, 5), "fp32")], ids=str)  # 64, 49
@pytest.mark.parametrize("ragged", [False, True])
def test_convolution_gradients_of_many_tokens(shape, dtype, ragged):
    """gw and gb: at most 64 tokens in a thread, 4 chunks in a block, then 64 slices
    of at most 5 blocks (13 components of the highest degree each) and 6 steps
    between them: 64 + 4 + 65 + 6 roundings, of 512 allowed; the factors as in the
    convolution's own test."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, W = shape
    print(f"[gpu] conv sums {shape} {dtype} {ragged}", flush=True)
    K = (L + 1) ** 2
    gen = torch.Generator(device="cuda").manual_seed(11)
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, g = f(B, N, K, C).to(tdtype(dtype)), f(B, N, K, C).to(tdtype(dtype))
    w, b = f(W, L + 1, C) / W ** 0.5, f(C)
    lengths = torch.tensor([N - 37 * i for i in range(B)], dtype=torch.int32, device="cuda") - 5 if ragged else None
    there = torch.ones(B, N, 1, 1, dtype=torch.float64, device="cuda")
    if ragged:
        there = (torch.arange(N, device="cuda")[None] < lengths[:, None]).double()[:, :, None, None]
    plan = P.SequencePlan(B, N, L, C)
    got = plan.conv_backward(x, w, b, g, lengths)
    ref = _conv_backward(torch, x, w, b, g, L, there)
    # magnitudes: of z, and of the gradients under a factor of at most 1.1 with 32 (1 + |z|) half steps
    xa, wa, ga = x.abs(), w.abs(), g.double().abs()
    m = sum(wa.double()[j, 0] * torch.cat([xa[:, :, 0].double().new_zeros(B, j, C), xa[:, :N - j, 0].double()], 1)
            for j in range(W)) + b.double().abs()
    ga[:, :, 0] *= 1 + m
    for name, a, r, mag, n, kind in zip(("gx", "gw", "gb"), got, ref, _conv_backward(torch, xa, wa, None, ga, L, there),
                                        (64, 512, 512), (dtype, "fp32", "fp32")):
        bound = n * U * 1.1 * mag
        bound = bound + HALF[kind] * (r.abs() + bound) + 1e-37
        worst = float(((a.double() - r).abs() / bound).max())
        assert worst <= 1, f"{name}: {worst:.3g} of the bound"
    again = plan.conv_backward(x, w, b, g, lengths)
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    plan.close()


def test_convolution_reference():
    """The float64 torch form above is the oracle's."""
    torch = torch_gpu()
    (x, xv), (w, wv), (b, bv), (g, gv), _, lengths = conv_tests._inputs((3, 19, 2, 5, 6), "fp32", 2, True)
    there = torch.from_numpy(S._there(3, 19, lengths)).cuda()
    for a, r in zip(_conv_backward(torch, x, w, b, g, 2, there), S.conv_backward(xv, wv, bv, gv, 2, lengths)):
        assert torch.allclose(a.cpu(), torch.from_numpy(r), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 19, 8, 3, 4), (2, 9, 7, 6, 2)], ids=str)
def test_convolution_of_the_highest_degrees(shape, dtype):
    conv_tests.test_forward_and_gradients(shape, True, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 18, 8, 5, 16), (2, 9, 7, 6, 8)], ids=str)
def test_scan_of_the_highest_degrees(shape, dtype):
    scan_tests.test_forward_and_gradients(shape, True, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("states", [1, 4, 5, 7, 8, 12, 18, 20, 24, 31])
@pytest.mark.parametrize("sizes", [(7, 0, 37), (3, 1, 50), (5, 0, 260), (2, 2, 17)], ids=str)
def test_steps_of_every_state_count(sizes, states, dtype):
    """Lane groups of four states: one to eight of them, whole groups and parts of one
    idle; one, two and four channels a thread; a last block in part."""
    B, L, C = sizes
    scan_tests.test_steps((B, 3, L, C, states), dtype)


def test_entry_points_of_the_c_interface():
    """The functions named as the C ABI's give what the plan's methods give."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    B, N, L, C, St, W = 2, 20, 1, 12, 8, 4
    t, (g, _), (h0, _), _ = scan_tests._inputs((B, N, L, C, St), "fp32", 3, False)
    d = {k: v[0] for k, v in t.items()}
    w, b, cw = (put(a)[0] for a in ([[1.5] * C, [0.5] * C], [0.25] * C, [[[0.5] * C] * (L + 1)] * W))
    plan = P.SequencePlan(B, N, L, C, states=St)
    h, stream = plan._h, torch.cuda.current_stream().cuda_stream
    p = lambda v: None if v is None else v.data_ptr()  # noqa: E731
    like = lambda ts: [None if v is None else torch.full_like(v, 7) for v in ts]  # noqa: E731
    assert P.cgconv_seq_plan_info(h) == plan.info() > 0

    def same(name, want, call):
        got = like(want)
        call(got, [p(v) for v in got])
        assert all(torch.equal(a, c) for a, c in zip(got, want)), name

    x = d["x"]
    norm = plan.norm(x, w, b, 1e-5, checkpoint=True)
    same("norm", norm, lambda _, o: P.cgconv_seq_norm(h, P.CGCONV_F32, p(x), p(w), p(b), 1e-5, *o, stream))
    y, mean, rstd, codes, scales = norm
    same("norm_backward", plan.norm_backward(x, w, mean, rstd, g),
         lambda _, o: P.cgconv_seq_norm_backward(h, P.CGCONV_F32, p(x), None, None, p(w), p(mean), p(rstd), p(g), *o,
                                                 stream))
    same("conv", plan.conv(x, cw, b),
         lambda _, o: P.cgconv_seq_conv(h, P.CGCONV_F32, W, p(x), p(cw), p(b), 1, None, None, *o, stream))
    same("conv_backward", plan.conv_backward(x, cw, b, g),
         lambda _, o: P.cgconv_seq_conv_backward(h, P.CGCONV_F32, W, p(x), p(cw), p(b), 1, None, p(g), *o, stream))
    args = [p(d[k]) for k in ("x", "delta", "A", "Bt", "Ct", "D", "bias")]
    same("scan", plan.scan(*(d[k] for k in scan_tests.ORDER)),
         lambda _, o: P.cgconv_seq_scan(h, P.CGCONV_F32, *args, None, None, *o, stream))
    same("scan_backward", plan.scan_backward(*(d[k] for k in scan_tests.ORDER[:-1]), g, d["bias"]),
         lambda _, o: P.cgconv_seq_scan_backward(h, P.CGCONV_F32, *args, None, p(g), *o, stream))
    xt, dt, bt, ct = (d[k][:, 0].clone(memory_format=torch.contiguous_format) for k in ("x", "delta", "Bt", "Ct"))
    cs, ss = torch.randn(B, W - 1, (L + 1) ** 2, C, device="cuda"), h0.clone()

    def step(f, state):
        state = state.clone()
        return f(state), state

    def conv_step(got, o):
        got[1].copy_(cs)
        P.cgconv_seq_conv_step(h, P.CGCONV_F32, W, p(xt), p(cw), p(b), 1, o[1], o[0], stream)

    def scan_step(got, o):
        got[1].copy_(ss)
        P.cgconv_seq_scan_step(h, P.CGCONV_F32, p(xt), p(dt), p(d["A"]), p(bt), p(ct), p(d["D"]), p(d["bias"]), o[1], o[0],
                               stream)

    same("conv_step", step(lambda s: plan.conv_step(xt, cw, b, s), cs), conv_step)
    same("scan_step", step(lambda s: plan.scan_step(xt, dt, d["A"], bt, ct, d["D"], s, d["bias"]), ss), scan_step)
    torch.cuda.synchronize()
    raw = P.cgconv_seq_plan_create(B, N, L, C)
    assert 0 < P.cgconv_seq_plan_info(raw) <= plan.info()
    P.cgconv_seq_plan_destroy(raw)
    plan.close()
