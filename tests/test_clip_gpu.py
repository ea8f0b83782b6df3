"""GPU parity of the clipping by the global norm against the float64 oracle: lists
of one to many tensors of every size and address, both types, in place and beside.

Bounds: the squares are added in 64 bits, so the norm is the rounded one, two half steps
with the factor's; a value passes the factor's rounding, the product's and the output's.
"""

import math

import numpy as np
import pytest

from oracle import memory as M
from tests.seq_util import HALF, U, get, torch_gpu

pytestmark = pytest.mark.gpu


def _list(torch, sizes, seed, types=("fp32", "bf16"), scale=1.0):
    gen = torch.Generator("cuda").manual_seed(seed)
    r = np.random.default_rng(seed)
    out = []
    for n in sizes:
        t = torch.bfloat16 if types[r.integers(len(types))] == "bf16" else torch.float32
        out.append((torch.randn(n, generator=gen, device="cuda") * (scale * math.exp(r.normal()))).to(t))
    return out


def _check(torch, P, grads, max_norm, eps=1e-6, inplace=False):
    norm, want = M.clip([get(g) for g in grads], max_norm, eps)
    held = [g.clone() for g in grads]
    out = None if inplace else [torch.full_like(g, 7) for g in grads]
    got = P.clip_gradients(grads, max_norm, eps=eps, out=out)
    assert got.dtype == torch.float32 and got.shape == () and abs(float(got) - norm) <= 2 * U * norm
    for g, h, o, w in zip(grads, held, grads if inplace else out, want):
        half = HALF["bf16" if g.dtype == torch.bfloat16 else "fp32"]
        assert (np.abs(get(o) - w) <= (3 * U + half) * np.abs(w) * (1 + half) + 1e-40).all()
        assert inplace or torch.equal(g, h)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [5, 8191, 8192, 8193, 16384 + 7], [1] * 300, [3, 100003, 17, 2000001],
                                   [1023, 1024, 1025] * 60, [40000] * 113], ids=lambda s: f"{len(s)}x{max(s)}")
def test_lists(sizes, inplace):
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    print(f"[gpu] clip {len(sizes)} tensors {inplace}", flush=True)
    for max_norm in (0.25, 1e9):
        _check(torch, P, _list(torch, sizes, len(sizes)), max_norm, inplace=inplace)


def test_more_sums_than_a_block_adds():
    """Over 4096 pieces: their sum is a launch of its own."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    _check(torch, P, _list(torch, [7] * 5000, 3), 1.0)


def test_addresses():
    """Tensors that start anywhere in a buffer, neighbours that are not touched."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.randn(70000, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(dtype)
        cuts = [(1, 8000), (8001, 8002), (8003, 30000), (30001, 69999)]
        whole = flat.clone()
        parts = [flat[a:b] for a, b in cuts]
        _, want = M.clip([get(p) for p in parts], 1.0, 1e-6)
        P.clip_gradients(parts, 1.0)
        half = HALF["bf16" if dtype == torch.bfloat16 else "fp32"]
        for (a, b), w in zip(cuts, want):
            assert (np.abs(get(flat[a:b]) - w) <= (3 * U + 2 * half) * np.abs(w)).all()
        for i in (0, 8000, 8002, 30000, 69999):
            assert flat[i] == whole[i]


def test_extremes():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    # squares beyond the range of fp32 either way
    for scale in (1e30, 1e-30):
        _check(torch, P, _list(torch, [1000, 77], 9, ("fp32",), scale), scale, eps=0.0)
    zero = [torch.zeros(100, device="cuda")]
    assert float(P.clip_gradients(zero, 1.0)) == 0 and (zero[0] == 0).all()
    assert float(P.clip_gradients([], 1.0)) == 0
    assert float(P.clip_gradients([torch.empty(0, device="cuda")], 1.0)) == 0
    g = _list(torch, [50, 60], 10)
    held = [x.clone() for x in g]
    assert float(P.clip_gradients(g, math.inf)) > 0 and all(torch.equal(a, b) for a, b in zip(g, held))
    P.clip_gradients(g, 0.0)
    assert all((x == 0).all() for x in g)
    g = [torch.ones(10, device="cuda"), torch.ones(10, device="cuda")]
    g[1][3] = math.inf
    out = [torch.empty_like(x) for x in g]
    assert math.isinf(float(P.clip_gradients(g, 1.0, out=out)))
    assert (out[0] == 0).all() and torch.isnan(out[1][3]) and int(torch.isnan(out[1]).sum()) == 1
    g[1][3] = math.nan
    assert math.isnan(float(P.clip_gradients(g, 1.0, out=out))) and all(torch.isnan(x).all() for x in out)


def test_no_limit_and_nothing_to_scale():
    """Without a limit the values stay, whatever their norm; zeros stay without eps too."""
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    for odd in (math.inf, math.nan):
        g = [torch.ones(10, device="cuda"), torch.ones(10, device="cuda", dtype=torch.bfloat16)]
        g[0][3] = odd
        held, out = [x.clone() for x in g], [torch.zeros_like(x) for x in g]
        for to in (None, out):
            norm = float(P.clip_gradients(g, math.inf, out=to))
            assert norm == odd or math.isnan(norm) and math.isnan(odd)
            assert all(torch.equal(a.nan_to_num(7.0, 8.0), b.nan_to_num(7.0, 8.0)) for a, b in zip(to or g, held))
    zero = [torch.zeros(100, device="cuda")]
    assert float(P.clip_gradients(zero, 0.0, eps=0.0)) == 0 and (zero[0] == 0).all()


def test_same_result_every_time_and_in_a_graph():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    a, b = _list(torch, [100003, 5, 70001], 11), _list(torch, [100003, 5, 70001], 11)
    for x in b:
        x.mul_(2)
    out, other = [torch.empty_like(x) for x in a], [torch.empty_like(x) for x in a]
    want = P.clip_gradients(a, 1.0, out=out)
    assert torch.equal(want, P.clip_gradients(a, 1.0, out=other)) and all(torch.equal(x, y) for x, y in zip(out, other))
    static = [x.clone() for x in a]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.clip_gradients(static, 1.0, out=other)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = P.clip_gradients(static, 1.0, out=other)
    for src in (a, b, a):
        for s, x in zip(static, src):
            s.copy_(x)
        graph.replay()
        got, eager = norm.clone(), P.clip_gradients(src, 1.0, out=out)
        torch.cuda.synchronize()
        assert torch.equal(got, eager) and all(torch.equal(x, y) for x, y in zip(out, other))


def test_refusals():
    torch = torch_gpu()
    import paper_2509_24093_amd as P
    a = torch.ones(100, device="cuda")
    for bad in (a.cpu(), a.half(), a[::2], None, 3):
        with pytest.raises(ValueError, match=r"grads\[1\]"):
            P.clip_gradients([a, bad], 1.0)
    for bad in ([a], [a, a[:50]], [a.clone(), torch.ones(100, device="cuda", dtype=torch.bfloat16)]):
        with pytest.raises(ValueError, match="out"):
            P.clip_gradients([a, a.clone()], 1.0, out=bad)
    for call in (lambda: P.clip_gradients([a, a], 1.0), lambda: P.clip_gradients([a[:60], a[50:]], 1.0),
                 lambda: P.clip_gradients([a[:50]], 1.0, out=[a[1:51]]),
                 lambda: P.clip_gradients([a, a], 1.0, out=[a.clone(), a])):
        with pytest.raises(P.CgconvError, match="overlap"):
            call()
    for bad in (-1.0, math.nan):
        with pytest.raises(P.CgconvError, match="max_norm"):
            P.clip_gradients([a], bad)
    assert (a == 1).all()
    # one tensor read twice, into places of its own
    out = [torch.empty_like(a), torch.empty_like(a)]
    assert abs(float(P.clip_gradients([a, a], 1.0, out=out)) - 200 ** 0.5) < 1e-5 and torch.equal(out[0], out[1])
