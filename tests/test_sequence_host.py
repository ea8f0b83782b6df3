"""Refusals of the sequence plan's entry points, on the CPU with stand-ins for
the HIP runtime (tests/host_runtime.py): nothing is launched for a bad call."""

import os

import pytest

import paper_2509_24093_amd as P
from tests.host_runtime import run

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libcgconv.so not built")

HEAD = """
lib = P.library()
def refused(status, word, want):
    got = status, P.cgconv_last_error()
    assert status == want and word in got[1], (got, word, want)
    assert launches() == []
INVALID, UNSUPPORTED, ALIGNMENT = P.CGCONV_ERR_INVALID_ARG, P.CGCONV_ERR_UNSUPPORTED, P.CGCONV_ERR_ALIGNMENT
"""


def test_plan_create_refuses_bad_sizes(tmp_path):
    run(tmp_path, HEAD + """
for args, word in (((0, 4, 1, 8, 0), "invalid sizes"), ((65536, 4, 1, 8, 0), "invalid sizes"),
                   ((1, 0, 1, 8, 0), "invalid sizes"), ((1, 4, 1, 0, 0), "invalid sizes"),
                   ((1, 4, 1, 8, -1), "invalid sizes"), ((1, 4, -1, 8, 0), "unsupported L_max"),
                   ((1, 4, 9, 8, 0), "unsupported L_max"), ((1, 4, 1, 8, 33), "unsupported states"),
                   ((1, 4, 0, 16385, 0), "unsupported C"), ((1, 4, 8, 964, 0), "unsupported C"),
                   ((1, 4, 8, 2**62, 0), "unsupported C"), ((2, 2**30, 0, 1, 0), "batch*N"),
                   ((65535, 2**62, 0, 1, 0), "batch*N"), ((1, 2**30, 0, 512, 0), "values"),
                   ((1, 2**29, 8, 64, 0), "values")):
    assert not lib.cgconv_seq_plan_create(*args), args
    assert word in P.cgconv_last_error(), (args, P.cgconv_last_error())
plan = P.cgconv_seq_plan_create(2, 8, 1, 16)
assert P.cgconv_seq_plan_info(plan) > 0
refused(lib.cgconv_seq_plan_info(None, None), "NULL", INVALID)
P.cgconv_seq_plan_destroy(plan)
P.cgconv_seq_plan_destroy(None)
""")


def test_norm_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
plan = P.cgconv_seq_plan_create(2, 8, 1, 16)
names = ("x", "weight", "bias", "eps", "y", "mean", "rstd", "codes", "scales")
def norm(plan=plan, dtype=0, **kw):
    a = dict(x=ptr(0), weight=ptr(1), bias=ptr(2), eps=1e-5, y=ptr(3), mean=ptr(4), rstd=ptr(5), codes=ptr(6), scales=ptr(7))
    a.update(kw)
    return lib.cgconv_seq_norm(plan, dtype, *(a[n] for n in names), None)
assert norm() == 0 and len(launches()) == 1
assert norm(weight=None, bias=None, mean=None, rstd=None, codes=None, scales=None) == 0 and len(launches()) == 1
refused(norm(plan=None), "plan is NULL", INVALID)
refused(norm(dtype=2), "dtype", INVALID)
refused(norm(x=None), "x must", INVALID)
refused(norm(y=None), "y must", INVALID)
refused(norm(mean=None), "together", INVALID)
refused(norm(codes=None), "together", INVALID)
refused(norm(eps=-1.0), "eps", INVALID)
refused(norm(eps=float("nan")), "eps", INVALID)
refused(norm(x=ptr(0) + 4), "aligned", ALIGNMENT)
refused(norm(scales=ptr(7) + 8), "aligned", ALIGNMENT)
refused(norm(y=ptr(0)), "overlap", INVALID)
refused(norm(y=ptr(0) + 2 * 8 * 4 * 16 * 4 - 16), "overlap", INVALID)
refused(norm(rstd=ptr(4)), "overlap", INVALID)
assert norm(y=ptr(0) + 2 * 8 * 4 * 16 * 4) == 0
launches()
names2 = ("x", "codes", "scales", "weight", "mean", "rstd", "grad_y", "grad_x", "grad_weight", "grad_bias")
def back(plan=plan, dtype=0, **kw):
    a = dict(x=ptr(0), codes=None, scales=None, weight=ptr(1), mean=ptr(2), rstd=ptr(3), grad_y=ptr(4), grad_x=ptr(5),
             grad_weight=ptr(6), grad_bias=ptr(7))
    a.update(kw)
    return lib.cgconv_seq_norm_backward(plan, dtype, *(a[n] for n in names2), None)
assert back() == 0 and len(launches()) == 2
assert back(grad_weight=None, grad_bias=None) == 0 and len(launches()) == 1
assert back(x=None, codes=ptr(8), scales=ptr(9)) == 0 and len(launches()) == 2
refused(back(plan=None), "plan is NULL", INVALID)
refused(back(x=None), "either x", INVALID)
refused(back(codes=ptr(8), scales=ptr(9)), "either x", INVALID)
refused(back(x=None, codes=ptr(8)), "either x", INVALID)
refused(back(mean=None), "mean must", INVALID)
refused(back(rstd=None), "rstd must", INVALID)
refused(back(grad_y=None), "grad_y must", INVALID)
refused(back(grad_x=None, grad_weight=None, grad_bias=None), "at least one", INVALID)
refused(back(grad_x=ptr(4)), "overlap", INVALID)
refused(back(grad_bias=ptr(6)), "overlap", INVALID)
""")


def test_pack_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
for f in (lib.cgconv_pack8, lib.cgconv_unpack8):
    assert f(0, 10, 40, ptr(0), ptr(1), ptr(2), None) == 0 and len(launches()) == 1
    refused(f(3, 10, 40, ptr(0), ptr(1), ptr(2), None), "dtype", INVALID)
    refused(f(0, 0, 40, ptr(0), ptr(1), ptr(2), None), "invalid sizes", INVALID)
    refused(f(0, 10, 0, ptr(0), ptr(1), ptr(2), None), "invalid sizes", INVALID)
    refused(f(0, 2**62, 2, ptr(0), ptr(1), ptr(2), None), "invalid sizes", INVALID)
    refused(f(0, 2**40, 32, ptr(0), ptr(1), ptr(2), None), "too many", UNSUPPORTED)
    refused(f(0, 10, 40, None, ptr(1), ptr(2), None), "non-NULL", INVALID)
    refused(f(0, 10, 40, ptr(0), ptr(1) + 8, ptr(2), None), "aligned", ALIGNMENT)
    refused(f(0, 10, 40, ptr(0), ptr(1), ptr(1), None), "overlap", INVALID)
""")


def test_norm_launches_are_within_limits(tmp_path):
    run(tmp_path, """
for L in range(9):
    for C in (1, 2, 3, 4, 7, 8, 16, 20, 32, 33, 64, 100, 128, 250, 256, 257, 500, 512, 963, 1000, 4096, 16384):
        if (2 * L + 1) * C > 16384:
            continue
        for B, N in ((1, 1), (3, 70), (8, 16384)):
            plan = P.cgconv_seq_plan_create(B, N, L, C)
            for dtype in (0, 1):
                big = lambda i: 1 << (44 + i) if i else 1 << 43
                assert P.library().cgconv_seq_norm(plan, dtype, big(0), big(1), big(2), 0.0, big(3), big(4), big(5), big(6), big(7), None) == 0, P.cgconv_last_error()
                assert P.library().cgconv_seq_norm_backward(plan, dtype, big(0), None, None, big(1), big(2), big(3), big(4), big(5), big(6), big(7), None) == 0, P.cgconv_last_error()
                for grid, block, lds, allowed in launches():
                    assert block[0] <= 1024 and block[0] % 64 == 0 and lds <= allowed and grid[1] <= 65535, (L, C, grid, block, lds)
            P.cgconv_seq_plan_destroy(plan)
""")


def test_conv_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
plan = P.cgconv_seq_plan_create(2, 8, 1, 16)
def conv(plan=plan, dtype=0, width=4, **kw):
    a = dict(x=ptr(0), weight=ptr(1), bias=ptr(2), activation=1, lengths=ptr(3), state_in=ptr(4), y=ptr(5), state_out=ptr(6))
    a.update(kw)
    return lib.cgconv_seq_conv(plan, dtype, width, *a.values(), None)
assert conv() == 0 and len(launches()) == 1
assert conv(bias=None, lengths=None, state_in=None, state_out=None) == 0 and len(launches()) == 1
refused(conv(plan=None), "plan is NULL", INVALID)
refused(conv(dtype=7), "dtype", INVALID)
refused(conv(width=1), "width", UNSUPPORTED)
refused(conv(width=9), "width", UNSUPPORTED)
refused(conv(x=None), "x must", INVALID)
refused(conv(weight=None), "weight must", INVALID)
refused(conv(y=None), "y must", INVALID)
refused(conv(x=ptr(0) + 8), "aligned", ALIGNMENT)
refused(conv(y=ptr(0)), "overlap", INVALID)
refused(conv(state_out=ptr(4)), "overlap", INVALID)
def step(plan=plan, dtype=0, width=4, **kw):
    a = dict(x=ptr(0), weight=ptr(1), bias=ptr(2), activation=1, state=ptr(4), y=ptr(5))
    a.update(kw)
    return lib.cgconv_seq_conv_step(plan, dtype, width, *a.values(), None)
assert step() == 0 and len(launches()) == 1
refused(step(plan=None), "plan is NULL", INVALID)
refused(step(width=0), "width", UNSUPPORTED)
refused(step(state=None), "state must", INVALID)
refused(step(y=ptr(4)), "overlap", INVALID)
refused(step(y=ptr(0)), "overlap", INVALID)
def back(plan=plan, dtype=0, width=4, **kw):
    a = dict(x=ptr(0), weight=ptr(1), bias=ptr(2), activation=1, lengths=ptr(3), grad_y=ptr(4), grad_x=ptr(5), grad_weight=ptr(6), grad_bias=ptr(7))
    a.update(kw)
    return lib.cgconv_seq_conv_backward(plan, dtype, width, *a.values(), None)
assert back() == 0 and len(launches()) == 2
assert back(grad_weight=None, grad_bias=None) == 0 and len(launches()) == 1
refused(back(plan=None), "plan is NULL", INVALID)
refused(back(width=-4), "width", UNSUPPORTED)
refused(back(grad_y=None), "grad_y must", INVALID)
refused(back(grad_x=None, grad_weight=None, grad_bias=None), "at least one", INVALID)
refused(back(grad_x=ptr(4)), "overlap", INVALID)
refused(back(grad_weight=ptr(1)), "overlap", INVALID)
""")


def test_scan_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
plan, none = P.cgconv_seq_plan_create(2, 8, 1, 16, 16), P.cgconv_seq_plan_create(2, 8, 1, 16)
INPUTS = dict(x=ptr(0), delta=ptr(1), A=ptr(2), Bt=ptr(3), Ct=ptr(4), D=ptr(5), delta_bias=ptr(6))
def scan(plan=plan, dtype=0, **kw):
    a = dict(INPUTS, lengths=ptr(7), state_in=ptr(8), y=ptr(9), state_out=ptr(10))
    a.update(kw)
    return lib.cgconv_seq_scan(plan, dtype, *a.values(), None)
def step(plan=plan, dtype=0, **kw):
    a = dict(INPUTS, state=ptr(8), y=ptr(9))
    a.update(kw)
    return lib.cgconv_seq_scan_step(plan, dtype, *a.values(), None)
GRADS = ("grad_x", "grad_delta", "grad_A", "grad_Bt", "grad_Ct", "grad_D", "grad_delta_bias")
def back(plan=plan, dtype=0, **kw):
    a = dict(INPUTS, lengths=ptr(7), grad_y=ptr(8), **{n: ptr(9 + i) for i, n in enumerate(GRADS)})
    a.update(kw)
    return lib.cgconv_seq_scan_backward(plan, dtype, *a.values(), None)
for f in (scan, step, back):
    assert f() == 0 and len(launches()) >= 1
    assert f(D=None, delta_bias=None) == 0 and len(launches()) >= 1
    refused(f(plan=None), "plan is NULL", INVALID)
    refused(f(plan=none), "no states", INVALID)
    refused(f(dtype=-1), "dtype", INVALID)
    for n in ("x", "delta", "A", "Bt", "Ct"):
        refused(f(**{n: None}), n + " must", INVALID)
        refused(f(**{n: ptr(20) + 4}), "aligned", ALIGNMENT)
assert scan(lengths=None, state_in=None, state_out=None) == 0
launches()
refused(scan(y=ptr(0)), "overlap", INVALID)
refused(scan(state_out=ptr(8)), "overlap", INVALID)
refused(step(state=None), "state must", INVALID)
refused(step(y=ptr(8)), "overlap", INVALID)
refused(back(grad_y=None), "grad_y must", INVALID)
refused(back(**dict.fromkeys(GRADS)), "at least one", INVALID)
refused(back(grad_x=ptr(8)), "overlap", INVALID)
refused(back(grad_Bt=ptr(13) + 16), "overlap", INVALID)
assert back(**dict(dict.fromkeys(GRADS), grad_D=ptr(14))) == 0
""")


def test_conv_and_scan_launches_are_within_limits(tmp_path):
    run(tmp_path, """
big = lambda i: 1 << (40 + i)
for L in (0, 1, 2, 3, 6, 8):
    for C in (1, 2, 3, 4, 20, 33, 64, 300, 1030):
        if (2 * L + 1) * C > 16384:
            continue
        for B, N in ((1, 1), (3, 70), (2, 8192), (200, 33)):
            for S in (1, 8, 16, 17):
                plan = P.cgconv_seq_plan_create(B, N, L, C, S)
                if not plan:
                    raise SystemExit(P.cgconv_last_error())
                lib = P.library()
                for dtype in (0, 1):
                    calls = [lib.cgconv_seq_scan(plan, dtype, *(big(i) for i in range(11)), None),
                             lib.cgconv_seq_scan_step(plan, dtype, *(big(i) for i in range(9)), None),
                             lib.cgconv_seq_scan_backward(plan, dtype, *(big(i) for i in range(16)), None)]
                    for W in (2, 8):
                        calls += [lib.cgconv_seq_conv(plan, dtype, W, big(0), big(1), big(2), 1, *(big(i) for i in range(3, 8)), None),
                                  lib.cgconv_seq_conv_step(plan, dtype, W, big(0), big(1), big(2), 1, big(3), big(4), None),
                                  lib.cgconv_seq_conv_backward(plan, dtype, W, big(0), big(1), big(2), 1, *(big(i) for i in range(3, 9)), None)]
                    assert not any(calls), (calls, P.cgconv_last_error())
                    for grid, block, lds, allowed in launches():
                        assert 64 <= block[0] <= 1024 and block[0] % 64 == 0 and lds <= allowed and grid[1] <= 65535 and grid[2] <= 65535, (L, C, grid, block, lds)
                P.cgconv_seq_plan_destroy(plan)
""")


def test_launches_of_the_largest_sizes(tmp_path):
    """A launch counts its threads along an axis in 32 bits: what fits is launched,
    the rest refused before its launch."""
    run(tmp_path, """
big = lambda i: 1 << (44 + i) if i else 1 << 43
lib = P.library()
def calls(plan, dtype):
    yield lib.cgconv_seq_norm(plan, dtype, big(0), big(1), big(2), 0.0, big(3), big(4), big(5), big(6), big(7), None)
    yield lib.cgconv_seq_norm_backward(plan, dtype, big(0), None, None, big(1), big(2), big(3), big(4), big(5), big(6), big(7), None)
    yield lib.cgconv_seq_conv(plan, dtype, 4, big(0), big(1), big(2), 1, *(big(i) for i in range(3, 7)), None)
    yield lib.cgconv_seq_conv_step(plan, dtype, 4, big(0), big(1), big(2), 1, big(3), big(4), None)
    yield lib.cgconv_seq_conv_backward(plan, dtype, 4, big(0), big(1), big(2), 1, *(big(i) for i in range(3, 8)), None)
refusals = 0
for B, N, L, C in ((1, 2**25, 0, 8), (1, 2**25, 0, 7), (4096, 8192, 2, 1), (65535, 512, 0, 8), (65535, 1, 8, 50), (16, 2**10, 0, 16381),
                   (1, 2**30, 0, 32), (1, 2**30, 0, 1), (1, 2**26, 0, 4096), (65535, 1, 8, 963), (1, 2**27, 3, 33)):
    plan = P.cgconv_seq_plan_create(B, N, L, C)
    assert plan, P.cgconv_last_error()
    ordinary = B * N * (L + 1) ** 2 * C <= 2**28 and B * N <= 2**25
    for dtype in (0, 1):
        for status in calls(plan, dtype):
            assert status in ((0,) if ordinary else (0, P.CGCONV_ERR_UNSUPPORTED)), (B, N, L, C, status, P.cgconv_last_error())
            if status:
                assert "more threads" in P.cgconv_last_error()
                refusals += 1
        for grid, block, lds, allowed in launches():
            assert all(g * b < 2**32 for g, b in zip(grid, block)) and 0 < grid[0] < 2**31, (B, N, L, C, grid, block)
    P.cgconv_seq_plan_destroy(plan)
assert refusals
for dtype in (0, 1):
    assert lib.cgconv_pack8(dtype, 2**29 - 32, 32, big(0), big(5), big(9), None) == 0
    assert lib.cgconv_pack8(dtype, 2**29 - 31, 32, big(0), big(5), big(9), None) == P.CGCONV_ERR_UNSUPPORTED
for grid, block, lds, allowed in launches():
    assert grid[0] * block[0] < 2**32
""")
