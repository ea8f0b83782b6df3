"""Refusals, launches over the whole range of sizes and reach of every kernel of the
delta rule, the norms around a residual connection and the clipping, on the CPU with
stand-ins for the HIP runtime (tests/host_runtime.py)."""

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
good = dict(batch=2, N=100, L=1, C=12, states=0, heads=4, key_heads=2, key_dim=16, backward=1)
def create(**kw):
    return lib.cgconv_seq_plan_create_rule(*{**good, **kw}.values())
for kw, word in ((dict(heads=0), "heads"), (dict(key_heads=0), "heads"), (dict(key_dim=0), "heads"), (dict(heads=-1), "heads"),
                 (dict(heads=5), "multiple"), (dict(key_heads=3), "multiple"), (dict(key_heads=8), "multiple"),
                 (dict(key_dim=129), "key_dim"), (dict(batch=0), "invalid sizes"), (dict(batch=65535), "batch*heads"),
                 (dict(batch=2**62), "batch*heads"), (dict(N=0), "invalid sizes"), (dict(C=0), "invalid sizes"),
                 (dict(C=-4), "invalid sizes"), (dict(L=9), "L_max"), (dict(states=33), "states"), (dict(N=2**30), "batch*N"),
                 (dict(C=16384 // 3 + 3), "unsupported C")):
    assert not create(**kw), kw
    assert word in P.cgconv_last_error(), (kw, P.cgconv_last_error())
plan, small, scans = create(), create(backward=0), create(states=16)
assert P.cgconv_seq_plan_info(plan) > P.cgconv_seq_plan_info(small) > 0
for p in (plan, small, scans):
    P.cgconv_seq_plan_destroy(p)
""")


def test_delta_rule_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
plan = P.cgconv_seq_plan_create_rule(2, 8, 1, 16, 0, 4, 2, 8, 1)
other = P.cgconv_seq_plan_create(2, 8, 1, 16, 4)
small = P.cgconv_seq_plan_create_rule(2, 8, 1, 16, 0, 4, 2, 8, 0)
ins = dict(q=ptr(0), k=ptr(1), v=ptr(2), decay=ptr(3), beta=ptr(4), scale=1.0, normalize=1)
def rule(plan=plan, dtype=0, **kw):
    a = dict(ins, lengths=ptr(5), state_in=ptr(6), y=ptr(7), state_out=ptr(8)); a.update(kw)
    return lib.cgconv_seq_delta_rule(plan, dtype, *a.values(), None)
def step(plan=plan, dtype=0, **kw):
    a = dict(ins, state=ptr(6), y=ptr(7)); a.update(kw)
    return lib.cgconv_seq_delta_rule_step(plan, dtype, *a.values(), None)
def back(plan=plan, dtype=0, **kw):
    a = dict(ins, lengths=ptr(5), state_in=ptr(6), grad_y=ptr(7), grad_state=ptr(8), gq=ptr(9), gk=ptr(10), gv=ptr(11),
             gdecay=ptr(12), gbeta=ptr(13), gstate=ptr(14)); a.update(kw)
    return lib.cgconv_seq_delta_rule_backward(plan, dtype, *a.values(), None)
for call, needed, written in ((rule, ("q", "k", "v", "decay", "beta", "y"), ("y", "state_out")),
                              (step, ("q", "k", "v", "decay", "beta", "state", "y"), ("y", "state")),
                              (back, ("q", "k", "v", "decay", "beta", "grad_y"), ("gq", "gk", "gv", "gdecay", "gbeta", "gstate"))):
    assert call() == 0 and launches()
    refused(call(plan=None), "plan is NULL", INVALID)
    refused(call(plan=other), "no delta rule", INVALID)
    refused(call(dtype=2), "dtype", INVALID)
    for n in needed:
        refused(call(**{n: None}), "non-NULL", INVALID)
        refused(call(**{n: ptr(0) + 4}), "aligned", ALIGNMENT)
    for n in written:
        refused(call(**{n: ptr(2)}), "overlap", INVALID)
        refused(call(**{n: ptr(2) + 16}), "overlap", INVALID)
    assert call(q=ptr(1)) == 0 and launches()  # the same tensor as key and query
assert rule(lengths=None, state_in=None, state_out=None) == 0 and launches()
assert rule(plan=small) == 0 and step(plan=small) == 0 and launches()
refused(back(plan=small), "backward", INVALID)
refused(back(gq=None, gk=None, gv=None, gdecay=None, gbeta=None, gstate=None), "at least one", INVALID)
assert back(lengths=None, state_in=None, grad_state=None, gq=None, gk=None, gdecay=None, gbeta=None, gstate=None) == 0
assert len(launches()) == 3  # only the values' gradient: no kernel for the others
for p in (plan, other, small):
    P.cgconv_seq_plan_destroy(p)
""")


def test_residual_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
plan = P.cgconv_seq_plan_create(2, 8, 1, 16, 0)
ins = dict(x=ptr(0), u=ptr(1), gate=ptr(2), post_weight=ptr(3), scale=ptr(4), weight=ptr(5))
def fwd(plan=plan, dtype=0, **kw):
    a = dict(ins, bias=ptr(6), eps=1e-5, r=ptr(7), y=ptr(8), stats=ptr(9)); a.update(kw)
    return lib.cgconv_seq_residual_norm(plan, dtype, *a.values(), None)
def back(plan=plan, dtype=0, **kw):
    a = dict(ins, stats=ptr(6), grad_r=ptr(7), grad_y=ptr(8), gx=ptr(9), gu=ptr(10), ggate=ptr(11), gpost=ptr(12),
             gscale=ptr(13), gw=ptr(14), gb=ptr(15)); a.update(kw)
    return lib.cgconv_seq_residual_norm_backward(plan, dtype, *a.values(), None)
for call, needed, written in ((fwd, ("x", "u", "r", "y"), ("r", "y", "stats")),
                              (back, ("x", "u", "stats", "grad_y"), ("gx", "gu", "ggate", "gpost", "gscale", "gw", "gb"))):
    assert call() == 0 and launches()
    refused(call(plan=None), "plan is NULL", INVALID)
    refused(call(dtype=-1), "dtype", INVALID)
    for n in needed:
        refused(call(**{n: None}), "non-NULL", INVALID)
    for n in needed + ("gate", "scale"):
        refused(call(**{n: ptr(20) + 8}), "aligned", ALIGNMENT)
    for n in written:
        refused(call(**{n: ptr(1)}), "overlap", INVALID)
assert fwd(gate=None, post_weight=None, scale=None, weight=None, bias=None, stats=None) == 0 and len(launches()) == 1
assert fwd(x=ptr(1)) == 0 and launches()
for eps in (-1.0, float("nan")):
    refused(fwd(eps=eps), "eps", INVALID)
refused(back(gate=None), "without a gate", INVALID)
refused(back(gx=None, gu=None, ggate=None, gpost=None, gscale=None, gw=None, gb=None), "at least one", INVALID)
assert back(gate=None, ggate=None, grad_r=None) == 0 and len(launches()) == 2
assert back(gpost=None, gscale=None, gw=None, gb=None) == 0 and len(launches()) == 1  # no sums over tokens
P.cgconv_seq_plan_destroy(plan)
""")


def test_clip_refuses_bad_calls(tmp_path):
    run(tmp_path, HEAD + """
def clip(n=2, dtypes=(0, 1), counts=(100, 50), grads=(ptr(0), ptr(1)), out=(ptr(2), ptr(3)), max_norm=1.0, eps=0.0,
         norm=ptr(4), workspace=ptr(5), size=1 << 16):
    return lib.cgconv_clip(n, dtypes and (ctypes.c_int32 * 2)(*dtypes), counts and (ctypes.c_int64 * 2)(*counts),
                           grads and (ctypes.c_void_p * 2)(*grads), out and (ctypes.c_void_p * 2)(*out), max_norm, eps,
                           norm, workspace, size, None)
assert clip() == 0 and len(launches()) == 2
assert clip(out=(ptr(0), ptr(1))) == 0 and len(launches()) == 2
assert clip(n=0, dtypes=None, counts=None, grads=None, out=None) == 0 and len(launches()) == 1
assert clip(counts=(0, 0), grads=(None, None), out=(None, None)) == 0 and len(launches()) == 1
assert clip(grads=(ptr(0), ptr(0))) == 0 and launches()
for kw, word in ((dict(n=-1), "list"), (dict(counts=None), "list"), (dict(dtypes=None), "dtypes"), (dict(grads=None), "grads"),
                 (dict(out=None), "out"), (dict(counts=(-1, 5)), "number of values"), (dict(counts=(2**60, 2**60)), "number of values"),
                 (dict(dtypes=(0, 2)), "dtype"), (dict(grads=(None, ptr(1))), "tensor 0"), (dict(out=(ptr(2), None)), "tensor 1"),
                 (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=float("nan")), "max_norm"), (dict(eps=-1.0), "eps"),
                 (dict(norm=None), "norm"), (dict(workspace=None), "workspace"), (dict(size=8), "workspace"), (dict(size=-1), "workspace"),
                 (dict(out=(ptr(0) + 4, ptr(3))), "overlap"), (dict(out=(ptr(2), ptr(2) + 96)), "overlap"),
                 (dict(out=(ptr(2), ptr(0))), "overlap"), (dict(norm=ptr(0)), "overlap"), (dict(workspace=ptr(2)), "overlap"),
                 (dict(workspace=ptr(4)), "overlap")):
    refused(clip(**kw), word, INVALID)
refused(clip(n=(1 << 20) + 1, dtypes=None, counts=(0, 0), grads=None, out=None) if False else
        lib.cgconv_clip((1 << 20) + 1, None, (ctypes.c_int64 * ((1 << 20) + 1))(), None, None, 1.0, 0.0, ptr(4), ptr(5), 1 << 16, None),
        "tensors", UNSUPPORTED)
for kw in (dict(grads=(ptr(0) + 2, ptr(1))), dict(out=(ptr(2), ptr(3) + 1)), dict(workspace=ptr(5) + 4), dict(norm=ptr(4) + 2)):
    refused(clip(**kw), "aligned", ALIGNMENT)
assert clip(grads=(ptr(0) + 4, ptr(1) + 2)) == 0 and launches()
assert lib.cgconv_clip_workspace(2, (ctypes.c_int64 * 2)(1, 0)) == 16
assert lib.cgconv_clip_workspace(1, (ctypes.c_int64 * 1)(-1)) == INVALID
assert lib.cgconv_clip_workspace(0, None) == 8
""")


def test_launches_of_the_largest_sizes(tmp_path):
    """What fits into a launch is launched, the rest refused before it; nothing up to 2^28
    values and 2^25 tokens is refused."""
    run(tmp_path, HEAD + """
big = lambda i: 1 << (44 + i) if i else 1 << 43
def calls(plan, dtype):
    yield lib.cgconv_seq_delta_rule(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, *(big(i) for i in range(5, 9)), None)
    yield lib.cgconv_seq_delta_rule_step(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, big(5), big(6), None)
    yield lib.cgconv_seq_delta_rule_backward(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, *(big(i) for i in range(5, 15)), None)
    yield lib.cgconv_seq_residual_norm(plan, dtype, *(big(i) for i in range(7)), 0.0, *(big(i) for i in range(7, 10)), None)
    yield lib.cgconv_seq_residual_norm_backward(plan, dtype, *(big(i) for i in range(16)), None)
refusals = 0
for B, N, L, C, H in ((1, 2**25, 0, 8, 1), (1, 2**25, 0, 7, 7), (4096, 8192, 2, 1, 1), (65535, 512, 0, 8, 1), (65535, 1, 8, 50, 1),
                      (3, 2**10, 0, 16384, 16384), (32, 2**20, 0, 1, 1), (1, 2**30, 0, 1, 1), (65535, 1, 8, 963, 1), (1, 2**27, 3, 33, 3),
                      (4095, 16384, 0, 240, 16)):
    for D in (1, 40, 128):
        plan = lib.cgconv_seq_plan_create_rule(B, N, L, C, 0, H, H, D, 1)
        if not plan:
            assert "workspace" in P.cgconv_last_error(), P.cgconv_last_error()
            continue
        ordinary = B * N * (L + 1) ** 2 * C <= 2**28 and B * N <= 2**25
        for dtype in (0, 1):
            for status in calls(plan, dtype):
                assert status in ((0,) if ordinary else (0, UNSUPPORTED)), (B, N, L, C, H, D, status, P.cgconv_last_error())
                if status:
                    assert "more threads" in P.cgconv_last_error()
                    refusals += 1
            for grid, block, lds, allowed in launches():
                assert all(g * b < 2**32 for g, b in zip(grid, block)) and 0 < grid[0] < 2**31, (B, N, L, C, H, D, grid, block)
                assert grid[1] <= 65535 and grid[2] <= 65535 and lds <= allowed, (B, N, L, C, H, D, grid, lds, allowed)
        P.cgconv_seq_plan_destroy(plan)
assert refusals
counts = (ctypes.c_int64 * 3)(2**40, 2**33 + 5, 1)
size = lib.cgconv_clip_workspace(3, counts)
assert lib.cgconv_clip(3, (ctypes.c_int32 * 3)(0, 1, 0), counts, (ctypes.c_void_p * 3)(big(0), big(1), big(2)),
                       (ctypes.c_void_p * 3)(big(3), big(4), big(5)), 1.0, 0.0, ptr(0), ptr(1), size, None) == 0
for grid, block, lds, allowed in launches():
    assert grid[0] <= 16384 + 3
""")


def test_every_kernel_is_reached(tmp_path):
    """No kernel that no call launches, and every size within the limits finds its kernel."""
    run(tmp_path, HEAD + """
big = lambda i: 1 << (44 + i) if i else 1 << 43
fake.fake_hip_idle.restype = ctypes.c_int64
KERNELS = ("rule_prepare_kernel", "rule_state_kernel", "rule_step_kernel", "rule_join_kernel", "rule_reverse_kernel",
           "rule_grads_kernel", "residual_rows_kernel", "residual_rows_bwd_kernel", "residual_wide_kernel",
           "residual_wide_bwd_kernel", "residual_channels_kernel", "residual_channels_bwd_kernel", "residual_sum_kernel",
           "clip_sum_kernel", "clip_total_kernel", "clip_scale_kernel")
def idle():
    buf = ctypes.create_string_buffer(fake.fake_hip_idle(None, ctypes.c_int64(0)) + 1)
    fake.fake_hip_idle(buf, ctypes.c_int64(len(buf)))
    return [n for n in buf.value.decode().split() if any("%d%s" % (len(k), k) in n for k in KERNELS)]
assert all(any("%d%s" % (len(k), k) in n for n in idle()) for k in KERNELS)
def ok(status, *case):
    assert status == 0, case + (P.cgconv_last_error(),)
for D in range(1, 129):
    for N, C, H in ((70, 16, 1), (2000, 16, 1), (70, 200, 1), (2000, 200, 1), (70, 4096, 1), (70, 6, 2)):
        if D % 16 and N == 2000:
            continue
        plan = P.cgconv_seq_plan_create_rule(1, N, 0, C, 0, H, 1, D, 1)
        for dtype in (0, 1):
            ok(lib.cgconv_seq_delta_rule(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, *(big(i) for i in range(5, 9)), None), D, N, C)
            ok(lib.cgconv_seq_delta_rule_step(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, big(5), big(6), None), D, N, C)
            ok(lib.cgconv_seq_delta_rule_backward(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, *(big(i) for i in range(5, 15)), None), D)
        P.cgconv_seq_plan_destroy(plan)
plan = P.cgconv_seq_plan_create_rule(64, 1, 0, 2048, 0, 16, 16, 128, 0)
for dtype in (0, 1):
    ok(lib.cgconv_seq_delta_rule_step(plan, dtype, *(big(i) for i in range(5)), 1.0, 1, big(5), big(6), None))
P.cgconv_seq_plan_destroy(plan)
fake.fake_hip_launches(None, ctypes.c_int64(0))
for L in range(9):
    most = 16384 // (2 * L + 1)
    for C in sorted({*range(1, most + 1, 1 if L < 3 else 7), most}):
        plan = P.cgconv_seq_plan_create(1, 3, L, C, 0)
        for dtype in (0, 1):
            ok(lib.cgconv_seq_residual_norm(plan, dtype, *(big(i) for i in range(7)), 0.0, *(big(i) for i in range(7, 10)), None), L, C)
            ok(lib.cgconv_seq_residual_norm_backward(plan, dtype, *(big(i) for i in range(16)), None), L, C)
        P.cgconv_seq_plan_destroy(plan)
    buf = (ctypes.c_int64 * (8 * 400000))()
    n = fake.fake_hip_launches(buf, ctypes.c_int64(400000))
    assert all(buf[8 * i + 6] <= buf[8 * i + 7] for i in range(n)), "LDS"
for n in (1, 5000):
    counts = (ctypes.c_int64 * n)(*[5] * n)
    at = lambda base: (ctypes.c_void_p * n)(*(base + 64 * i for i in range(n)))
    ok(lib.cgconv_clip(n, (ctypes.c_int32 * n)(), counts, at(big(0)), at(big(1)), 1.0, 0.0, ptr(0), ptr(1), 1 << 17, None))
assert not idle(), "\\n".join(idle())
""")
