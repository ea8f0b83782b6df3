"""Launches of the sequence operators over their whole range of sizes, on the CPU
with stand-ins for the HIP runtime (tests/host_runtime.py)."""

import os

import pytest

import paper_2509_24093_amd as P
from tests.host_runtime import run

pytestmark = pytest.mark.skipif(not os.path.exists(P.LIB_PATH), reason="libcgconv.so not built")


def test_scan_launches_of_the_largest_sizes(tmp_path):
    """A launch counts its threads along an axis in 32 bits: what fits is launched,
    the rest refused before its launch; nothing is refused up to 2^28 values and 2^25
    tokens."""
    run(tmp_path, """
big = lambda i: 1 << (44 + i) if i else 1 << 43
lib = P.library()
def calls(plan, dtype):
    yield lib.cgconv_seq_scan(plan, dtype, *(big(i) for i in range(11)), None)
    yield lib.cgconv_seq_scan_step(plan, dtype, *(big(i) for i in range(9)), None)
    yield lib.cgconv_seq_scan_backward(plan, dtype, *(big(i) for i in range(16)), None)
refusals = 0
for B, N, L, C in ((1, 2**25, 0, 8), (1, 2**25, 0, 7), (4096, 8192, 2, 1), (65535, 512, 0, 8), (65535, 1, 8, 50),
                   (16, 2**10, 0, 16381), (32, 2**20, 0, 1), (1, 2**30, 0, 32), (1, 2**30, 0, 1), (65535, 1, 8, 963),
                   (1, 2**27, 3, 33), (65535, 16384, 0, 255)):
    for S in (1, 8, 16, 20, 32):
        plan = P.cgconv_seq_plan_create(B, N, L, C, S)
        ordinary = B * N * (L + 1) ** 2 * C <= 2**28 and B * N <= 2**25
        for dtype in (0, 1):
            for status in calls(plan, dtype):
                assert status in ((0,) if ordinary else (0, P.CGCONV_ERR_UNSUPPORTED)), (B, N, L, C, S, status, P.cgconv_last_error())
                if status:
                    assert "more threads" in P.cgconv_last_error()
                    refusals += 1
            for grid, block, lds, allowed in launches():
                assert all(g * b < 2**32 for g, b in zip(grid, block)) and 0 < grid[0] < 2**31, (B, N, L, C, S, grid, block)
                assert grid[1] <= 65535 and grid[2] <= 65535 and lds <= allowed, (B, N, L, C, S, grid, lds)
        P.cgconv_seq_plan_destroy(plan)
assert refusals
""")


def test_every_kernel_is_reached(tmp_path):
    """The sequence operators have no kernel that no call launches, and every size
    within the documented limits finds its kernel."""
    run(tmp_path, """
big = lambda i: 1 << (44 + i) if i else 1 << 43
lib = P.library()
fake.fake_hip_idle.restype = ctypes.c_int64
def idle():
    buf = ctypes.create_string_buffer(fake.fake_hip_idle(None, ctypes.c_int64(0)) + 1)
    fake.fake_hip_idle(buf, ctypes.c_int64(len(buf)))
    names = buf.value.decode().split()
    return [n for n in names if any("%d%s" % (len(k), k) in n for k in KERNELS)]
KERNELS = ("norm_rows_kernel", "norm_wide_kernel", "norm_rows_bwd_kernel", "norm_wide_bwd_kernel", "norm_sum_kernel",
           "pack_kernel", "conv_kernel", "conv_step_kernel", "conv_bwd_kernel", "conv_sum_kernel", "scan_kernel",
           "carry_kernel", "prepare_kernel", "scan_step_kernel", "ends_kernel", "scan_bwd_kernel", "sum_bc_kernel",
           "delta_kernel", "sum_units_kernel")
before = idle()
assert all(any("%d%s" % (len(k), k) in n for n in before) for k in KERNELS)
def ok(status, *case):
    assert status == 0, case + (P.cgconv_last_error(),)
for L in range(9):
    for C in range(1, 16384 // (2 * L + 1) + 1):
        plan = P.cgconv_seq_plan_create(1, 3, L, C)
        for dtype in (0, 1):
            for codes in ((None, None), (big(6), big(7))):
                ok(lib.cgconv_seq_norm(plan, dtype, big(0), None, None, 0.0, big(3), big(4), big(5), *codes, None), L, C, dtype)
                ok(lib.cgconv_seq_norm_backward(plan, dtype, None if codes[0] else big(0), *codes, None, big(2), big(3), big(4), big(5),
                                                big(8), big(9), None), L, C, dtype)
        P.cgconv_seq_plan_destroy(plan)
    fake.fake_hip_launches(None, ctypes.c_int64(0))
for dtype in (0, 1):
    for rows, C in ((4, 32), (4, 33), (2**23, 32), (2**23, 33)):
        ok(lib.cgconv_pack8(dtype, rows, C, big(0), big(5), big(9), None), rows, C)
        ok(lib.cgconv_unpack8(dtype, rows, C, big(5), big(9), big(0), None), rows, C)
    for C in (1, 2, 4):
        plan = P.cgconv_seq_plan_create(1, 3, 1, C)
        for W in (2, 8):
            ok(lib.cgconv_seq_conv(plan, dtype, W, big(0), big(1), big(2), 1, *(big(i) for i in range(3, 7)), None), C, W)
            ok(lib.cgconv_seq_conv_step(plan, dtype, W, big(0), big(1), big(2), 1, big(3), big(4), None), C, W)
            ok(lib.cgconv_seq_conv_backward(plan, dtype, W, big(0), big(1), big(2), 1, *(big(i) for i in range(3, 8)), None), C, W)
        P.cgconv_seq_plan_destroy(plan)
    for L in range(9):
        for S in range(1, 33):
            for N in (16, 64, 128, 1024, 8192):
                plan = P.cgconv_seq_plan_create(1, N, L, 4, S)
                ok(lib.cgconv_seq_scan(plan, dtype, *(big(i) for i in range(11)), None), L, S, N)
                ok(lib.cgconv_seq_scan_backward(plan, dtype, *(big(i) for i in range(16)), None), L, S, N)
                P.cgconv_seq_plan_destroy(plan)
    for C in (1, 2, 4):
        plan = P.cgconv_seq_plan_create(1, 3, 1, C, 4)
        ok(lib.cgconv_seq_scan_step(plan, dtype, *(big(i) for i in range(9)), None), C)
        P.cgconv_seq_plan_destroy(plan)
assert not idle(), "\\n".join(idle())
""")
