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
