"""Helpers of the sequence operators' tests: inputs in a storage type, errors
against a bound per element."""

import numpy as np

U = 2.0 ** -24  # half a step of fp32
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


def torch_gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    torch.cuda.set_device(0)
    return torch


def tdtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def put(a, dtype="fp32"):
    """a on the GPU in dtype, and the values it then has (float64)."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(tdtype(dtype))
    return t, t.float().cpu().numpy().astype(np.float64)


def get(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def check(name, got, ref, magnitude, roundings, dtype="fp32"):
    """|got - ref| <= roundings * 2^-24 * magnitude (the fp32 arithmetic: at most
    that many roundings of values up to magnitude on the way to an element)
    plus the half step of the output's own rounding."""
    got = get(got) if hasattr(got, "detach") else got
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.isfinite(got).all(), name
    bound = roundings * U * magnitude
    bound = bound + HALF[dtype] * (np.abs(ref) + bound) + 1e-37
    worst = np.max(np.abs(got - ref) / bound) if ref.size else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} of the bound"
