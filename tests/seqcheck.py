"""Helpers of the sequence-core operators' GPU tests."""

import sys

import numpy as np
import torch

from oracle import seq

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print("[gpu-test]", *a, flush=True)
    sys.stdout.flush()


def dev(a, dtype=None):
    """A device tensor of a numpy array, rounded to ``dtype``."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.to("cuda") if dtype is None else t.to(torch.float32).to(TORCH[dtype]).to("cuda")


def host(t):
    """What a device tensor holds, as float64 (bf16 values are exact)."""
    return t.detach().double().cpu().numpy()


def rounded(rng, shape, dtype, scale=1.0):
    """Seeded normal values that ``dtype`` holds exactly, float64."""
    t = torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32))
    return t.to(TORCH[dtype]).double().numpy()


def within(got, ref, bound, dtype, what):
    """|got - ref| <= bound, plus one rounding of the output where it is bf16
    (and the smallest fp32 normal, below which values may be flushed)."""
    lim = bound + (seq.U16 * (np.abs(ref) + bound) if dtype == "bf16" else 0.0) + 2.0 ** -126
    d = np.abs(got - ref)
    bad = ~(d <= lim)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(d / lim):.3g} of the bound"


def guarded(shape, dtype, pad=64):
    """A contiguous tensor inside a larger one filled with a known value, and
    a function that checks that the surroundings still hold it."""
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * pad,), 12345.0, dtype=dtype, device="cuda")

    def check(what):
        torch.cuda.synchronize()
        edge = torch.cat([whole[:pad], whole[pad + n:]])
        assert bool((edge == torch.full_like(edge, 12345.0)).all()), f"{what}: written outside the output"

    return whole[pad:pad + n].view(shape), check
