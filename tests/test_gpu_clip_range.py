"""GPU tests of gradient clipping at the ends of fp32's range: norms beyond it,
and factors below its normal numbers."""

import numpy as np
import pytest
import torch

from oracle import seq
from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, host, say, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


@pytest.mark.parametrize("limit", [0.0, 1.0, 3e38])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_norm_beyond_fp32_shows_and_nothing_is_clipped(dtype, limit):
    """Finite gradients whose norm fp32 cannot hold: the caller sees an
    infinite norm, and with one the values are the gradients."""
    g = torch.full((5000,), 3e38, device="cuda").to(TORCH[dtype])
    h = torch.randn(40001, device="cuda")
    plan = wm.ClipPlan([g, h], [torch.zeros_like(g), torch.zeros_like(h)])
    norm = wm.clip_grads(plan, limit)
    assert bool(torch.isinf(norm).all())
    assert torch.equal(plan.outs[0], g) and torch.equal(plan.outs[1], h)


def test_the_largest_norm_that_fp32_holds_is_clipped():
    g = torch.full((4,), 1.7e38, device="cuda")  # norm 3.4e38
    plan = wm.ClipPlan([g], [torch.zeros_like(g)])
    assert bool(torch.isfinite(wm.clip_grads(plan, 1.0)).all())
    within(host(plan.outs[0]), np.full(4, 0.5), np.full(4, 3 * seq.U32), "fp32", "out")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [5000, 40003])
@pytest.mark.parametrize("size,limit", [  # factors from 8e-37 down to 0
    (1e30, 1e-12), (1e36, 1e-3), (1e30, 1e-30), (1e36, 1e-40), (3e33, 0.1)])
@pytest.mark.parametrize("place", ["out", "in"])
def test_factors_far_below_one(size, limit, n, dtype, place):
    say("clip factor", size, limit, n, dtype, place)
    rng = np.random.default_rng(n)
    a = host(dev(size * rng.uniform(-1, 1, n), dtype))
    g = dev(a, dtype)
    plan = wm.ClipPlan([g], None if place == "in" else [torch.zeros_like(g)])
    limit = float(np.float32(limit))
    norm = wm.clip_grads(plan, limit)
    total, f, (ref,) = seq.clip([a], limit)
    assert f < 2.0 ** -119 and abs(float(norm) - total) <= 2 * seq.U32 * total  # (below fp32's normal numbers, or near)
    # the factor's rounding and the product's, and the spacing of the type's least numbers
    within(host(plan.outs[0]), ref, 3 * seq.U32 * np.abs(ref) + 2.0 ** -149, dtype, "out")
