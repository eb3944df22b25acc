"""GPU tests of the gated linear recurrence on infinities inside a
trajectory: a state that is infinite stays so until the trajectory ends,
whatever the product of the gates over a tile, a segment or a fan is in fp32,
and both ways of going through the steps agree on it."""

import numpy as np
import pytest
import torch

from oracle import seq
from paper_2205_01435_amd import _lib as wm
from seqcheck import dev, host, say
from test_gpu_linrec import _bufs, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


def _kind(a):
    """0 finite, 1 infinite, -1 minus infinite, 2 NaN."""
    return np.where(np.isnan(a), 2, np.where(np.isinf(a), np.sign(a), 0))


# one tile, one work-group, segments, fans; a wave for all steps
SIZES = [(12, 3, 8), (40, 3, 8), (200, 3, 8), (700, 3, 8), (3000, 2, 8), (40, 1700, 64)]


@pytest.mark.parametrize("T,B,H", SIZES)
@pytest.mark.parametrize("mean", [-110.0, -95.0, -20.0, -7.0, 2.0, 110.0])
@pytest.mark.parametrize("resets", [False, True])
def test_infinities_go_through(T, B, H, mean, resets):
    say("linrec inf", T, B, H, mean, resets)
    d, t = _inputs(T, B, H, "fp32", False, T + H)
    inf = np.inf
    d["gate"] = (d["gate"] + (mean - 2.0)).astype(np.float32).astype(np.float64)
    d["x"] = d["x"].copy()
    d["x"][T // 3, :, 0], d["x"][T // 2, :, 1], d["x"][0, :, 2] = inf, -inf, inf
    d["x"][T // 3, :, 3], d["x"][2 * T // 3, :, 3] = inf, -inf  # NaN from there on
    d["h0"][:, 4], d["h0"][:, 5] = inf, -inf
    d["dy"][2 * T // 3, :, 0], d["dy"][T - 1, :, 6] = -inf, inf
    d["dh_T"][:, 7] = inf
    if resets:
        d["resets"] = np.zeros((T, B), np.uint8)
        d["resets"][T // 2 + 3, 0] = d["resets"][T // 4, 1] = 1
    for k in ("x", "gate", "dy"):
        t[k] = dev(d[k], "fp32")
    t.update(h0=dev(d["h0"].astype(np.float32)), dh_T=dev(d["dh_T"].astype(np.float32)),
             resets=dev(d["resets"]) if resets else None)
    bufs, check = _bufs(T, B, H, "fp32")
    _run(t, bufs)
    check()
    with np.errstate(all="ignore"):
        f = seq.linrec(d["x"], d["gate"], d["h0"], d["resets"])
        o = seq.linrec_grad(d["x"], d["gate"], d["dy"], d["dh_T"], d["h0"], d["resets"])
    for k, ref in (("y", f["y"]), ("h_T", f["h_T"]), ("dx", o["dx"]), ("dh0", o["dh0"])):
        np.testing.assert_array_equal(_kind(host(getattr(bufs, k))), _kind(ref), err_msg=k)
    # (a factor of a gate's derivative may vanish in fp32 beside an infinite one)
    np.testing.assert_array_equal(np.isfinite(host(bufs.dgate)), np.isfinite(o["dgate"]), err_msg="dgate")


@pytest.mark.parametrize("T,B,H", SIZES)
def test_a_gate_of_minus_infinity_forgets(T, B, H):
    """a = 0: what finite state was there is gone, an infinite one leaves NaN (0 times infinity)."""
    d, t = _inputs(T, B, H, "fp32", False, 3)
    d["gate"] = d["gate"].copy()
    d["gate"][T // 2] = -np.inf
    d["h0"][:, 0] = np.inf
    t.update(gate=dev(d["gate"], "fp32"), h0=dev(d["h0"].astype(np.float32)))
    bufs, check = _bufs(T, B, H, "fp32")
    _run(t, bufs)
    check()
    y = host(bufs.y)
    assert np.isposinf(y[:T // 2, :, 0]).all() and np.isnan(y[T // 2:, :, 0]).all()
    np.testing.assert_array_equal(y[T // 2, :, 1:], d["x"][T // 2, :, 1:])
    assert np.isfinite(y[..., 1:]).all()


@pytest.mark.parametrize("T,B,H", [(20, 4, 18), (600, 4, 18), (40, 600, 256)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masked_places_of_the_lowest_value(T, B, H, dtype):
    """Padding that holds the type's lowest value, as masks are often filled."""
    _, t = _inputs(T, B, H, dtype, True, 21)
    clean, _ = _bufs(T, B, H, dtype)
    _run(t, clean)
    pad = (torch.arange(T, device="cuda")[:, None] >= t["lengths"][None, :])[..., None]
    assert bool(pad.any())
    low = torch.finfo(t["x"].dtype).min
    dirty = dict(t, **{k: t[k].masked_fill(pad, low) for k in ("x", "gate", "dy")})
    got, _ = _bufs(T, B, H, dtype)
    _run(dirty, got)
    for k in ("y", "h_T", "dxg", "dh0"):
        assert torch.equal(getattr(got, k), getattr(clean, k)), k
