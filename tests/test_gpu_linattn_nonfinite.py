"""GPU tests of linear attention with values that are not finite (wm_linattn,
wm_linattn_grad): they reach what the recurrences take them into, and no earlier
step (in the gradient: no later one), no other trajectory, sequence or head, over
chunks that several trajectories share, split time axes and single steps."""

import numpy as np
import pytest
import torch

from oracle import attend
from oracle.seq import U16, U32
from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, host, rounded, say

pytestmark = pytest.mark.gpu
NAMES = ("y", "h_T", "dq", "dk", "dv", "dh0")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


def _make(T, B, N, K, V, dtype, masks):
    rng = np.random.default_rng(T + B + N + K + V)
    x = {n: rounded(rng, (T, B, N, w), dtype) for n, w in (("q", K), ("k", K), ("v", V), ("dy", V))}
    x["decay"] = np.array([(0.9, 1.0, 0.0, 0.99)[n % 4] for n in range(N)], np.float32)
    x["h0"], x["dh_T"] = (rng.standard_normal((B, N, K, V)).astype(np.float32) for _ in range(2))
    x["resets"], x["lengths"] = np.zeros((T, B), np.uint8), np.full(B, T, np.int32)
    if masks:
        x["resets"][rng.random((T, B)) < 0.04] = 1
        x["resets"][T // 2] = 1
        x["lengths"][1::2] = T - T // 5
    return x


def _check(x, dtype, scale=0.25):
    T, B, N, K = x["q"].shape
    V = x["v"].shape[3]
    d = {n: dev(x[n], dtype) for n in ("q", "k", "v", "dy")}
    e = {n: dev(x[n]) for n in ("decay", "h0", "dh_T", "resets", "lengths")}
    bufs = wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype])
    w = dict(h0=e["h0"], resets=e["resets"], lengths=e["lengths"], bufs=bufs)
    wm.linattn(d["q"], d["k"], d["v"], e["decay"], scale, **w)
    wm.linattn_grad(d["q"], d["k"], d["v"], e["decay"], d["dy"], scale, dh_T=e["dh_T"], **w)
    a, m = [x[n] for n in ("q", "k", "v")], dict(h0=x["h0"], resets=x["resets"], lengths=x["lengths"], dtype=dtype)
    with np.errstate(all="ignore"):
        r = attend.linattn(*a, x["decay"], scale, **m)
        r.update(attend.linattn_grad(*a, x["dy"], x["decay"], scale, dh_T=x["dh_T"], **m))
    for n in NAMES:
        got, ref, bound = host(getattr(bufs, n)), r[n], r[n + "_err"]
        ok = np.isfinite(ref)
        assert np.isfinite(got[ok]).all(), f"{n}: {int((~np.isfinite(got[ok])).sum())} of {int(ok.sum())} finite values are not"
        assert not np.isfinite(got[~ok]).any(), f"{n}: finite where the definition is not"
        # sequences with values that are not finite may go step by step: two roundings of the state
        # a step next to the bound's own
        c, steps = attend._ops(T, max(K, V)) * U32, 2 * T * U32
        bound = bound[ok] * (1 + steps / c)
        lim = bound + (U16 * (np.abs(ref[ok]) + bound) if dtype == "bf16" and n not in ("h_T", "dh0") else 0.0) + 2.0 ** -126
        bad = ~(np.abs(got[ok] - ref[ok]) <= lim)
        assert not bad.any(), f"{n}: {int(bad.sum())} of {bad.size} off"
    return bufs


SIZES = [  # T, B, N, K, V, dtype
    (1, 3, 2, 16, 8, "fp32"), (40, 3, 3, 64, 64, "bf16"), (64, 3, 3, 32, 32, "fp32"), (100, 3, 3, 50, 37, "bf16"), (100, 2, 2, 61, 64, "fp32"),
    (130, 3, 4, 64, 64, "fp32"), (130, 3, 4, 64, 32, "bf16"), (130, 2, 2, 128, 100, "bf16"), (130, 2, 2, 100, 128, "fp32"),
    (130, 70, 4, 32, 64, "bf16"), (130, 70, 4, 64, 32, "fp32"), (300, 2, 3, 64, 64, "bf16"), (300, 2, 3, 33, 20, "fp32"), (400, 1, 2, 128, 128, "bf16"),
]


@pytest.mark.parametrize("masks", [False, True])
@pytest.mark.parametrize("T,B,N,K,V,dtype", SIZES)
def test_what_they_reach(T, B, N, K, V, dtype, masks):
    kinds = (("q", np.inf), ("k", np.nan), ("v", np.inf), ("dy", -np.inf), ("v", np.nan), ("k", -np.inf), ("dy", np.nan), ("q", np.nan))
    for k, (name, bad) in enumerate(kinds if B < 10 else kinds[1 + masks:4:2]):  # (the oracle goes step by step)
        say("linattn not finite", T, B, N, K, V, dtype, masks, name, bad)
        x = _make(T, B, N, K, V, dtype, masks)
        for t, b, n, c in ((T // 2 - 3, 0, 0, 0), (T // 3, B - 1, N - 1, 5 + k)):
            x[name][max(t, 0), b, n, c % x[name].shape[3]] = bad
        _check(x, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_whole_trajectory(dtype):
    """NaN from one reset to the next leaves the trajectories on both sides as they
    are: within the bounds, and bit for bit before the chunks that they share (the state
    that leaves these is summed in another order)."""
    T, B, N, K, V = 200, 2, 2, 64, 64
    x = _make(T, B, N, K, V, dtype, False)
    x["resets"][[70, 110], 0] = 1
    want = _check(x, dtype)
    for n in ("q", "k", "v", "dy"):
        x[n][70:110, 0, 1] = np.nan
    got = _check(x, dtype)
    for n in ("y", "dq", "dk", "dv"):
        keep = torch.ones(T, B, N, dtype=torch.bool, device="cuda")
        keep[slice(64, T) if n in ("y", "dq") else slice(0, 128), 0, 1] = False
        assert torch.equal(getattr(got, n)[keep], getattr(want, n)[keep]), n


@pytest.mark.parametrize("dtype,big", [("fp32", 2.0 ** 100), ("bf16", 2.0 ** 90)])
def test_products_past_the_range(dtype, big):
    """Finite values whose products with another trajectory's overflow."""
    T, B, N, K, V = 130, 2, 2, 32, 32
    x = _make(T, B, N, K, V, dtype, False)
    x["resets"][[30, 31], 0] = 1
    for n in ("q", "k"):
        x[n][30, 0, 0] = 0.0
    x["k"][30, 0, 0] = big  # its own query is 0
    x["q"][31, 0, 0, :] = big * np.arange(1, K + 1)  # sees k of its own step, 0
    x["k"][31, 0, 0] = 0.0
    x["v"][31, 0, 0] = x["dy"][30:32, 0, 0] = 0.0
    _check(x, dtype)


@pytest.mark.parametrize("T", [1, 90, 400])
def test_in_place_and_repeated(T):
    """h_T = h0 and dh0 = dh_T, twice, bit for bit."""
    B, N, K, V = 2, 2, 48, 32
    x = _make(T, B, N, K, V, "fp32", True)
    x["v"][T // 3, 0, 0, 2] = np.nan
    d = {n: dev(x[n], "fp32") for n in ("q", "k", "v", "dy")}
    e = {n: dev(x[n]) for n in ("decay", "h0", "dh_T", "resets", "lengths")}
    runs = []
    for inplace in (False, True, True):
        b = wm.LinattnBuffers(T, B, N, K, V)
        h, g = e["h0"], e["dh_T"]
        if inplace:
            b.h_T.copy_(h)
            b.dh0.copy_(g)
            h, g = b.h_T, b.dh0
        w = dict(resets=e["resets"], lengths=e["lengths"], bufs=b)
        wm.linattn(d["q"], d["k"], d["v"], e["decay"], 0.3, h0=h, **w)
        wm.linattn_grad(d["q"], d["k"], d["v"], e["decay"], d["dy"], 0.3, h0=e["h0"], dh_T=g, **w)
        runs.append([getattr(b, n).clone() for n in NAMES])
    for r in runs[1:]:
        for n, a, b in zip(NAMES, runs[0], r):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)), n
