"""GPU tests of the gated linear recurrence with gates that remember hundreds
to thousands of steps: what enters a segment of 128 steps leaves it again, so
that the composition of segment maps counts."""

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, host, say
from test_gpu_linrec import _bufs, _compare, _inputs, _run

pytestmark = pytest.mark.gpu
OUTS = ("y", "h_T", "dxg", "dh0")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


@pytest.mark.parametrize("T", [8192, 32768])
@pytest.mark.parametrize("mean", [6.0, 8.0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_same_bits_again(T, mean, dtype):
    """Alone and beside products that take the device's work-groups: which
    maps a segment finds published differs, its results do not."""
    say("linrec again", T, mean, dtype)
    H = 1024
    g = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    t = dict(x=r(T, 1, H), gate=r(T, 1, H) + mean, dy=r(T, 1, H))
    t = {k: v.to(TORCH[dtype]) for k, v in t.items()}
    t.update(h0=r(1, H), dh_T=r(1, H), resets=None, lengths=None)
    first, again = (wm.LinrecBuffers(T, 1, H, TORCH[dtype]) for _ in range(2))
    _run(t, first)
    m, side = r(4096, 4096).bfloat16(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(8):
        if i % 2:
            with torch.cuda.stream(side):
                for _ in range(1 + i):
                    m @ m
        _run(t, again)
        torch.cuda.synchronize()
        wm.status(again)
        for k in OUTS:
            assert torch.equal(getattr(first, k), getattr(again, k)), (k, i)


@pytest.mark.parametrize("T,B,H,dtype,mean,masks", [  # segments, one fan, several, more than one launch takes
    (1100, 2, 40, "fp32", 7.0, False), (1100, 5, 33, "bf16", 9.0, True), (1300, 3, 70, "fp32", 6.0, True),
    (5000, 1, 130, "fp32", 8.0, False), (5100, 4, 10, "bf16", 6.0, True), (8191, 3, 22, "fp32", 9.0, True),
    (20000, 1, 65, "bf16", 7.0, False), (20000, 2, 9, "fp32", 9.0, True), (140001, 1, 3, "fp32", 8.0, False),
    (140001, 3, 1, "bf16", 9.0, True),
    (100, 2, 64, "fp32", 8.0, False), (256, 3, 50, "bf16", 7.0, True),   # a single segment
    (60, 301, 437, "fp32", 7.0, True)])                                  # a wave for all steps
def test_slow_gates(T, B, H, dtype, mean, masks):
    say("linrec slow", T, B, H, dtype, mean, masks)
    d, t = _inputs(T, B, H, dtype, masks, T + B + H)
    t["gate"] = dev(d["gate"] + (mean - 2.0), dtype)
    d["gate"] = host(t["gate"])
    bufs, check = _bufs(T, B, H, dtype)
    _run(t, bufs)
    check()
    _compare(d, bufs, dtype)
