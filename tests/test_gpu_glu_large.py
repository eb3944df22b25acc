"""GPU tests of the gated projection where its products take the large tiles
(wm_glu, wm_glu_grad): every value against the same formulas in 64 bits on the
device, within the bounds of oracle/attend.py (written again for device tensors),
at sizes off every tile's edge; and repeated calls, bit for bit."""

import math

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, guarded, say

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


def _close(got, ref, bound, half, what):
    """Within the bound and, for bf16, one rounding of what is stored (and fp32's
    smallest normal number)."""
    lim = bound + half * (ref.abs() + bound) + 2.0 ** -126
    d = (got.double() - ref).abs()
    bad = ~(d <= lim)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((d / lim).max()):.3g} of the bound"


def _act(act, g):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    p = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


CASES = [  # rows, D, F, dtype, act, columns around the rows of x
    (4200, 1000, 2100, "bf16", "silu", 0), (4352, 1024, 2304, "bf16", "gelu", 0), (4107, 1032, 2056, "bf16", "silu", 24),
    (16641, 264, 1000, "bf16", "gelu", 0), (257, 512, 8200, "bf16", "silu", 0), (9000, 8, 2048, "bf16", "silu", 0),
    (2000, 1024, 300, "bf16", "silu", 0), (4200, 1001, 2100, "bf16", "silu", 0), (4500, 520, 1100, "fp32", "gelu", 0),
    (3000, 260, 700, "fp32", "silu", 4), (8192, 256, 256, "bf16", "silu", 0),
    (40000, 1024, 2816, "bf16", "silu", 0), (1100, 64, 4100, "bf16", "silu", 2 ** 20 + 8), (300, 36, 100, "fp32", "gelu", 2 ** 20 + 4),
]


@pytest.mark.parametrize("rows,D,F,dtype,act,wide", CASES)
def test_projection_and_gradient(rows, D, F, dtype, act, wide):
    say("glu large", rows, D, F, dtype, act, wide)
    gen = torch.Generator(device="cuda").manual_seed(rows + D + F)
    dt, half = TORCH[dtype], 2.0 ** -8 if dtype == "bf16" else 0.0
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, W, dh = r(rows, D + wide).to(dt)[:, :D], (r(2 * F, D) / math.sqrt(D)).to(dt), r(rows, F).to(dt)
    bufs, checks = wm.GluBuffers(rows, D, F, dt), []
    for n in ("h", "dx", "dW"):
        t, c = guarded(tuple(getattr(bufs, n).shape), dt)
        setattr(bufs, n, t)
        checks.append((n, c))
    first = None
    for _ in range(3):
        bufs.workspace.fill_(255)
        wm.glu(x, W, act, bufs=bufs)
        wm.glu_grad(x, W, dh, act, bufs=bufs)
        for n, c in checks:
            c(n)
        got = [getattr(bufs, n).clone() for n in ("h", "dx", "dW")]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got
    X, Wd, dH = x.double(), W.double(), dh.double()
    pre, mag = X @ Wd.t(), (D + 1) * U32 * (X.abs() @ Wd.abs().t())
    g, u = pre[:, :F], pre[:, F:]
    a, da = _act(act, g)
    err = (1.13 * mag[:, :F] + 16 * U32 * g.abs()) * u.abs() + a.abs() * mag[:, F:] + U32 * (a * u).abs()
    _close(bufs.h, a * u, err, half, "h")
    cut = 2.0 ** -15 if dtype == "bf16" else 0.0  # of what is saved
    eg, eu = mag[:, :F] + cut * g.abs(), mag[:, F:] + cut * u.abs()
    dg, du = dH * u * da, dH * a
    edg = dH.abs() * (u.abs() * (eg + 16 * U32) + da.abs() * eu) + (half + 2 * U32) * dg.abs()
    edu = dH.abs() * (1.13 * eg + 16 * U32 * g.abs()) + (half + 2 * U32) * du.abs()
    d, e = torch.cat([dg, du], 1), torch.cat([edg, edu], 1) * (1 + half)
    _close(bufs.dx, d @ Wd, e @ Wd.abs() + (2 * F + 1) * U32 * (d.abs() @ Wd.abs()), half, "dx")
    _close(bufs.dW, d.t() @ X, e.t() @ X.abs() + (rows + 1) * U32 * (d.abs().t() @ X.abs()), half, "dW")
    # without what the gradient reads
    alone = wm.glu(x, W, act, bufs=wm.GluBuffers(rows, D, F, dt, grad=False))
    assert torch.equal(alone.h, bufs.h)


def test_more_than_2_31_values():
    """The last rows of factors whose offsets pass 32 bits, against 64 bits."""
    rows, D, F = 530000, 16, 2056
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, D, generator=gen, device="cuda").bfloat16()
    W = (torch.randn(2 * F, D, generator=gen, device="cuda") / 4).bfloat16()
    dh = torch.zeros(rows, F, dtype=torch.bfloat16, device="cuda")
    dh[-200:].normal_(generator=gen)
    bufs = wm.glu(x, W)
    wm.glu_grad(x, W, dh, bufs=bufs)
    X, Wd, dH = x[-200:].double(), W.double(), dh[-200:].double()
    pre, mag, half = X @ Wd.t(), (D + 1) * U32 * (X.abs() @ Wd.abs().t()), 2.0 ** -8
    g, u = pre[:, :F], pre[:, F:]
    a, da = _act("silu", g)
    err = (1.13 * mag[:, :F] + 16 * U32 * g.abs()) * u.abs() + a.abs() * mag[:, F:] + U32 * (a * u).abs()
    _close(bufs.h[-200:], a * u, err, half, "h")
    d = torch.cat([dH * u * da, dH * a], 1)
    e = (half + 2.0 ** -13) * (dH.abs().repeat(1, 2) * torch.cat([u.abs(), g.abs()], 1) * 1.13 + d.abs())
    _close(bufs.dx[-200:], d @ Wd, e @ Wd.abs(), half, "dx")
    # (every other row's gradient is 0)
    assert not bool(bufs.dx[:-200].any())
    _close(bufs.dW, d.t() @ X, e.t() @ X.abs() + 2.0 ** -14 * (d.abs().t() @ X.abs()), half, "dW")


def test_every_kernel_runs():
    """The large tiles' launches and their kernels' names (a case above takes each)."""
    wm.profile_reset()
    wm.profile_enable("glu")
    rows, D, F = 4200, 1000, 2100
    x, W = torch.randn(rows, D, device="cuda").bfloat16(), torch.randn(2 * F, D, device="cuda").bfloat16()
    bufs = wm.glu(x, W)
    wm.glu_grad(x, W, bufs.h.clone(), bufs=bufs)
    torch.cuda.synchronize()
    count = {n: wm.profile_read(n)[1] for n in ("glu_back", "glu_dx", "glu_dw", "glu_sum")}
    wm.profile_enable(None)
    wm.profile_reset()
    assert count == {"glu_back": 1, "glu_dx": 1, "glu_dw": 1, "glu_sum": 2}, count
