"""GPU tests of the gated projection's weight gradient in the large tiles where
the rows of x are parts of wider ones that lie on 16-byte boundaries and their
width is not a multiple of 8 (wm_glu_grad): every value against the same formulas
in 64 bits, the last columns and every step's last row among them, with NaN in what
follows each row."""

import math

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from seqcheck import say
from test_gpu_glu_large import U32, _act, _close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


CASES = [  # rows, D, F, columns behind the rows of x
    (4096, 1003, 4012, 501), (4104, 1002, 4012, 6), (4096, 1001, 4012, 7), (512, 1019, 2048, 5), (4040, 683, 2732, 341), (8, 257, 8192, 7),
]


@pytest.mark.parametrize("last", [False, True])
@pytest.mark.parametrize("rows,D,F,wide", CASES)
def test_weight_gradient(rows, D, F, wide, last):
    """``last``: only the last row of each 64 (and of all) is not 0, so that no other
    row's rounding hides its part."""
    say("glu odd", rows, D, F, wide, last)
    gen = torch.Generator(device="cuda").manual_seed(rows + D + F)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    whole = r(rows, D + wide)
    if last:
        row = torch.arange(rows, device="cuda")
        whole[(row % 64 != 63) & (row != rows - 1)] = 0
    whole[:, D:] = float("nan")
    x, W, dh, half = whole[:, :D], (r(2 * F, D) / math.sqrt(D)).bfloat16(), r(rows, F), 2.0 ** -8
    bufs = wm.glu(x, W)
    wm.glu_grad(x, W, dh, bufs=bufs)
    X, Wd, dH = x.double(), W.double(), dh.double()
    pre, mag = X @ Wd.t(), (D + 1) * U32 * (X.abs() @ Wd.abs().t())
    g, u = pre[:, :F], pre[:, F:]
    a, da = _act("silu", g)
    # the bounds of tests/test_gpu_glu_large.py: sums, 16 significant bits of what is saved, dg and du rounded
    eg, eu = mag[:, :F] + 2.0 ** -15 * g.abs(), mag[:, F:] + 2.0 ** -15 * u.abs()
    dg, du = dH * u * da, dH * a
    edg = dH.abs() * (u.abs() * (eg + 16 * U32) + da.abs() * eu) + (half + 2 * U32) * dg.abs()
    edu = dH.abs() * (1.13 * eg + 16 * U32 * g.abs()) + (half + 2 * U32) * du.abs()
    d, e = torch.cat([dg, du], 1), torch.cat([edg, edu], 1) * (1 + half)
    _close(bufs.dW, d.t() @ X, e.t() @ X.abs() + (rows + 1) * U32 * (d.abs().t() @ X.abs()), half, "dW")
    _close(bufs.dx, d @ Wd, e @ Wd.abs() + (2 * F + 1) * U32 * (d.abs() @ Wd.abs()), half, "dx")


def test_last_column_is_its_neighbour():
    """The same values in the last two columns give the same sums, bit for bit."""
    rows, D, F = 4096, 1003, 4012
    gen = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x, W, dh = r(rows, D + 5)[:, :D], (r(2 * F, D) / 32).bfloat16(), r(rows, F)
    x[:, D - 1] = x[:, D - 2]
    bufs = wm.glu(x, W)
    wm.glu_grad(x, W, dh, bufs=bufs)
    assert torch.equal(bufs.dW[:, D - 1], bufs.dW[:, D - 2])
