"""GPU tests of the gated projection and its gradient (wm_glu, wm_glu_grad):
every value against the oracle within the bound that follows from the roundings,
over sizes around the products' tiles, strided rows and few rows."""

import numpy as np
import pytest
import torch

from oracle import attend
from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, guarded, host, rounded, say, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


CASES = [  # rows, D, F, dtype, act
    (1, 1, 1, "fp32", "silu"), (1, 8, 16, "bf16", "gelu"), (1, 512, 700, "bf16", "silu"), (1, 300, 77, "fp32", "gelu"),
    (2, 64, 64, "bf16", "silu"), (5, 33, 65, "fp32", "silu"), (16, 1024, 200, "bf16", "gelu"), (16, 256, 128, "fp32", "silu"),
    (17, 100, 130, "bf16", "silu"), (31, 367, 97, "fp32", "gelu"), (33, 31, 63, "bf16", "gelu"), (64, 128, 64, "fp32", "silu"),
    (65, 129, 66, "bf16", "silu"), (127, 63, 191, "fp32", "gelu"), (128, 64, 128, "bf16", "silu"), (129, 65, 129, "bf16", "silu"),
    (200, 512, 300, "fp32", "silu"), (300, 367, 979, "bf16", "gelu"), (1000, 40, 24, "fp32", "silu"), (1030, 72, 56, "bf16", "silu"),
    (257, 256, 512, "bf16", "gelu"), (500, 96, 1000, "fp32", "silu"), (2100, 17, 33, "bf16", "gelu"),
    (193, 1000, 40, "bf16", "silu"), (255, 130, 100, "bf16", "gelu"), (256, 61, 130, "fp32", "silu"), (300, 1, 5, "fp32", "gelu"),
]


def _make(rows, D, F, dtype, seed=None):
    rng = np.random.default_rng(rows + D + F if seed is None else seed)
    return (rounded(rng, (rows, D), dtype), rounded(rng, (2 * F, D), dtype, D ** -0.5), rounded(rng, (rows, F), dtype))


def _check(bufs, x, W, dh, act, dtype, grad=True):
    f = attend.glu(x, W, act)
    within(host(bufs.h), f["h"], f["h_err"], dtype, "h")
    if grad:
        g = attend.glu_grad(x, W, dh, act, dtype)
        within(host(bufs.dx), g["dx"], g["dx_err"], dtype, "dx")
        within(host(bufs.dW), g["dW"], g["dW_err"], dtype, "dW")


@pytest.mark.parametrize("rows,D,F,dtype,act", CASES)
def test_projection_and_gradient(rows, D, F, dtype, act):
    say("glu", rows, D, F, dtype, act)
    x, W, dh = _make(rows, D, F, dtype)
    X, Wd, dH = dev(x, dtype), dev(W, dtype), dev(dh, dtype)
    bufs, checks = wm.GluBuffers(rows, D, F, TORCH[dtype]), []
    for n in ("h", "dx", "dW"):
        t, c = guarded(tuple(getattr(bufs, n).shape), TORCH[dtype])
        setattr(bufs, n, t)
        checks.append((n, c))
    # what is saved, between bytes that stay
    whole = torch.full((bufs.saved_bytes + 512,), 77, dtype=torch.uint8, device="cuda")
    bufs.saved = whole[256:256 + bufs.saved_bytes]
    first = None
    for _ in range(2):
        bufs.workspace.fill_(255)
        wm.glu(X, Wd, act, bufs=bufs)
        wm.glu_grad(X, Wd, dH, act, bufs=bufs)
        for n, c in checks:
            c(n)
        assert bool((whole[:256] == 77).all()) and bool((whole[256 + bufs.saved_bytes:] == 77).all())
        _check(bufs, x, W, dh, act, dtype)
        got = [getattr(bufs, n).clone() for n in ("h", "dx", "dW")]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got
    alone = wm.glu(X, Wd, act, bufs=wm.GluBuffers(rows, D, F, TORCH[dtype], grad=False))
    assert torch.equal(alone.h, bufs.h)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,D,F,at,wide", [(50, 40, 30, 3, 57), (130, 64, 64, 8, 96), (9, 31, 40, 1, 33), (200, 128, 65, 0, 131)])
def test_strided_rows(rows, D, F, at, wide, dtype):
    rng = np.random.default_rng(rows)
    x, dh = rounded(rng, (rows, wide), dtype), rounded(rng, (rows, F + 5), dtype)
    W = rounded(rng, (2 * F, D), dtype, D ** -0.5)
    X, dH = dev(x, dtype)[:, at:at + D], dev(dh, dtype)[:, 5:]
    bufs = wm.glu(X, dev(W, dtype))
    wm.glu_grad(X, dev(W, dtype), dH, bufs=bufs)
    _check(bufs, x[:, at:at + D], W, dh[:, 5:], "silu", dtype)


def test_leading_dimensions():
    x, W, dh = _make(12, 24, 20, "bf16")
    a = wm.glu(dev(x, "bf16"), dev(W, "bf16"))
    b = wm.glu(dev(x, "bf16").view(3, 4, 24), dev(W, "bf16"))
    assert torch.equal(a.h, b.h)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_values_that_are_not_finite(dtype):
    """They reach what they enter, as in the plain products, and nothing else."""
    rows, D, F = 150, 70, 90
    x, W, dh = _make(rows, D, F, dtype)
    X, Wd, dH = dev(x, dtype), dev(W, dtype), dev(dh, dtype)
    want = wm.glu(X, Wd)
    wm.glu_grad(X, Wd, dH, bufs=want)
    X[3, 5], X[140, 69] = float("inf"), float("nan")
    dH[77, 88] = float("-inf")
    X[9, 0] = 3.4e38 if dtype == "fp32" else 3.3e38  # finite, at the end of the range
    got = wm.glu(X, Wd)
    wm.glu_grad(X, Wd, dH, bufs=got)
    rows_ok = torch.ones(rows, dtype=torch.bool, device="cuda")
    rows_ok[[3, 9, 140]] = False
    assert torch.equal(got.h[rows_ok], want.h[rows_ok]) and bool(torch.isfinite(got.h[rows_ok]).all())
    assert bool(got.h[140].isnan().all())
    # the signs of the infinite row's factors, against the formulas
    f = Wd[:, 5].float()
    g, u = f[:F] * float("inf"), f[F:] * float("inf")
    pos = (g > 0) & (u != 0)
    assert torch.equal(got.h[3][pos].float(), (g * u)[pos])
    # the large row: products of the range's end with the weights, in 64 bits
    ref = X[9].double() @ Wd.double().t()
    h = torch.nn.functional.silu(ref[:F]) * ref[F:]
    big, small = h.abs() > 3.5e38, h.abs() < 1e30
    assert bool(torch.isinf(got.h[9][big]).all()) and bool(torch.isfinite(got.h[9][small & (ref[:F].abs() > 1e30)]).all())
    rows_ok[77] = False
    assert torch.equal(got.dx[rows_ok], want.dx[rows_ok])
    assert bool((~torch.isfinite(got.dx[77])).all())


def test_large_and_small_gates():
    """Both ends of the activation: exact zeros and the identity."""
    g = np.array([-1e4, -100.0, -20.0, -1e-30, 0.0, 1e-30, 20.0, 100.0, 1e4], np.float32)
    for act in ("silu", "gelu"):
        x = g[:, None]
        W = np.array([[1.0], [1.0]], np.float32)  # g = u = x
        b = wm.glu(dev(x), dev(W), act)
        wm.glu_grad(dev(x), dev(W), torch.ones(len(g), 1, device="cuda"), act, bufs=b)
        f, r = attend.glu(x, W, act), attend.glu_grad(x, W, np.ones((len(g), 1)), act)
        within(host(b.h), f["h"], f["h_err"], "fp32", "h")
        within(host(b.dx), r["dx"], r["dx_err"], "fp32", "dx")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_against_differences(act):
    x, W, dh = (a.astype(np.float32) for a in _make(20, 12, 10, "fp32"))
    rng = np.random.default_rng(1)
    b = wm.glu(dev(x), dev(W), act)
    wm.glu_grad(dev(x), dev(W), dev(dh), act, bufs=b)
    eps = 2.0 ** -7
    for n, a, got in (("x", x, b.dx), ("W", W, b.dW)):
        v = (rng.standard_normal(a.shape) / np.sqrt(a.shape[-1])).astype(np.float32)
        hs = [host(wm.glu(dev(x + s * v) if n == "x" else dev(x), dev(W + s * v) if n == "W" else dev(W), act).h)
              for s in (eps, -eps)]
        slope = float(((hs[0] - hs[1]) * dh).sum()) / (2 * eps)
        # roundings over 2 eps; the third-order term: third derivatives of act(g) u along v are
        # at most 3 (|u| + 3) times the cube of the factors' change a unit step
        f = attend.glu(x, W, act)
        dv = np.abs(v) @ np.abs(W).T if n == "x" else np.abs(x) @ np.abs(v).T
        third = np.maximum(dv[:, :10], dv[:, 10:]) ** 3 * 3 * (np.abs(f["u"]) + 3)
        tol = float((2 * f["h_err"] * np.abs(dh)).sum()) / eps + eps ** 2 / 6 * float((third * np.abs(dh)).sum())
        assert abs(slope - float((host(got) * v).sum())) <= tol, n


@pytest.mark.parametrize("rows,D,F,dtype", [(4, 256, 300, "bf16"), (300, 130, 90, "fp32"), (2000, 64, 40, "bf16")])
def test_graph_and_streams(rows, D, F, dtype):
    X, Wd, dH = (dev(a, dtype) for a in _make(rows, D, F, dtype))
    bufs, eager = (wm.GluBuffers(rows, D, F, TORCH[dtype]) for _ in range(2))

    def run(b):
        wm.glu(X, Wd, bufs=b)
        wm.glu_grad(X, Wd, dH, bufs=b)

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        run(bufs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run(bufs)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(4):
        for t in (X, Wd, dH):
            t.normal_(generator=gen)
        run(eager)
        for n in ("h", "dx", "dW"):
            getattr(bufs, n).zero_()
        torch.cuda.synchronize()
        graph.replay()
        run(eager)
        torch.cuda.synchronize()
        for n in ("h", "dx", "dW"):
            assert torch.equal(getattr(bufs, n), getattr(eager, n)), (i, n)


def test_no_rows():
    W = torch.randn(12, 8, device="cuda")
    x = torch.empty(0, 8, device="cuda")
    bufs = wm.glu(x, W)
    bufs.dW.fill_(1.0)
    wm.glu_grad(x, W, torch.empty(0, 6, device="cuda"), bufs=bufs)
    assert not bool(bufs.dW.any())


def test_buffers_of_another_shape():
    """Arrays that a caller puts in the place of the buffers' own."""
    x, W, dh = torch.zeros(4, 8, device="cuda"), torch.zeros(12, 8, device="cuda"), torch.zeros(4, 6, device="cuda")
    for name, shape in (("h", (3, 6)), ("h", (4, 5)), ("dx", (3, 8)), ("dx", (4, 7)), ("dW", (11, 8)), ("dW", (6, 16))):
        bufs = wm.GluBuffers(4, 8, 6)
        setattr(bufs, name, torch.zeros(shape, device="cuda"))
        with pytest.raises(ValueError):
            wm.glu(x, W, bufs=bufs)
            wm.glu_grad(x, W, dh, bufs=bufs)


def test_refusals():
    x, W, dh = torch.zeros(4, 8, device="cuda"), torch.zeros(12, 8, device="cuda"), torch.zeros(4, 6, device="cuda")
    for bad in (dict(x=x.double()), dict(W=W.bfloat16()), dict(W=W[:11]), dict(W=W[:, :7]), dict(W=W.t().contiguous().t()),
                dict(x=x[:, :7]), dict(act="relu"), dict(bufs=wm.GluBuffers(4, 8, 7)),
                dict(x=torch.zeros(8, 4, device="cuda").t())):
        with pytest.raises(ValueError):
            wm.glu(**{**dict(x=x, W=W), **bad})
    with pytest.raises(ValueError):
        wm.glu_grad(x, W, dh)
    with pytest.raises(ValueError):
        wm.glu_grad(x, W, dh, bufs=wm.GluBuffers(4, 8, 6, grad=False))
    with pytest.raises(ValueError):
        wm.glu_grad(x, W, dh[:3], bufs=wm.GluBuffers(4, 8, 6))
    bufs = wm.GluBuffers(4, 8, 6)
    bufs.ws_bytes -= 1
    with pytest.raises(wm.WmError) as e:
        wm.glu_grad(x, W, dh, bufs=bufs)
    assert e.value.status == wm.WM_ERR_WORKSPACE
    bufs = wm.GluBuffers(4, 8, 6)
    bufs.saved_bytes -= 1
    for f in (lambda: wm.glu(x, W, bufs=bufs), lambda: wm.glu_grad(x, W, dh, bufs=bufs)):
        with pytest.raises(wm.WmError) as e:
            f()
        assert e.value.status == wm.WM_ERR_WORKSPACE
