"""GPU tests of layer norm and its gradient (wm_layer_norm,
wm_layer_norm_grad): every value against the oracle within the bound that
follows from the roundings, over row counts and widths around the kernels'
tiles, strided rows, rows of constant or huge values."""

import numpy as np
import pytest
import torch

from oracle import seq
from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, guarded, host, rounded, say, within

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


CASES = [  # rows, H, dtype, affine
    (1, 1, "fp32", True), (1, 256, "fp32", True), (2, 7, "bf16", False), (5, 63, "fp32", True), (4, 64, "bf16", True),
    (3, 65, "bf16", True), (16, 1024, "bf16", True), (17, 511, "bf16", True), (9, 513, "fp32", False),
    (700, 367, "fp32", True), (3001, 24, "bf16", True), (2100, 130, "fp32", True), (6, 2047, "bf16", True),
    (6, 2049, "fp32", True), (5, 4100, "bf16", True), (3, 8191, "bf16", True), (4, 8192, "fp32", True),
    (1500, 1024, "fp32", False), (5000, 257, "bf16", True), (270, 2048, "fp32", True),
]


def _bufs(rows, H, dtype):
    b = wm.LayerNormBuffers(rows, H, TORCH[dtype])
    checks = []
    for k, shape, dt in (("y", (rows, H), TORCH[dtype]), ("dx", (rows, H), TORCH[dtype]), ("mean", (rows,), torch.float32),
                         ("rstd", (rows,), torch.float32), ("dgamma", (H,), torch.float32),
                         ("dbeta", (H,), torch.float32)):
        t, c = guarded(shape, dt)
        setattr(b, k, t)
        checks.append((k, c))
    return b, lambda: [c(k) for k, c in checks]


@pytest.mark.parametrize("rows,H,dtype,affine", CASES)
def test_layer_norm_and_gradient(rows, H, dtype, affine):
    say("norm", rows, H, dtype, affine)
    rng = np.random.default_rng(rows + H)
    x = rounded(rng, (rows, H), dtype) + 0.5
    x, dy = host(dev(x, dtype)), rounded(rng, (rows, H), dtype)
    g = (1 + 0.3 * rng.standard_normal(H)).astype(np.float32) if affine else None
    b = (0.3 * rng.standard_normal(H)).astype(np.float32) if affine else None
    bufs, check = _bufs(rows, H, dtype)
    X, G, Bt = dev(x, dtype), None if g is None else dev(g), None if b is None else dev(b)
    wm.layer_norm(X, G, Bt, EPS, bufs=bufs)
    y, mu, r = seq.layer_norm(x, g, b, EPS)
    yb, dxh = seq.layer_norm_bound(x, g, b, EPS)
    within(host(bufs.y), y, yb, dtype, "y")
    within(host(bufs.mean), mu, seq.norm_ops(H) * seq.U32 * np.abs(x).mean(-1), "fp32", "mean")
    bufs.workspace.fill_(255)
    first = None
    for _ in range(2):
        wm.layer_norm_grad(X, dev(dy, dtype), G, bufs=bufs)
        check()
        ref, bound = seq.layer_norm_grad(x, dy, g, EPS), seq.layer_norm_grad_bound(x, dy, g, EPS)
        for k, v, e in zip(("dx", "dgamma", "dbeta"), ref, bound):
            within(host(getattr(bufs, k)), v, e, dtype if k == "dx" else "fp32", k)
        got = [bufs.dx.clone(), bufs.dgamma.clone(), bufs.dbeta.clone()]
        assert first is None or all(torch.equal(p, q) for p, q in zip(first, got))
        first = got


@pytest.mark.parametrize("rows,H,dtype", [  # several wide rows a work-group, and around 64 rows of partial sums
    (64, 2000, "fp32"), (65, 2000, "bf16"), (256, 4096, "fp32"), (259, 1025, "bf16"), (300, 8191, "bf16"),
    (1100, 1500, "fp32"), (260, 1024, "fp32"), (261, 100, "bf16")])
def test_column_sums(rows, H, dtype):
    test_layer_norm_and_gradient(rows, H, dtype, True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,at,wide", [(40, 3, 57), (512, 1, 515), (367, 0, 550), (1024, 8, 1040)])
def test_strided_rows(dtype, H, at, wide):
    rng = np.random.default_rng(H)
    x, dy = rounded(rng, (50, 3, wide), dtype), rounded(rng, (50, 3, wide), dtype)
    xs, ds = x[..., at:at + H], dy[..., wide - H:]
    g = rng.standard_normal(H).astype(np.float32)
    X, D = dev(x, dtype)[..., at:at + H], dev(dy, dtype)[..., wide - H:]
    bufs = wm.layer_norm(X, dev(g), None, EPS)
    wm.layer_norm_grad(X, D, dev(g), bufs=bufs)
    within(host(bufs.y).reshape(xs.shape), seq.layer_norm(xs, g, None, EPS)[0], seq.layer_norm_bound(xs, g, None, EPS)[0],
           dtype, "y")
    for k, v, e in zip(("dx", "dgamma", "dbeta"), seq.layer_norm_grad(xs, ds, g, EPS),
                       seq.layer_norm_grad_bound(xs, ds, g, EPS)):
        within(host(getattr(bufs, k)).reshape(v.shape), v, e, dtype if k == "dx" else "fp32", k)


def test_rows_that_can_go_wrong():
    H = 300
    x = np.zeros((6, H))
    x[1] = 5.0                       # constant: variance 0
    x[2] = 1e4 + np.arange(H) % 2    # mean far above the spread
    x[3] = 1e18 * (-1.0) ** np.arange(H)
    x[4, 7] = np.nan
    x[5, 9] = np.inf
    x = x.astype(np.float32).astype(np.float64)
    y = host(wm.layer_norm(dev(x, "fp32"), eps=EPS).y)
    assert not y[0].any()
    ref, bound = seq.layer_norm(x[1:4], None, None, EPS)[0], seq.layer_norm_bound(x[1:4], None, None, EPS)[0]
    # the mean's own error over the standard deviation sqrt(eps) of a constant row
    within(y[1:4], ref, bound, "fp32", "y")
    assert np.isnan(y[4]).all() and np.isnan(y[5]).all()  # and no other row


def test_gradient_against_differences():
    rng = np.random.default_rng(11)
    rows, H, eps = 8, 96, 2.0 ** -6
    x, dy, v = (rng.standard_normal((rows, H)).astype(np.float32) for _ in range(3))
    g, b = rng.standard_normal(H).astype(np.float32), rng.standard_normal(H).astype(np.float32)
    loss = lambda a: float((host(wm.layer_norm(dev(a), dev(g), dev(b)).y) * dy).sum())  # noqa: E731
    bufs = wm.layer_norm(dev(x), dev(g), dev(b))
    wm.layer_norm_grad(dev(x), dev(dy), dev(g), bufs=bufs)
    slope = (loss(x + eps * v) - loss(x - eps * v)) / (2 * eps)
    # roundings of the outputs over 2 eps, and the third-order term eps^2 / 6 times a few
    y = host(bufs.y)
    tol = 40 * seq.U32 * np.abs(y * dy).sum() / eps + 4 * eps ** 2 * np.abs(dy * g).sum()
    assert abs(slope - float((host(bufs.dx) * v).sum())) <= tol


def test_outputs_larger_than_the_cache():
    """The rows of a large call are those of its parts, bit for bit."""
    rows, H = 140001, 512
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.randn(rows, H, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    g, b = torch.randn(H, generator=gen, device="cuda"), torch.randn(H, generator=gen, device="cuda")
    whole = wm.layer_norm(x, g, b)
    wm.layer_norm_grad(x, dy, g, bufs=whole)
    for lo, hi in ((0, 60000), (60000, rows)):
        part = wm.layer_norm(x[lo:hi], g, b)
        wm.layer_norm_grad(x[lo:hi], dy[lo:hi], g, bufs=part)
        for k in ("y", "mean", "rstd", "dx"):
            assert torch.equal(getattr(whole, k)[lo:hi], getattr(part, k)), k


def test_no_rows():
    bufs = wm.LayerNormBuffers(0, 16)
    x = torch.empty(0, 16, device="cuda")
    wm.layer_norm(x, bufs=bufs)
    wm.layer_norm_grad(x, x, bufs=bufs)
    assert not bool(bufs.dgamma.any()) and not bool(bufs.dbeta.any())


def test_refusals():
    x = torch.zeros(4, 32, device="cuda")
    with pytest.raises(ValueError):
        wm.layer_norm(x.double())
    with pytest.raises(ValueError):
        wm.layer_norm(x, torch.ones(31, device="cuda"))
    with pytest.raises(ValueError):
        wm.layer_norm(torch.zeros(32, 4, device="cuda").t())
    with pytest.raises(ValueError):
        wm.layer_norm(x, bufs=wm.LayerNormBuffers(5, 32))
    with pytest.raises(ValueError):
        wm.layer_norm_grad(x, x, bufs=wm.LayerNormBuffers(4, 32, grad=False))
    with pytest.raises(wm.WmError) as e:
        wm.layer_norm(torch.zeros(2, 8193, device="cuda"), bufs=wm.LayerNormBuffers(2, 8193, grad=False))
    assert e.value.status == wm.WM_ERR_UNSUPPORTED
    with pytest.raises(wm.WmError):
        wm.layer_norm(x, eps=float("nan"))
