"""GPU tests of the norm and rotation of queries and keys and their gradient
(wm_qk_norm, wm_qk_norm_grad): every value against the oracle within the bound
that follows from the roundings, over head widths, rotated widths, both orders of
pairs, shared keys, strided rows and positions of any size."""

from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

from oracle import attend
from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, guarded, host, rounded, say, within

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


CASES = [  # rows, Hq, Hk, D, R, neighbours, dtype, affine
    (1, 1, 1, 1, 0, False, "fp32", True), (1, 1, 1, 2, 2, False, "bf16", True), (3, 2, 1, 2, 2, True, "fp32", False),
    (1, 16, 16, 64, 64, False, "bf16", True), (16, 16, 4, 64, 64, False, "fp32", True), (5, 3, 3, 64, 32, False, "bf16", True),
    (7, 4, 2, 64, 64, True, "bf16", True), (33, 6, 3, 61, 34, True, "fp32", True), (33, 6, 3, 61, 34, False, "bf16", True),
    (9, 2, 2, 128, 64, True, "fp32", False), (10, 5, 1, 96, 96, False, "bf16", True), (6, 3, 2, 100, 100, False, "fp32", True),
    (4, 2, 2, 256, 256, False, "bf16", True), (4, 2, 1, 255, 254, False, "fp32", True), (3, 1, 1, 256, 254, False, "fp32", True), (5, 2, 1, 253, 126, True, "fp32", True),
    (3, 2, 2, 251, 128, True, "bf16", True), (6, 2, 1, 201, 30, False, "bf16", True), (6, 1, 1, 3, 2, False, "bf16", True), (6, 2, 1, 7, 6, True, "fp32", True), (700, 2, 1, 48, 16, False, "bf16", True), (2500, 8, 8, 64, 64, False, "fp32", True),
    (2049, 1, 1, 8, 8, False, "fp32", True), (3000, 3, 2, 32, 32, True, "bf16", True), (20000, 2, 1, 16, 8, False, "bf16", True),
    (5, 24, 24, 128, 128, False, "bf16", True), (64, 7, 7, 40, 24, False, "fp32", True), (2, 1024, 3, 4, 2, True, "fp32", True),
]


def _inputs(rng, rows, Hq, Hk, D, dtype, affine, far):
    x = {n: rounded(rng, (rows, h, D), dtype, 1.5) for n, h in (("q", Hq), ("k", Hk), ("dq", Hq), ("dk", Hk))}
    g = {n: (1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if affine else None for n in "qk"}
    return x, g, rng.integers(-far // 4, far, rows).astype(np.int32)


def _check(bufs, x, g, pos, R, base, nb, dtype, grad=True):
    for n in "qk":
        y, bound = attend.qk_norm(x[n], pos, g[n], EPS, R, base, nb)
        within(host(getattr(bufs, n)).reshape(y.shape), y, bound, dtype, n)
        if grad:
            r = attend.qk_norm_grad(x[n], x["d" + n], pos, g[n], EPS, R, base, nb)
            within(host(getattr(bufs, "d" + n)).reshape(y.shape), r["dx"], r["dx_err"], dtype, "d" + n)
            within(host(getattr(bufs, "dgamma_" + n)), r["dgamma"], r["dgamma_err"], "fp32", "dgamma_" + n)


@pytest.mark.parametrize("rows,Hq,Hk,D,R,nb,dtype,affine", CASES)
def test_norm_rotation_and_gradient(rows, Hq, Hk, D, R, nb, dtype, affine):
    say("qk_norm", rows, Hq, Hk, D, R, nb, dtype, affine)
    rng = np.random.default_rng(rows + D)
    x, g, pos = _inputs(rng, rows, Hq, Hk, D, dtype, affine, 40000)
    rot = wm.Rotary(R, 10000.0, nb)
    bufs, checks = wm.QkNormBuffers(rows, Hq, Hk, D, TORCH[dtype]), []
    for n, h in (("q", Hq), ("k", Hk), ("dq", Hq), ("dk", Hk)):
        t, c = guarded((rows, h, D), TORCH[dtype])
        setattr(bufs, n, t)
        checks.append((n, c))
    for n in ("dgamma_q", "dgamma_k"):
        t, c = guarded((D,), torch.float32)
        setattr(bufs, n, t)
        checks.append((n, c))
    d = {n: dev(v, dtype) for n, v in x.items()}
    w = {"gamma_" + n: None if v is None else dev(v) for n, v in g.items()}
    P = dev(pos)
    wm.qk_norm(d["q"], d["k"], P, rot, **w, eps=EPS, bufs=bufs)
    first = None
    for _ in range(2):
        bufs.workspace.fill_(255)
        wm.qk_norm_grad(d["q"], d["k"], d["dq"], d["dk"], P, rot, **w, eps=EPS, bufs=bufs)
        for n, c in checks:
            c(n)
        _check(bufs, x, g, pos, R, 10000.0, nb, dtype)
        got = [getattr(bufs, n).clone() for n in ("dq", "dk", "dgamma_q", "dgamma_k")]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,R,nb,extra", [(64, 64, False, 0), (64, 32, True, 5), (37, 20, False, 3), (32, 32, True, 1)])
def test_parts_of_one_projection(dtype, D, R, nb, extra):
    rng = np.random.default_rng(D + extra)
    T, B, Hq, Hk = 5, 3, 4, 2
    wide = (Hq + 2 * Hk) * D + extra
    rows = rounded(rng, (T, B, wide), dtype)
    dy = rounded(rng, (T, B, wide), dtype)
    cut = lambda a: (a[..., extra:extra + Hq * D].reshape(T, B, Hq, D),  # noqa: E731
                     a[..., extra + Hq * D:extra + (Hq + Hk) * D].reshape(T, B, Hk, D))
    view = lambda t: (t[..., extra:extra + Hq * D].unflatten(2, (Hq, D)),  # noqa: E731
                      t[..., extra + Hq * D:extra + (Hq + Hk) * D].unflatten(2, (Hk, D)))
    pos = rng.integers(0, 1000, (T, B)).astype(np.int32)
    (q, k), (dq, dk) = view(dev(rows, dtype)), view(dev(dy, dtype))
    rot = wm.Rotary(R, 500.0, nb)
    bufs = wm.QkNormBuffers(T * B, Hq, Hk, D, TORCH[dtype])
    wm.qk_norm(q, k, dev(pos), rot, eps=EPS, bufs=bufs)
    wm.qk_norm_grad(q, k, dq, dk, dev(pos), rot, eps=EPS, bufs=bufs)
    x = {n: a.reshape(T * B, -1, D) for n, a in zip(("q", "k", "dq", "dk"), (*cut(rows), *cut(dy)))}
    _check(bufs, x, {"q": None, "k": None}, pos.reshape(-1), R, 500.0, nb, dtype)


def test_far_positions_turn_exactly():
    # a table of the caller's own: a quarter and three eighths of a turn a step, at positions
    # where a float32 or float64 angle has lost whole turns
    rot = wm.Rotary(4)
    rot.table = torch.tensor([1 << 62, 3 << 61], dtype=torch.int64, device="cuda")
    pos = torch.tensor([0, 1, 2, 3, 2 ** 31 - 1, 2 ** 31 - 2, -1, -2 ** 31, -2 ** 31 + 5], dtype=torch.int32, device="cuda")
    x = torch.tensor([1.0, 1.0, 0.0, 0.0], device="cuda").repeat(len(pos), 1, 1)
    y = host(wm.qk_norm(x, None, pos, rot, eps=0.0).q)[:, 0] / np.sqrt(2.0)
    for i, p in enumerate(host(pos).astype(np.int64)):
        a, b = 2 * np.pi * (p % 4) / 4, 2 * np.pi * (3 * p % 8) / 8
        ref = np.array([np.cos(a), np.cos(b), np.sin(a), np.sin(b)])
        # sine and cosine within 4 u, the norm's 23 u
        assert np.abs(y[i] - ref).max() <= 27 * 2.0 ** -24, int(p)


@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_the_table(base):
    # against 40 decimal digits: rounded to the nearest unit (1/2), and 80-bit arithmetic with a
    # power, a quotient and a constant, within 8 half-units of 2^-63 of a value below 2^62
    getcontext().prec = 40
    pi = Decimal("3.14159265358979323846264338327950288419716939937510")
    R = 128
    t = [int(v) % (1 << 64) for v in wm.Rotary(R, base).table.cpu()]
    assert len(t) == R // 2
    for i, v in enumerate(t):
        f = (-Decimal(2 * i) / R * Decimal(base).ln()).exp() / (2 * pi) * 2 ** 64
        assert abs(v - f) <= Decimal("0.5") + 4 * f / 2 ** 62, i


def test_in_place_and_queries_alone():
    rng = np.random.default_rng(2)
    q, k = dev(rounded(rng, (50, 4, 64), "bf16"), "bf16"), dev(rounded(rng, (50, 2, 64), "bf16"), "bf16")
    pos, rot = dev(np.arange(50, dtype=np.int32)), wm.Rotary(64)
    want = wm.qk_norm(q, k, pos, rot)
    alone = wm.qk_norm(q, None, pos, rot)
    assert torch.equal(alone.q, want.q) and alone.k.numel() == 0
    bufs = wm.QkNormBuffers(50, 4, 2, 64, torch.bfloat16)
    bufs.q, bufs.k = q.clone(), k.clone()
    wm.qk_norm(bufs.q, bufs.k, pos, rot, bufs=bufs)
    assert torch.equal(bufs.q, want.q) and torch.equal(bufs.k, want.k)
    # the gradients in place of those of the outputs
    dq, dk = q.flip(0).contiguous(), k.flip(0).contiguous()
    ref = wm.qk_norm_grad(q, k, dq, dk, pos, rot)
    bufs.dq, bufs.dk = dq.clone(), dk.clone()
    wm.qk_norm_grad(q, k, bufs.dq, bufs.dk, pos, rot, bufs=bufs)
    for n in ("dq", "dk", "dgamma_q", "dgamma_k"):
        assert torch.equal(getattr(bufs, n), getattr(ref, n)), n
    # queries alone: the keys' weights get no gradient
    b = wm.qk_norm_grad(q, None, dq, None, pos, rot)
    assert torch.equal(b.dq, ref.dq) and not bool(b.dgamma_k.any())
    # (the order of its sums goes by the call's sizes, the number of keys among them)
    r = attend.qk_norm_grad(host(q), host(dq), np.arange(50), None, EPS, 64, 10000.0, 0)
    within(host(b.dgamma_q), r["dgamma"], r["dgamma_err"], "fp32", "dgamma_q")
    # without a rotation: angles of 0
    assert torch.equal(wm.qk_norm(q, k, pos, None).q, wm.qk_norm(q, k, torch.zeros_like(pos), rot).q)


def test_outputs_inside_a_projection():
    """In place on the parts of one projection, and gradients as such parts."""
    rng = np.random.default_rng(8)
    qkv = dev(rounded(rng, (6, 5, 7, 32), "fp32"), "fp32")
    dy = dev(rounded(rng, (6, 5, 7, 32), "fp32"), "fp32")
    pos, rot = dev(np.arange(30, dtype=np.int32).reshape(6, 5)), wm.Rotary(32)
    want = wm.qk_norm_grad(qkv[:, :, :4], qkv[:, :, 4:6], dy[:, :, :4], dy[:, :, 4:6], pos, rot)
    wm.qk_norm(qkv[:, :, :4], qkv[:, :, 4:6], pos, rot, bufs=want)
    b, mine, grad = wm.QkNormBuffers(30, 4, 2, 32), qkv.clone(), torch.full_like(qkv, 3.0)
    b.dq, b.dk = grad[:, :, :4], grad[:, :, 4:6]
    wm.qk_norm_grad(qkv[:, :, :4], qkv[:, :, 4:6], dy[:, :, :4], dy[:, :, 4:6], pos, rot, bufs=b)
    b.q, b.k = mine[:, :, :4], mine[:, :, 4:6]
    wm.qk_norm(b.q, b.k, pos, rot, bufs=b)
    assert torch.equal(b.q.reshape(30, 4, 32), want.q) and torch.equal(b.k.reshape(30, 2, 32), want.k)
    assert torch.equal(mine[:, :, 6], qkv[:, :, 6]) and bool((grad[:, :, 6] == 3.0).all())
    assert torch.equal(b.dq.reshape(30, 4, 32), want.dq) and torch.equal(b.dk.reshape(30, 2, 32), want.dk)
    b.q = torch.empty(29, 4, 32, device="cuda")
    with pytest.raises(ValueError):
        wm.qk_norm(qkv[:, :, :4], qkv[:, :, 4:6], pos, rot, bufs=b)


def test_more_than_2_31_values():
    """The last rows of arrays whose offsets pass 32 bits are those of a small call."""
    rows, H, D = 1700000, 21, 64
    x = torch.empty(rows, H, D, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x[:5].normal_(generator=gen)
    x[5:-300] = 1.0
    x[-300:].normal_(generator=gen)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    rot = wm.Rotary(D)
    b = wm.QkNormBuffers(rows, 20, 1, D, torch.bfloat16, grad=True)
    wm.qk_norm(x[:, :20], x[:, 20:], pos, rot, bufs=b)
    wm.qk_norm_grad(x[:, :20], x[:, 20:], x[:, :20], x[:, 20:], pos, rot, bufs=b)
    for part in (slice(0, 300), slice(rows - 300, rows)):
        y = x[part].contiguous()
        s = wm.qk_norm_grad(y[:, :20], y[:, 20:], y[:, :20], y[:, 20:], pos[part].contiguous(), rot)
        wm.qk_norm(y[:, :20], y[:, 20:], pos[part].contiguous(), rot, bufs=s)
        for n in ("q", "k", "dq", "dk"):
            assert torch.equal(getattr(b, n)[part], getattr(s, n)), n


def test_rows_that_can_go_wrong():
    D = 64
    x = np.zeros((5, 2, D), np.float32)
    x[1, 0] = 1e-20                  # squares below fp32's normal numbers
    x[2, 0] = 1e18
    x[3, 1, 5] = np.nan
    x[4, 0, 7] = np.inf
    pos = dev(np.arange(5, dtype=np.int32))
    y = host(wm.qk_norm(dev(x), None, pos, wm.Rotary(D), eps=EPS).q)
    assert not y[0].any()
    ref, bound = attend.qk_norm(x[1:3], np.arange(1, 3), None, EPS, D, 10000.0, 0)
    within(y[1:3], ref, bound, "fp32", "y")
    # a head's own values only
    assert np.isnan(y[3, 1]).all() and np.isfinite(y[3, 0]).all() and np.isnan(y[4, 0]).any() and np.isfinite(y[4, 1]).all()


def test_gradient_against_differences():
    rng = np.random.default_rng(4)
    shape, eps = (6, 3, 16), 2.0 ** -6
    x, dy, v = (rng.standard_normal(shape).astype(np.float32) for _ in range(3))
    g, pos, rot = rng.standard_normal(16).astype(np.float32), dev(np.arange(6, dtype=np.int32) * 7), wm.Rotary(16)
    f = lambda a: host(wm.qk_norm(dev(a), None, pos, rot, gamma_q=dev(g)).q)  # noqa: E731
    b = wm.qk_norm_grad(dev(x), None, dev(dy), None, pos, rot, gamma_q=dev(g))
    slope = float(((f(x + eps * v) - f(x - eps * v)) * dy).sum()) / (2 * eps)
    # the outputs' roundings over 2 eps, and the third-order term: third derivatives of x r
    # are at most some tens over the square of a head's root mean square (here above 0.5)
    tol = 40 * 2.0 ** -24 * np.abs(f(x) * dy).sum() / eps + 10 * eps ** 2 * np.abs(dy * g).sum()
    assert abs(slope - float((host(b.dq) * v).sum())) <= tol


def test_no_rows():
    q = torch.empty(0, 2, 8, device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    bufs = wm.QkNormBuffers(0, 2, 2, 8)
    bufs.dgamma_q.fill_(1.0)
    wm.qk_norm(q, q, pos, wm.Rotary(8), bufs=bufs)
    wm.qk_norm_grad(q, q, q, q, pos, wm.Rotary(8), bufs=bufs)
    assert not bool(bufs.dgamma_q.any()) and not bool(bufs.dgamma_k.any())


def test_buffers_of_another_shape():
    """Arrays that a caller puts in the place of the buffers' own."""
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    q, k, pos, rot = z(4, 2, 8), z(4, 1, 8), torch.zeros(4, dtype=torch.int32, device="cuda"), wm.Rotary(8)
    for name, t in (("q", z(3, 2, 8)), ("k", z(4, 2, 8)), ("dq", z(3, 2, 8)), ("dk", z(4, 1, 7)), ("dgamma_q", z(7)),
                    ("dgamma_k", z(16)[::2]), ("dgamma_k", z(8).double())):
        bufs = wm.QkNormBuffers(4, 2, 1, 8, grad=True)
        setattr(bufs, name, t)
        with pytest.raises(ValueError):
            wm.qk_norm(q, k, pos, rot, bufs=bufs)
            wm.qk_norm_grad(q, k, q, k, pos, rot, bufs=bufs)


def test_refusals():
    q, k = torch.zeros(4, 2, 8, device="cuda"), torch.zeros(4, 1, 8, device="cuda")
    pos, rot = torch.zeros(4, dtype=torch.int32, device="cuda"), wm.Rotary(8)
    for bad in (dict(q=q.double()), dict(k=k.bfloat16()), dict(k=k[:3]), dict(k=k[..., :4]), dict(pos=pos.long()),
                dict(pos=pos[:3]), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(q=q[:, :, 0]),
                dict(gamma_q=torch.ones(7, device="cuda")), dict(bufs=wm.QkNormBuffers(5, 2, 1, 8)),
                dict(q=q.expand(4, 2, 8).as_strided((4, 2, 8), (8, 8, 1)))):
        a = dict(q=q, k=k, pos=pos, gamma_q=None, bufs=None)
        a.update(bad)
        with pytest.raises(ValueError):
            wm.qk_norm(a["q"], a["k"], a["pos"], rot, gamma_q=a["gamma_q"], bufs=a["bufs"])
    with pytest.raises(ValueError):
        wm.qk_norm_grad(q, k, q, k, pos, rot, bufs=wm.QkNormBuffers(4, 2, 1, 8, grad=False))
    for r in (wm.Rotary(10), None):
        with pytest.raises(wm.WmError):
            wm.qk_norm(q, k, pos, r, eps=float("nan") if r is None else 1e-6)
    for R, base in ((7, 10.0), (-2, 10.0), (258, 10.0), (8, 0.5), (8, float("inf")), (8, float("nan"))):
        with pytest.raises(wm.WmError):
            wm.Rotary(R, base)
    with pytest.raises(wm.WmError) as e:
        wm.qk_norm(torch.zeros(1, 1, 257, device="cuda"), None, pos[:1], rot)
    assert e.value.status == wm.WM_ERR_UNSUPPORTED
