"""GPU tests of linear attention with one decay a head and its gradient
(wm_linattn, wm_linattn_grad): every value against the oracle within the bound
that follows from the roundings, over lengths around the chunks of 64 steps and
the split of the time axis, odd head widths, resets, padding and strides."""

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


def _make(T, B, N, K, V, dtype, masks, seed=None):
    rng = np.random.default_rng(T + 7 * B + N + K + V if seed is None else seed)
    x = {n: rounded(rng, (T, B, N, w), dtype) for n, w in (("q", K), ("k", K), ("v", V), ("dy", V))}
    x["decay"] = np.array([(1.0, 0.9, 0.99, 0.0, 0.5, 1 - 2.0 ** -10)[n % 6] for n in range(N)], np.float32)
    x["h0"], x["dh_T"] = (rng.standard_normal((B, N, K, V)).astype(np.float32) for _ in range(2))
    x["resets"] = x["lengths"] = None
    if masks:
        x["resets"] = (rng.random((T, B)) < max(2.0 / max(T, 1), 0.02)).astype(np.uint8)
        if T:
            x["resets"][0, ::2] = 1
            x["resets"][T - 1, ::3] = 1
        x["lengths"] = rng.integers(0, T + 1, B).astype(np.int32)
        x["lengths"][:3] = (T, 0, min(T, 1))[:B]
    return x


def _device(x, dtype):
    d = {n: dev(x[n], dtype) for n in ("q", "k", "v", "dy")}
    d.update({n: None if x[n] is None else dev(x[n]) for n in ("decay", "h0", "dh_T", "resets", "lengths")})
    return d


def _guard(bufs):
    checks = []
    for n in ("y", "h_T", "dq", "dk", "dv", "dh0"):
        t = getattr(bufs, n)
        if t is None:
            continue
        g, c = guarded(tuple(t.shape), t.dtype)
        setattr(bufs, n, g)
        checks.append((n, c))
    return lambda: [c(n) for n, c in checks]


def _run(d, bufs, scale, h0=True, grad=True):
    w = dict(scale=scale, h0=d["h0"] if h0 else None, resets=d["resets"], lengths=d["lengths"], bufs=bufs)
    wm.linattn(d["q"], d["k"], d["v"], d["decay"], **w)
    if grad:
        wm.linattn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], dh_T=d["dh_T"] if h0 else None, **w)


def _check(bufs, x, scale, dtype, h0=True, grad=True):
    a = [x[n] for n in ("q", "k", "v")]
    w = dict(h0=x["h0"] if h0 else None, resets=x["resets"], lengths=x["lengths"], dtype=dtype)
    r = attend.linattn(*a, x["decay"], scale, **w)
    if grad:
        r.update(attend.linattn_grad(*a, x["dy"], x["decay"], scale, dh_T=x["dh_T"] if h0 else None, **w))
    for n in ("y", "h_T") + (("dq", "dk", "dv", "dh0") if grad else ()):
        within(host(getattr(bufs, n)), r[n], r[n + "_err"], "fp32" if n in ("h_T", "dh0") else dtype, n)


CASES = [  # T, B, N, K, V, dtype, masks
    (1, 1, 1, 1, 1, "fp32", False), (1, 3, 2, 64, 64, "fp32", True), (1, 5, 2, 50, 37, "bf16", True), (2, 4, 3, 16, 8, "bf16", True),
    (1, 2, 3, 128, 128, "bf16", False), (1, 3, 1, 33, 1, "fp32", True),
    (3, 1, 6, 32, 32, "fp32", False), (63, 5, 2, 64, 64, "bf16", True), (64, 5, 2, 64, 64, "fp32", True),
    (65, 5, 2, 64, 64, "bf16", True), (64, 2, 1, 1, 128, "fp32", True), (70, 3, 2, 128, 1, "bf16", True),
    (127, 4, 6, 40, 24, "fp32", True), (128, 6, 2, 64, 32, "bf16", False), (130, 3, 2, 31, 33, "fp32", True),
    (100, 2, 2, 128, 128, "fp32", True), (150, 2, 2, 128, 128, "bf16", True), (145, 4, 3, 50, 37, "bf16", True),
    (96, 3, 2, 65, 66, "fp32", True), (96, 3, 2, 127, 95, "bf16", True), (66, 2, 3, 5, 3, "bf16", True), (66, 2, 3, 2, 34, "fp32", True),
    # heads around the numbers by which work-groups are formed
    (130, 70, 4, 50, 37, "bf16", True), (129, 85, 3, 33, 64, "fp32", True), (66, 100, 4, 61, 40, "bf16", True), (70, 128, 3, 64, 64, "fp32", True),
    # split time axis
    (255, 2, 2, 32, 32, "fp32", True), (256, 2, 2, 32, 32, "bf16", True), (300, 3, 6, 24, 40, "fp32", True),
    (577, 2, 3, 64, 64, "bf16", True), (640, 1, 2, 64, 64, "fp32", False), (1000, 3, 1, 17, 70, "bf16", True),
    (1025, 1, 2, 100, 128, "fp32", True), (2000, 1, 6, 16, 16, "fp32", True),
]


@pytest.mark.parametrize("T,B,N,K,V,dtype,masks", CASES)
def test_attention_and_gradient(T, B, N, K, V, dtype, masks):
    say("linattn", T, B, N, K, V, dtype, masks)
    x = _make(T, B, N, K, V, dtype, masks)
    d, scale = _device(x, dtype), K ** -0.5
    first = None
    for _ in range(2):
        bufs = wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype])
        check = _guard(bufs)
        bufs.workspace.fill_(255)
        _run(d, bufs, scale)
        check()
        _check(bufs, x, scale, dtype)
        got = [getattr(bufs, n).clone() for n in ("y", "h_T", "dq", "dk", "dv", "dh0")]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got
    # without the states that the gradient reads
    alone = wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype], grad=False)
    _run(d, alone, scale, grad=False)
    assert torch.equal(alone.y, bufs.y) and torch.equal(alone.h_T, bufs.h_T)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_steps_far_apart(dtype):
    """Inputs whose steps lie more than 2^31 / 65 bytes apart."""
    T, B, N, K, V = 66, 2, 2, 64, 32
    say("linattn far", dtype)
    x = _make(T, B, N, K, V, dtype, True)
    d, step = _device(x, dtype), 2 ** 24 + 2 ** 20
    wide = torch.empty(T, step, dtype=TORCH[dtype], device="cuda")
    at = 0
    for n in ("q", "k", "v", "dy"):
        w = B * N * d[n].shape[3]
        part = wide[:, at:at + w].view(T, B, N, -1)
        part.copy_(d[n])
        d[n], at = part, at + w
    bufs = wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype])
    _run(d, bufs, 0.25)
    _check(bufs, x, 0.25, dtype)


@pytest.mark.parametrize("T,B,N,K,V,dtype", [(1, 2, 2, 8, 8, "fp32"), (70, 2, 2, 20, 20, "bf16"), (400, 1, 2, 32, 48, "fp32")])
def test_without_states(T, B, N, K, V, dtype):
    """No h0 and no dh_T are zeros; negative scales too."""
    x = _make(T, B, N, K, V, dtype, True)
    bufs = wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype])
    _run(_device(x, dtype), bufs, -0.3, h0=False)
    _check(bufs, x, -0.3, dtype, h0=False)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [1, 90, 300])
def test_parts_of_one_projection(T, dtype):
    B, N, K, V, extra = 3, 2, 24, 40, 3
    x = _make(T, B, N, K, V, dtype, True)
    row = np.concatenate([x[n].reshape(T, B, -1) for n in ("q", "k", "v", "dy")] + [np.full((T, B, extra), 7.0)], 2)
    whole, d = dev(row, dtype), _device(x, dtype)
    want, got = (wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype]) for _ in range(2))
    _run(d, want, 0.2)
    e, at = dict(d), 0
    for n, w in (("q", K), ("k", K), ("v", V), ("dy", V)):
        e[n] = whole[..., at:at + N * w].unflatten(2, (N, w))
        at += N * w
    _run(e, got, 0.2)
    # rows that come batch first
    f = {n: t.transpose(0, 1).contiguous().transpose(0, 1) if n in ("q", "k", "v", "dy") else t for n, t in d.items()}
    third = wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype])
    _run(f, third, 0.2)
    for n in ("y", "h_T", "dq", "dk", "dv", "dh0"):
        assert torch.equal(getattr(got, n), getattr(want, n)) and torch.equal(getattr(third, n), getattr(want, n)), n


@pytest.mark.parametrize("T", [1, 90, 400])
def test_gradients_inside_wider_rows(T):
    B, N, K = 2, 2, 32
    x = _make(T, B, N, K, K, "fp32", True)
    d = _device(x, "fp32")
    want, got = (wm.LinattnBuffers(T, B, N, K, K) for _ in range(2))
    _run(d, want, 0.2)
    whole = torch.full((T, B, 4, N, K), 5.0, device="cuda")
    got.dq, got.dk, got.dv = whole[:, :, 0], whole[:, :, 1], whole[:, :, 3]
    _run(d, got, 0.2)
    for n in ("dq", "dk", "dv"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n
    assert bool((whole[:, :, 2] == 5.0).all())
    got.y = torch.empty(T, B, 2 * N, K, device="cuda")[:, :, :N]
    if T > 1:
        with pytest.raises(ValueError):
            _run(d, got, 0.2)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min])
@pytest.mark.parametrize("T", [1, 100, 300])
def test_padding_enters_nothing(T, bad):
    x = _make(T, 4, 2, 32, 32, "bf16", True)
    d = _device(x, "bf16")
    want, got = (wm.LinattnBuffers(T, 4, 2, 32, 32, torch.bfloat16) for _ in range(2))
    _run(d, want, 0.2)
    pad = torch.arange(T, device="cuda")[:, None] >= d["lengths"][None]
    for n in ("q", "k", "v", "dy"):
        d[n] = torch.where(pad[..., None, None], bad, d[n])
    d["resets"] = torch.where(pad, 1, d["resets"]).to(torch.uint8)
    _run(d, got, 0.2)
    for n in ("y", "h_T", "dq", "dk", "dv", "dh0"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n
    assert not bool(got.y[pad].any()) and not bool(got.dq[pad].any()) and not bool(got.dk[pad].any())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T", [1, 70, 400])
def test_a_reset_drops_the_state(T, bad):
    """States that are not finite end at a reset, in both directions."""
    x = _make(T, 2, 2, 16, 16, "fp32", False)
    x["resets"] = np.zeros((T, 2), np.uint8)
    x["resets"][0] = 1
    d = _device(x, "fp32")
    want, got = (wm.LinattnBuffers(T, 2, 2, 16, 16) for _ in range(2))
    _run(d, want, 0.2)
    d["h0"] = torch.full_like(d["h0"], bad)
    _run(d, got, 0.2)
    for n in ("y", "h_T", "dq", "dk", "dv", "dh0"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n
    assert not bool(got.dh0.any())
    # from the end: only the last trajectory's steps see dh_T
    if T > 1:
        cut = T - 5
        d = _device(x, "fp32")
        d["resets"][cut] = 1
        _run(d, want, 0.2)
        d["dh_T"] = torch.full_like(d["dh_T"], bad)
        _run(d, got, 0.2)
        edge = cut // 64 * 64  # the chunk that the reset lies in
        for n in ("dk", "dv"):
            assert torch.equal(getattr(got, n)[:edge], getattr(want, n)[:edge]), n
        assert torch.equal(got.dh0, want.dh0) and torch.equal(got.dq, want.dq)


def test_a_sequence_and_head_of_its_own():
    """Values that are not finite reach no other sequence and no other head, and
    no earlier chunk of their own."""
    T, B, N = 300, 3, 2
    x = _make(T, B, N, 32, 16, "bf16", False)
    d = _device(x, "bf16")
    want, got = (wm.LinattnBuffers(T, B, N, 32, 16, torch.bfloat16) for _ in range(2))
    _run(d, want, 0.2, grad=False)
    d["v"][200, 1, 1, 3] = float("nan")
    _run(d, got, 0.2, grad=False)
    keep = torch.ones(T, B, N, dtype=torch.bool, device="cuda")
    keep[192:, 1, 1] = False
    assert torch.equal(got.y[keep], want.y[keep])
    assert bool(got.y[200:, 1, 1].isnan().any())


def test_steps_are_the_sequence():
    """One step at a time from a kept state, in place, against the whole."""
    T, B, N, K, V = 40, 3, 2, 48, 20
    x = _make(T, B, N, K, V, "fp32", True)
    x["lengths"] = None
    d = _device(x, "fp32")
    whole = wm.linattn(d["q"], d["k"], d["v"], d["decay"], 0.25, h0=d["h0"], resets=d["resets"])
    bufs = wm.LinattnBuffers(1, B, N, K, V, grad=False)
    bufs.h_T.copy_(d["h0"])
    ys = []
    for t in range(T):
        s = slice(t, t + 1)
        wm.linattn(d["q"][s], d["k"][s], d["v"][s], d["decay"], 0.25, h0=bufs.h_T, resets=d["resets"][s], bufs=bufs)
        ys.append(bufs.y[0].clone())
    r = attend.linattn(x["q"], x["k"], x["v"], x["decay"], 0.25, x["h0"], x["resets"])
    # both are off by at most the bound
    assert (np.abs(host(torch.stack(ys)) - host(whole.y)) <= 2 * r["y_err"] + 1e-30).all()
    assert (np.abs(host(bufs.h_T) - host(whole.h_T)) <= 2 * r["h_T_err"] + 1e-30).all()


@pytest.mark.parametrize("T", [60, 500])
def test_states_in_place(T):
    x = _make(T, 2, 2, 32, 32, "bf16", True)
    d = _device(x, "bf16")
    want, got = (wm.LinattnBuffers(T, 2, 2, 32, 32, torch.bfloat16) for _ in range(2))
    _run(d, want, 0.2)
    got.h_T.copy_(d["h0"])
    wm.linattn(d["q"], d["k"], d["v"], d["decay"], 0.2, h0=got.h_T, resets=d["resets"], lengths=d["lengths"], bufs=got)
    got.dh0.copy_(d["dh_T"])
    wm.linattn_grad(d["q"], d["k"], d["v"], d["decay"], d["dy"], 0.2, h0=d["h0"], dh_T=got.dh0, resets=d["resets"],
                    lengths=d["lengths"], bufs=got)
    for n in ("y", "h_T", "dq", "dk", "dv", "dh0"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n


def test_decays_outside_act_as_clamped_and_lengths_too():
    x = _make(80, 4, 2, 16, 16, "fp32", True)
    d = _device(x, "fp32")
    d["decay"] = torch.tensor([1.0, 0.0], device="cuda")
    want, got = (wm.LinattnBuffers(80, 4, 2, 16, 16) for _ in range(2))
    d["lengths"] = torch.tensor([80, 0, 80, 0], dtype=torch.int32, device="cuda")
    _run(d, want, 0.2)
    d["decay"] = torch.tensor([1.5, -0.5], device="cuda")
    d["lengths"] = torch.tensor([10 ** 9, -5, 81, -2 ** 31], dtype=torch.int32, device="cuda")
    _run(d, got, 0.2)
    for n in ("y", "h_T", "dq", "dk", "dv", "dh0"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n


def test_gradient_against_differences():
    x = _make(75, 2, 2, 12, 10, "fp32", True)
    d, rng = _device(x, "fp32"), np.random.default_rng(9)
    bufs = wm.LinattnBuffers(75, 2, 2, 12, 10)
    _run(d, bufs, 0.3)
    loss = lambda e: [host(t) * w for t, w in zip(_fwd(e), (x["dy"], x["dh_T"]))]  # noqa: E731

    def _fwd(e):
        b = wm.linattn(e["q"], e["k"], e["v"], e["decay"], 0.3, h0=e["h0"], resets=e["resets"], lengths=e["lengths"])
        return b.y, b.h_T

    eps = 2.0 ** -3
    for n, gn in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("h0", "dh0")):
        v = rng.standard_normal(x[n].shape).astype(np.float32)
        up, down = (loss({**d, n: d[n] + s * eps * dev(v)}) for s in (1.0, -1.0))
        slope = sum(float((a - b).sum()) for a, b in zip(up, down)) / (2 * eps)
        # linear in each input: no term but the outputs' roundings (bounds of y and h_T), and that of
        # the moved input, 2 u of it, which the bounds' own operations include
        r = attend.linattn(x["q"], x["k"], x["v"], x["decay"], 0.3, x["h0"], x["resets"], x["lengths"])
        grow = 1 + eps * np.abs(v).max() * 4  # magnitudes at the moved input, entry by entry at most
        tol = grow * (float((r["y_err"] * np.abs(x["dy"])).sum()) + float((r["h_T_err"] * np.abs(x["dh_T"])).sum())) / eps
        assert abs(slope - float((host(getattr(bufs, gn)) * v).sum())) <= 2 * tol, n


@pytest.mark.parametrize("T,B,N,K,V,dtype", [(1, 5, 2, 64, 64, "fp32"), (90, 4, 2, 64, 64, "bf16"), (700, 2, 2, 40, 64, "fp32")])
def test_graph_and_streams(T, B, N, K, V, dtype):
    x = _make(T, B, N, K, V, dtype, True)
    d = _device(x, dtype)
    bufs, eager = (wm.LinattnBuffers(T, B, N, K, V, TORCH[dtype]) for _ in range(2))
    names = ("y", "h_T", "dq", "dk", "dv", "dh0")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        _run(d, bufs, 0.2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        _run(d, bufs, 0.2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(4):
        for n in ("q", "k", "v", "dy", "h0", "dh_T"):
            d[n].normal_(generator=gen)
        _run(d, eager, 0.2)
        for n in names:
            getattr(bufs, n).zero_()
        torch.cuda.synchronize()
        graph.replay()
        # eager work with its own buffers beside the replay
        _run(d, eager, 0.2)
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(getattr(bufs, n), getattr(eager, n)), (i, n)


def test_nothing_to_do():
    e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    decay = torch.ones(2, device="cuda")
    h0 = torch.randn(3, 2, 8, 4, device="cuda")
    q, v = e(0, 3, 2, 8), e(0, 3, 2, 4)
    bufs = wm.LinattnBuffers(0, 3, 2, 8, 4)
    wm.linattn(q, q, v, decay, h0=h0, bufs=bufs)
    wm.linattn_grad(q, q, v, decay, v, dh_T=h0, bufs=bufs)
    assert torch.equal(bufs.h_T, h0) and torch.equal(bufs.dh0, h0)
    bufs = wm.LinattnBuffers(5, 0, 2, 8, 4)
    wm.linattn(e(5, 0, 2, 8), e(5, 0, 2, 8), e(5, 0, 2, 4), decay, bufs=bufs)
    wm.linattn_grad(e(5, 0, 2, 8), e(5, 0, 2, 8), e(5, 0, 2, 4), decay, e(5, 0, 2, 4), bufs=bufs)


def test_buffers_of_another_shape():
    """Arrays that a caller puts in the place of the buffers' own."""
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    q, v, decay = z(4, 2, 3, 8), z(4, 2, 3, 5), z(3)
    for name, t in (("y", z(3, 2, 3, 5)), ("y", z(4, 2, 3, 5).bfloat16()), ("y", z(4, 2, 3, 10)[..., :5]), ("h_T", z(2, 3, 5, 8)),
                    ("h_T", z(1, 3, 8, 5)), ("h_T", z(2, 3, 8, 5).double()), ("dh0", z(2, 3, 5, 8)), ("dh0", z(2, 3, 8, 10)[..., :5]),
                    ("dq", z(3, 2, 3, 8)), ("dk", z(4, 2, 3, 5)), ("dv", z(4, 2, 3, 8))):
        bufs = wm.LinattnBuffers(4, 2, 3, 8, 5)
        setattr(bufs, name, t)
        with pytest.raises(ValueError):
            wm.linattn(q, q, v, decay, bufs=bufs)
            wm.linattn_grad(q, q, v, decay, v, bufs=bufs)


def test_refusals():
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    q, v, decay = z(4, 2, 3, 8), z(4, 2, 3, 5), z(3)
    ok = dict(q=q, k=q, v=v, decay=decay)
    for bad in (dict(q=q.double()), dict(k=q.bfloat16()), dict(k=q[:, :, :2]), dict(v=v[:3]), dict(decay=z(2)),
                dict(decay=decay.double()), dict(h0=z(2, 3, 5, 8)), dict(resets=torch.zeros(4, 2, device="cuda")),
                dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(q=q[0]),
                dict(q=z(4, 2, 3, 16)[..., :8]), dict(q=z(4, 2, 8, 3).transpose(2, 3)),
                dict(bufs=wm.LinattnBuffers(4, 2, 3, 8, 6))):
        with pytest.raises(ValueError):
            wm.linattn(**{**ok, **bad})
    with pytest.raises(ValueError):
        wm.linattn_grad(**ok, dy=v, bufs=wm.LinattnBuffers(4, 2, 3, 8, 5, grad=False))
    with pytest.raises(ValueError):
        wm.linattn_grad(**ok, dy=v)
    with pytest.raises(ValueError):
        wm.linattn_grad(**ok, dy=q, bufs=wm.LinattnBuffers(4, 2, 3, 8, 5))
    with pytest.raises(wm.WmError) as e:
        wm.linattn(z(2, 1, 1, 129), z(2, 1, 1, 129), z(2, 1, 1, 4), z(1))
    assert e.value.status == wm.WM_ERR_UNSUPPORTED
    with pytest.raises(wm.WmError):
        wm.linattn(**ok, scale=float("nan"))
    bufs = wm.LinattnBuffers(600, 1, 1, 8, 8)
    bufs.ws_bytes -= 1
    long = z(600, 1, 1, 8)
    with pytest.raises(wm.WmError) as e:
        wm.linattn_grad(long, long, long, z(1), long, bufs=bufs)
    assert e.value.status == wm.WM_ERR_WORKSPACE
    bufs = wm.LinattnBuffers(600, 1, 1, 8, 8)
    bufs.states_bytes -= 1
    for f in (lambda: wm.linattn(long, long, long, z(1), bufs=bufs), lambda: wm.linattn_grad(long, long, long, z(1), long, bufs=bufs)):
        with pytest.raises(wm.WmError) as e:
            f()
        assert e.value.status == wm.WM_ERR_WORKSPACE
