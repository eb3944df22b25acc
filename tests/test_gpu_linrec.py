"""GPU tests of the gated linear recurrence and its gradient (wm_linrec,
wm_linrec_grad): every value against the oracle within the bound that follows
the recurrence, from one step to tens of thousands, odd widths, strided
halves, resets, lengths of zero, values that masks must keep out, chunks that
continue each other."""

import numpy as np
import pytest
import torch

from oracle import seq
from paper_2205_01435_amd import _lib as wm
from seqcheck import TORCH, dev, guarded, host, rounded, say, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


def _inputs(T, B, H, dtype, masks, seed, packed=False):
    rng = np.random.default_rng(seed)
    xg = rounded(rng, (T, B, 2 * H), dtype)
    xg[..., H:] = host(dev(xg[..., H:] + 2, dtype))
    x, g = xg[..., :H], xg[..., H:]
    d = dict(x=x, gate=g, dy=rounded(rng, (T, B, H), dtype), h0=rounded(rng, (B, H), "fp32"),
             dh_T=rounded(rng, (B, H), "fp32"), resets=None, lengths=None)
    if masks:
        d["resets"] = (rng.random((T, B)) < min(0.5, 3.0 / max(T, 1))).astype(np.uint8)
        d["resets"][:, B // 2] = 255  # a row that starts anew at every step
        d["lengths"] = rng.integers(-1, T + 2, B).astype(np.int32)
        d["lengths"][0] = 0
    if packed:
        X = dev(xg, dtype)
        t = dict(x=X[..., :H], gate=X[..., H:])
    else:
        t = dict(x=dev(x, dtype), gate=dev(g, dtype))
    t.update(dy=dev(d["dy"], dtype), h0=dev(d["h0"].astype(np.float32)), dh_T=dev(d["dh_T"].astype(np.float32)),
             resets=None if d["resets"] is None else dev(d["resets"]),
             lengths=None if d["lengths"] is None else dev(d["lengths"]))
    return d, t


def _bufs(T, B, H, dtype):
    b = wm.LinrecBuffers(T, B, H, TORCH[dtype])
    checks = []
    for k, shape, dt in (("y", (T, B, H), TORCH[dtype]), ("dxg", (T, B, 2 * H), TORCH[dtype]),
                         ("h_T", (B, H), torch.float32), ("dh0", (B, H), torch.float32)):
        t, c = guarded(shape, dt)
        setattr(b, k, t)
        checks.append((k, c))
    b.dx, b.dgate = b.dxg[..., :H], b.dxg[..., H:]
    b.workspace.fill_(255)
    b.states.fill_(255)
    return b, lambda: [c(k) for k, c in checks]


def _run(t, bufs):
    wm.linrec(t["x"], t["gate"], t["h0"], t["resets"], t["lengths"], bufs=bufs)
    wm.linrec_grad(t["x"], t["gate"], t["dy"], t["dh_T"], t["resets"], t["lengths"], bufs=bufs)


def _compare(d, bufs, dtype):
    f = seq.linrec(d["x"], d["gate"], d["h0"], d["resets"], d["lengths"])
    within(host(bufs.y), f["y"], f["y_err"], dtype, "y")
    within(host(bufs.h_T), f["h_T"], f["h_T_err"], "fp32", "h_T")
    o = seq.linrec_grad(d["x"], d["gate"], d["dy"], d["dh_T"], d["h0"], d["resets"], d["lengths"])
    within(host(bufs.dx), o["dx"], o["dx_err"], dtype, "dx")
    within(host(bufs.dgate), o["dgate"], o["dgate_err"], dtype, "dgate")
    within(host(bufs.dh0), o["dh0"], o["dh0_err"], "fp32", "dh0")


CASES = [  # T, B, H, dtype, masks, packed
    (1, 1, 1, "fp32", False, False), (1, 3, 7, "bf16", True, False), (1, 256, 512, "fp32", True, True),
    (2, 5, 64, "bf16", False, True), (8, 2, 130, "fp32", True, False), (15, 3, 33, "bf16", True, False),
    (16, 4, 64, "fp32", False, False), (17, 2, 65, "fp32", True, True), (31, 1, 367, "bf16", True, False),
    (45, 100, 36, "bf16", True, False), (64, 70, 2, "fp32", True, False), (100, 9, 1, "bf16", True, True),
    (127, 2, 96, "fp32", True, True), (128, 8, 64, "bf16", False, True), (129, 2, 50, "bf16", True, False),
    (255, 1, 64, "fp32", False, False), (257, 3, 24, "fp32", True, False), (300, 130, 3, "bf16", True, True),
    (513, 1, 31, "bf16", True, True), (1000, 2, 40, "fp32", True, True), (2048, 1, 66, "bf16", False, True),
    (4099, 2, 10, "fp32", True, False), (20000, 1, 5, "fp32", False, False), (33000, 1, 2, "bf16", True, True),
    (70001, 1, 2, "fp32", True, False),
]


@pytest.mark.parametrize("T,B,H,dtype,masks,packed", CASES)
def test_linrec_and_gradient(T, B, H, dtype, masks, packed):
    say("linrec", T, B, H, dtype, masks, packed)
    d, t = _inputs(T, B, H, dtype, masks, T + B + H, packed)
    bufs, check = _bufs(T, B, H, dtype)
    _run(t, bufs)
    check()
    _compare(d, bufs, dtype)
    got = [v.clone() for v in (bufs.y, bufs.h_T, bufs.dxg, bufs.dh0)]
    _run(t, bufs)  # the same bits again, on a workspace that has been used
    assert all(torch.equal(p, q) for p, q in zip(got, (bufs.y, bufs.h_T, bufs.dxg, bufs.dh0)))


@pytest.mark.parametrize("T,B,H,dtype,packed", [  # (the masks take one row's steps and start another's anew at each)
    (8, 4, 130, "fp32", False), (17, 4, 65, "fp32", True), (31, 5, 367, "bf16", False), (127, 6, 96, "fp32", True),
    (513, 4, 31, "bf16", True), (1000, 4, 40, "fp32", True), (2049, 3, 70, "bf16", False), (4099, 5, 10, "fp32", False),
    (20000, 3, 5, "bf16", True)])
def test_masks_on_several_rows(T, B, H, dtype, packed):
    test_linrec_and_gradient(T, B, H, dtype, True, packed)


@pytest.mark.parametrize("T,B,H,dtype,masks,packed", [  # one tile, few channels and many
    (2, 1, 1, "fp32", False, False), (2, 1700, 64, "bf16", True, True), (3, 100, 1000, "fp32", True, False),
    (15, 140, 1024, "bf16", False, True), (16, 2100, 65, "bf16", True, False), (16, 1600, 64, "fp32", False, False)])
def test_a_single_tile(T, B, H, dtype, masks, packed):
    test_linrec_and_gradient(T, B, H, dtype, masks, packed)


def test_more_steps_than_one_launch_takes():
    test_linrec_and_gradient(140001, 3, 1, "bf16", True, False)


@pytest.mark.parametrize("T,B,H,dtype,masks,packed", [  # around the longest single segment
    (129, 70, 3, "bf16", True, False), (144, 3, 66, "fp32", True, True), (145, 2, 64, "bf16", False, True),
    (200, 5, 100, "fp32", True, False), (241, 1, 130, "bf16", True, True), (256, 3, 130, "bf16", True, False),
    (256, 2, 64, "fp32", False, True), (257, 2, 64, "bf16", False, False), (272, 3, 70, "fp32", True, True)])
def test_one_segment_or_several(T, B, H, dtype, masks, packed):
    test_linrec_and_gradient(T, B, H, dtype, masks, packed)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_without_state_and_optional_arrays(dtype):
    d, t = _inputs(70, 3, 20, dtype, False, 1)
    bufs = wm.LinrecBuffers(70, 3, 20, TORCH[dtype])
    wm.linrec(t["x"], t["gate"], bufs=bufs)
    wm.linrec_grad(t["x"], t["gate"], t["dy"], bufs=bufs)
    _compare(dict(d, h0=np.zeros((3, 20)), dh_T=np.zeros((3, 20))), bufs, dtype)
    only = wm.linrec(t["x"], t["gate"], bufs=wm.LinrecBuffers(70, 3, 20, TORCH[dtype], grad=False))
    assert torch.equal(only.y, bufs.y) and torch.equal(only.h_T, bufs.h_T)


@pytest.mark.parametrize("T", [1, 40, 700])
def test_batch_major_views(T):
    """[B, T, H] data through transposed views, dx and dgate included."""
    B, H = 5, 34
    d, t = _inputs(T, B, H, "fp32", True, 3)
    bm = {k: t[k].transpose(0, 1).contiguous().transpose(0, 1) for k in ("x", "gate", "dy")}
    bufs = wm.LinrecBuffers(T, B, H)
    whole = torch.zeros(B, T, 2 * H, device="cuda")
    bufs.dxg = whole.transpose(0, 1)
    bufs.dx, bufs.dgate = bufs.dxg[..., :H], bufs.dxg[..., H:]
    _run(dict(t, **bm), bufs)
    _compare(d, bufs, "fp32")


def test_one_gate_for_all_steps_and_rows():
    """Broadcast inputs: strides of 0 (their gradient is the caller's sum)."""
    T, B, H = 50, 4, 24
    d, t = _inputs(T, B, H, "fp32", False, 4)
    g = t["gate"][:1, :1].expand(T, B, H)
    bufs = wm.LinrecBuffers(T, B, H)
    _run(dict(t, gate=g), bufs)
    _compare(dict(d, gate=np.broadcast_to(d["gate"][:1, :1], (T, B, H))), bufs, "fp32")


@pytest.mark.parametrize("T", [20, 600])
def test_masked_places_may_hold_anything(T):
    B, H = 4, 18
    d, t = _inputs(T, B, H, "fp32", False, 5)
    lengths = np.array([T, T // 2, 0, T - 1], np.int32)
    resets = np.zeros((T, B), np.uint8)
    resets[T // 3, 0], resets[0, 3], resets[T // 2 + 1, 1] = 1, 1, 1  # the last lies in padding
    d.update(lengths=lengths, resets=resets)
    t.update(lengths=dev(lengths), resets=dev(resets))
    clean, _ = _bufs(T, B, H, "fp32")
    _run(t, clean)
    _compare(d, clean, "fp32")
    pad = torch.arange(T, device="cuda")[:, None] >= t["lengths"][None, :]
    dirty = dict(t)
    for k, v in (("x", float("nan")), ("gate", float("inf")), ("dy", float("-inf"))):
        dirty[k] = t[k].masked_fill(pad[..., None], v)
    dirty["h0"] = t["h0"].clone()
    dirty["h0"][3] = float("nan")  # step 0 of row 3 starts anew
    got, _ = _bufs(T, B, H, "fp32")
    _run(dirty, got)
    for k in ("y", "h_T", "dxg", "dh0"):
        assert torch.equal(getattr(got, k), getattr(clean, k)), k
    # an infinity in the trajectory before a reset ends there, both ways
    x = t["x"].clone()
    x[T // 3 - 1, 0] = float("inf")
    got2, _ = _bufs(T, B, H, "fp32")
    _run(dict(t, x=x), got2)
    assert torch.equal(got2.y[T // 3:], clean.y[T // 3:])
    assert not bool(torch.isfinite(got2.y[T // 3 - 1, 0]).any())
    dy = t["dy"].clone()
    dy[T // 3, 0] = float("nan")
    got3, _ = _bufs(T, B, H, "fp32")
    _run(dict(t, dy=dy), got3)
    assert torch.equal(got3.dxg[:T // 3], clean.dxg[:T // 3]) and torch.equal(got3.dh0, clean.dh0)


def test_a_nan_stays_to_the_end_of_its_trajectory():
    T, B, H = 900, 1, 70
    d, t = _inputs(T, B, H, "fp32", False, 6)
    x = t["x"].clone()
    x[10, 0, 5] = float("nan")
    y = wm.linrec(x, t["gate"], t["h0"]).y
    nan = torch.isnan(y)
    assert bool(nan[10:, 0, 5].all()) and int(nan.sum()) == T - 10


@pytest.mark.parametrize("T", [12, 40])
@pytest.mark.parametrize("gate", [float("-inf"), float("inf"), -200.0, 200.0, -88.0, -0.0, 0.0, -3.4028234e38])
def test_extreme_gates(gate, T):
    B, H = 2, 16
    d, t = _inputs(T, B, H, "fp32", False, 7)
    d["gate"] = np.full((T, B, H), gate)
    t["gate"] = torch.full((T, B, H), gate, device="cuda")
    bufs = wm.LinrecBuffers(T, B, H)
    _run(t, bufs)
    _compare(d, bufs, "fp32")


@pytest.mark.parametrize("dtype,masks,packed", [("fp32", True, True), ("bf16", True, False), ("bf16", False, True)])
def test_many_channels(dtype, masks, packed):
    """Enough channels that a wave takes all steps of its own: rows that share
    a wave (H 437), several tiles, a last one that is short."""
    T, B, H = 50, 301, 437
    d, t = _inputs(T, B, H, dtype, masks, 13, packed)
    bufs, check = _bufs(T, B, H, dtype)
    _run(t, bufs)
    check()
    _compare(d, bufs, dtype)


def test_many_rows_of_one_channel():
    T, B, H = 35, 131073, 1
    d, t = _inputs(T, B, H, "fp32", True, 14)
    bufs, check = _bufs(T, B, H, "fp32")
    _run(t, bufs)
    check()
    _compare(d, bufs, "fp32")


def test_masked_places_may_hold_anything_where_a_wave_takes_all_steps():
    T, B, H = 40, 600, 256
    _, t = _inputs(T, B, H, "fp32", True, 15)
    clean, _ = _bufs(T, B, H, "fp32")
    _run(t, clean)
    pad = torch.arange(T, device="cuda")[:, None] >= t["lengths"][None, :]
    dirty = {k: (t[k].masked_fill(pad[..., None], v) if k in ("x", "gate", "dy") else t[k])
             for k, v in (("x", float("nan")), ("gate", float("inf")), ("dy", float("nan")), ("h0", 0), ("dh_T", 0),
                          ("resets", 0), ("lengths", 0))}
    first = (t["resets"][0] != 0) & (t["lengths"] > 0)
    dirty["h0"] = t["h0"].masked_fill(first[:, None], float("nan"))
    got, _ = _bufs(T, B, H, "fp32")
    _run(dirty, got)
    assert bool(first.any())
    for k in ("y", "h_T", "dxg", "dh0"):
        assert torch.equal(getattr(got, k), getattr(clean, k)), k


@pytest.mark.parametrize("T,B,H,dtype", [(64, 600, 1024, "fp32"), (3000, 24, 1024, "bf16")])
def test_outputs_larger_than_the_cache(T, B, H, dtype):
    """The rows of a large call are those of two halves, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32).to(TORCH[dtype])  # noqa: E731
    t = dict(x=r(T, B, H), gate=r(T, B, H) + 2, dy=r(T, B, H), h0=torch.randn(B, H, generator=g, device="cuda"),
             dh_T=torch.randn(B, H, generator=g, device="cuda"),
             resets=(torch.rand(T, B, generator=g, device="cuda") < 0.02).to(torch.uint8),
             lengths=torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32))
    whole = wm.LinrecBuffers(T, B, H, TORCH[dtype])
    _run(t, whole)
    for lo, hi in ((0, B // 2), (B // 2, B)):
        cut = {k: v[:, lo:hi].contiguous() if v.dim() > 1 and v.shape[0] == T and v.shape[1] == B else v[lo:hi].contiguous()
               for k, v in t.items()}
        part = wm.LinrecBuffers(T, hi - lo, H, TORCH[dtype])
        _run(cut, part)
        assert torch.equal(whole.y[:, lo:hi], part.y) and torch.equal(whole.dxg[:, lo:hi], part.dxg)
        assert torch.equal(whole.h_T[lo:hi], part.h_T) and torch.equal(whole.dh0[lo:hi], part.dh0)


def test_steps_continue_a_sequence():
    T, B, H = 37, 6, 48
    d, t = _inputs(T, B, H, "fp32", False, 8)
    d["resets"] = (np.random.default_rng(8).random((T, B)) < 0.1).astype(np.uint8)
    r = dev(d["resets"])
    f = seq.linrec(d["x"], d["gate"], d["h0"], d["resets"])
    step = wm.LinrecBuffers(1, B, H, grad=False)
    h = t["h0"]
    for i in range(T):
        wm.linrec(t["x"][i:i + 1], t["gate"][i:i + 1], h, r[i:i + 1], bufs=step)
        h = step.h_T  # the state in place
        within(host(step.y[0]), f["y"][i], f["y_err"][i], "fp32", f"step {i}")
    within(host(h), f["h_T"], f["h_T_err"], "fp32", "h_T")


@pytest.mark.parametrize("T", [5, 200, 900, 131500])
def test_state_and_its_gradient_in_place(T):
    d, t = _inputs(T, 2, 40, "fp32", True, 9)
    bufs = wm.LinrecBuffers(T, 2, 40)
    bufs.h_T.copy_(t["h0"])
    bufs.dh0.copy_(t["dh_T"])
    wm.linrec(t["x"], t["gate"], bufs.h_T, t["resets"], t["lengths"], bufs=bufs)
    wm.linrec_grad(t["x"], t["gate"], t["dy"], bufs.dh0, t["resets"], t["lengths"], bufs=bufs)
    _compare(d, bufs, "fp32")


def test_no_steps_and_no_rows():
    h0 = torch.randn(3, 8, device="cuda")
    e = torch.empty(0, 3, 8, device="cuda")
    bufs = wm.LinrecBuffers(0, 3, 8)
    wm.linrec(e, e, h0, bufs=bufs)
    wm.linrec_grad(e, e, e, h0, bufs=bufs)
    assert torch.equal(bufs.h_T, h0) and torch.equal(bufs.dh0, h0)
    e = torch.empty(4, 0, 8, device="cuda")
    bufs = wm.LinrecBuffers(4, 0, 8)
    wm.linrec(e, e, bufs=bufs)
    wm.linrec_grad(e, e, e, bufs=bufs)


def test_gradient_against_differences():
    T, B, H, eps = 60, 2, 20, 2.0 ** -6
    d, t = _inputs(T, B, H, "fp32", True, 10)
    rng = np.random.default_rng(11)
    v = {k: rng.standard_normal(d[k].shape) for k in ("x", "gate", "h0")}

    def loss(s):
        p = {k: dev((d[k] + s * v[k]).astype(np.float32)) for k in v}
        b = wm.linrec(p["x"], p["gate"], p["h0"], t["resets"], t["lengths"])
        return float((host(b.y) * d["dy"]).sum() + (host(b.h_T) * d["dh_T"]).sum())

    bufs = wm.LinrecBuffers(T, B, H)
    _run(t, bufs)
    slope = (loss(eps) - loss(-eps)) / (2 * eps)
    got = sum(float((host(g) * v[k]).sum()) for k, g in (("x", bufs.dx), ("gate", bufs.dgate), ("h0", bufs.dh0)))
    # roundings of inputs and outputs over 2 eps; the third-order term over a memory of ten steps
    f = seq.linrec(d["x"], d["gate"], d["h0"], d["resets"], d["lengths"])
    size = np.abs(f["y"] * d["dy"]).sum() + np.abs(f["h_T"] * d["dh_T"]).sum()
    assert abs(slope - got) <= 60 * seq.U32 * size / eps + 20 * eps ** 2 * np.abs(d["dy"]).sum() / 6


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_status_of_the_workspace(dtype):
    """Calls whose time axis is split over work-groups and not, in a workspace of any contents."""
    for T, B, H in ((300, 2, 70), (300, 410, 256), (300, 520, 256)):
        x, gate = torch.ones(T, B, H, device="cuda").to(TORCH[dtype]), torch.zeros(T, B, H, device="cuda").to(TORCH[dtype])
        bufs = wm.LinrecBuffers(T, B, H, TORCH[dtype])
        if not bufs.ws_bytes:  # enough channels for either type
            continue
        bufs.workspace.fill_(255)
        wm.linrec(x, gate, bufs=bufs)
        wm.status(bufs)
        bufs.workspace.fill_(255)
        wm.linrec_grad(x, gate, x, bufs=bufs)
        wm.status(bufs)


def test_two_streams_at_once():
    """Calls whose work-groups wait for each other's maps share the device with each other and with
    products that fill it: the same bits, and no wait at its bound."""
    T, B, H = 5000, 1, 640
    sets = [_inputs(T, B, H, "bf16", False, 30 + i)[1] for i in range(2)]
    alone = [wm.LinrecBuffers(T, B, H, torch.bfloat16) for _ in sets]
    for t, b in zip(sets, alone):
        _run(t, b)
    both = [wm.LinrecBuffers(T, B, H, torch.bfloat16) for _ in sets]
    streams = [torch.cuda.Stream() for _ in range(3)]
    m = torch.randn(4096, 4096, device="cuda").bfloat16()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(streams[2]):
            for _ in range(3):
                m @ m
        for t, b, s in zip(sets, both, streams):
            with torch.cuda.stream(s):
                _run(t, b)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        wm.status(b)
        for k in ("y", "h_T", "dxg", "dh0"):
            assert torch.equal(getattr(a, k), getattr(b, k)), k


def test_under_a_graph():
    """Captured once, replayed with new inputs, eager work in between."""
    T, B, H = 700, 1, 64
    d, t = _inputs(T, B, H, "bf16", False, 12)
    bufs = wm.LinrecBuffers(T, B, H, torch.bfloat16)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        _run(t, bufs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        _run(t, bufs)
    for i in range(4):
        new, nt = _inputs(T, B, H, "bf16", False, 20 + i)
        for k in ("x", "gate", "dy", "h0", "dh_T"):
            t[k].copy_(nt[k])
        eager = wm.LinrecBuffers(T, B, H, torch.bfloat16)
        _run(nt, eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in ("y", "h_T", "dxg", "dh0"):
            assert torch.equal(getattr(bufs, k), getattr(eager, k)), (i, k)


def test_refusals():
    x = torch.zeros(4, 2, 8, device="cuda")
    with pytest.raises(ValueError):
        wm.linrec(x, x[:3])
    with pytest.raises(ValueError):
        wm.linrec(x, x.bfloat16())
    with pytest.raises(ValueError):
        wm.linrec(x, x, h0=torch.zeros(2, 8, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        wm.linrec(x, x, resets=torch.zeros(4, 3, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        wm.linrec(x, x, lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        wm.linrec(x.transpose(1, 2).contiguous().transpose(1, 2), x)
    with pytest.raises(ValueError):
        wm.linrec(x, x, bufs=wm.LinrecBuffers(4, 2, 9))
    with pytest.raises(ValueError):
        wm.linrec_grad(x, x, x, bufs=wm.LinrecBuffers(4, 2, 8, grad=False))
    b = wm.LinrecBuffers(4, 2, 8)
    b.dx = b.dxg[:1, :, :8].expand(4, 2, 8)  # overlapping output rows
    with pytest.raises(wm.WmError) as e:
        wm.linrec_grad(x, x, x, bufs=b)
    assert e.value.status == wm.WM_ERR_INVALID_ARG
    b = wm.LinrecBuffers(4000, 2, 8)
    b.ws_bytes = 0
    z = torch.zeros(4000, 2, 8, device="cuda")
    with pytest.raises(wm.WmError) as e:
        wm.linrec(z, z, bufs=b)
    assert e.value.status == wm.WM_ERR_WORKSPACE
