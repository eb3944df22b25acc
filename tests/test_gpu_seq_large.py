"""GPU tests of the sequence-core operators on arrays of more than 2^31 values
(byte offsets beyond 2^32): the places beyond against the same operator on
these places alone, sums against sums in 64 bits."""

import pytest
import torch

from oracle import seq
from paper_2205_01435_amd import _lib as wm
from seqcheck import say

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def memory():
    if torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("needs 64 GB of device memory")
    yield
    torch.cuda.empty_cache()


def _normal(shape, seed):
    return torch.empty(shape, dtype=BF, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed))


def test_embed():
    n, V, H = 2100001, 700, 1030
    say("embed", n, V, H)
    tok = (torch.arange(n, device="cuda") * 7919 % (V + 1) - 1).int()  # a code among them
    table = _normal((V, H), 1)
    out = wm.embed(table, tok)
    for lo in (0, 2 ** 31 // H - 50, n - 100):
        t = tok[lo:lo + 100].long()
        assert torch.equal(out[lo:lo + 100], torch.where((t >= 0)[:, None], table[t.clamp(min=0)], 0))
    out.copy_(out.sign())  # sums of these are exact in fp32
    g = wm.embed_grad(tok, out, V).grad
    ref = torch.zeros(V + 1, H, device="cuda")
    for lo in range(0, n, 300000):
        ref.index_add_(0, tok[lo:lo + 300000].long() + 1, out[lo:lo + 300000].float())
    assert torch.equal(g, ref[1:])


def test_layer_norm():
    rows, H = 2100001, 1030
    say("norm", rows, H)
    x, dy = _normal((rows, H), 2), _normal((rows, H), 3)
    gamma, beta = torch.rand(H, device="cuda"), torch.rand(H, device="cuda")
    b = wm.layer_norm(x, gamma, beta)
    wm.layer_norm_grad(x, dy, gamma, bufs=b)
    for lo in (0, 2 ** 31 // H - 50, rows - 100):
        p = slice(lo, lo + 100)
        a = wm.layer_norm(x[p], gamma, beta)
        wm.layer_norm_grad(x[p], dy[p], gamma, bufs=a)
        for k in ("y", "mean", "rstd", "dx"):
            assert torch.equal(getattr(a, k), getattr(b, k)[p]), (k, lo)
    sums = [torch.zeros(H, dtype=torch.float64, device="cuda") for _ in range(4)]
    for lo in range(0, rows, 100000):
        p = slice(lo, lo + 100000)
        d = dy[p].double()
        v = d * ((x[p].double() - b.mean[p, None].double()) * b.rstd[p, None].double())
        for s, t in zip(sums, (v, d, v.abs(), d.abs())):
            s += t.sum(0)
    # a column's terms, three roundings each, are added along at most as many as one lane's rows
    # (at least 256 work-groups) and the partial sums after them
    m = rows // 256 + 1024 + 4
    for got, ref, mag in ((b.dgamma, sums[0], sums[2]), (b.dbeta, sums[1], sums[3])):
        assert bool(((got.double() - ref).abs() <= m * seq.U32 * mag).all())


def _windows(T, B, H, starts, rows):
    """The whole against windows of 600 steps (the state that enters one is
    forgotten within 200: a product of that many gates below 1/2 on average),
    the first 200 of a window left out going forward, the last ones going back."""
    x, gate, dy = _normal((T, B, H), 4), _normal((T, B, H), 5), _normal((T, B, H), 6)
    b = wm.LinrecBuffers(T, B, H, BF)
    wm.linrec(x, gate, bufs=b)
    wm.linrec_grad(x, gate, dy, bufs=b)
    for t0 in starts:
        p = (slice(t0, min(t0 + 600, T)), rows)
        xs, gs, ds = (t[p].contiguous() for t in (x, gate, dy))
        a = wm.LinrecBuffers(*xs.shape, BF)
        wm.linrec(xs, gs, bufs=a)
        wm.linrec_grad(xs, gs, ds, bufs=a)
        n = xs.shape[0]
        lo, hi = (0 if t0 == 0 else 200), (n if t0 + n == T else n - 200)
        # both are within the fp32 bound of the same value, and rounded once: a bf16 step, or the
        # few fp32 roundings (16 steps' worth, carried states below 8) of values near 0
        for k, f, e in (("y", lo, n), ("dx", 0, hi), ("dgate", lo, hi)):
            u, v = getattr(a, k)[f:e].float(), getattr(b, k)[p][f:e].float()
            assert bool(((u - v).abs() <= 2.0 ** -7 * torch.maximum(u.abs(), v.abs()) + 2.0 ** -14).all()), (k, t0)


def test_linrec_split():
    T, B, H = 36007, 60, 1000
    say("linrec", T, B, H)
    at = 2 ** 31 // (B * H)
    _windows(T, B, H, (0, at - 300, T - 600), slice(B - 3, B))


def test_linrec_walked():
    T, B, H = 1200, 1800, 1000
    say("linrec", T, B, H)
    at = 2 ** 31 // (B * H)
    _windows(T, B, H, (0, at - 550, T - 600), slice(B - 3, B))


@pytest.mark.parametrize("T", [20, 300])
def test_linrec_rows_far_apart(T):
    """Batch-major rows of a longer array, more than 2 GiB from one to the next."""
    B, H, far = 3, 128, (1 << 30) + 640
    say("linrec, rows far apart", T)
    bufs = [torch.empty((B - 1) * far + T * H, dtype=BF, device="cuda") for _ in range(3)]
    views = [b.as_strided((T, B, H), (H, far, 1)) for b in bufs]
    for i, v in enumerate(views):
        v.copy_(_normal((T, B, H), 8 + i))
    near = [v.contiguous() for v in views]
    a, b = wm.LinrecBuffers(T, B, H, BF), wm.LinrecBuffers(T, B, H, BF)
    for q, (x, gate, dy) in ((a, near), (b, views)):
        wm.linrec(x, gate, bufs=q)
        wm.linrec_grad(x, gate, dy, bufs=q)
    for k in ("y", "h_T", "dxg", "dh0"):
        assert torch.equal(getattr(a, k), getattr(b, k)), k
    with pytest.raises(wm.WmError) as e:  # 64 channels of several such rows
        wm.linrec(views[0][..., :100], views[1][..., :100])
    assert e.value.status == wm.WM_ERR_UNSUPPORTED


def test_clip():
    n = 2200000003
    say("clip", n)
    g = _normal((n,), 7)
    h = torch.ones(1001, device="cuda")
    total = 1001.0
    for lo in range(0, n, 1 << 28):
        total += float((g[lo:lo + (1 << 28)].double() ** 2).sum())
    plan = wm.ClipPlan([h, g], [torch.empty_like(h), torch.empty_like(g)])
    norm = float(wm.clip_grads(plan, total ** 0.5 / 2))
    assert abs(norm - total ** 0.5) <= 2 * seq.U32 * total ** 0.5
    for lo in (0, 2 ** 31 - 500, n - 1000):
        a = g[lo:lo + 1000]
        # half of a value is exact; the factor may be off by its rounding, which can move the result's by one step
        assert bool(((plan.outs[1][lo:lo + 1000].float() - a.float() / 2).abs() <= 2.0 ** -8 * a.float().abs()).all())
