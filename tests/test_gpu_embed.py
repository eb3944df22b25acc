"""GPU tests of the scaled embedding and its gradient (wm_embed,
wm_embed_grad): every value against the oracle, from one token to tens of
thousands, one table row to the widest action space, odd widths, strided
rows, codes outside the table, and tokens that all name one row."""

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


def _tokens(rng, n, V, how):
    if how == "one":
        return np.full(n, V // 2, np.int32)
    if how == "none":
        return np.where(np.arange(n) % 2, -1, V).astype(np.int32)
    if how == "rising":
        return np.sort(rng.integers(0, V, n)).astype(np.int32)
    t = (V * rng.random(n) ** 2).astype(np.int64)
    return np.where(rng.random(n) < 0.1, rng.choice([-1, -2, V, 2 ** 31 - 1, -2 ** 31], n), t).astype(np.int32)


CASES = [  # n, V, H, dtype, tokens
    (1, 1, 1, "fp32", "any"), (1, 64, 256, "bf16", "any"), (3, 5, 7, "bf16", "any"), (63, 2, 33, "fp32", "any"),
    (64, 64, 64, "bf16", "any"), (65, 300, 96, "fp32", "none"), (1000, 50, 367, "bf16", "any"),
    (1000, 50, 367, "fp32", "any"), (4097, 3, 130, "fp32", "one"), (5000, 257, 65, "bf16", "rising"),
    (20000, 2048, 24, "fp32", "any"), (20000, 2049, 16, "bf16", "any"), (30011, 57600, 8, "fp32", "any"),
    (9000, 70001, 9, "bf16", "any"), (300, 20, 2050, "bf16", "any"), (70000, 17, 5, "fp32", "any"),
    (130, 9, 1024, "bf16", "one"), (33000, 5, 12, "bf16", "one"),
]


@pytest.mark.parametrize("n,V,H,dtype,how", CASES)
def test_embed(n, V, H, dtype, how):
    say("embed", n, V, H, dtype, how)
    rng = np.random.default_rng(n + V + H)
    table, tok, scale = rounded(rng, (V, H), dtype), _tokens(rng, n, V, how), float(np.float32(H ** 0.5))
    out, check = guarded((n, H), TORCH[dtype])
    y = wm.embed(dev(table, dtype), dev(tok), scale, out=out)
    check("embed")
    assert y.data_ptr() == out.data_ptr()
    # one product in fp32, then one rounding: the same bits
    prod = torch.from_numpy(np.float32(scale) * table.astype(np.float32)).to(TORCH[dtype])
    ok = (tok >= 0) & (tok < V)
    ref = torch.where(torch.from_numpy(ok)[:, None], prod[np.where(ok, tok, 0)], torch.zeros((), dtype=TORCH[dtype]))
    assert torch.equal(y.cpu(), ref)


@pytest.mark.parametrize("n,V,H,dtype,how", CASES)
def test_embed_grad(n, V, H, dtype, how):
    say("embed_grad", n, V, H, dtype, how)
    rng = np.random.default_rng(n + V + H + 1)
    dy, tok, scale = rounded(rng, (n, H), dtype), _tokens(rng, n, V, how), float(np.float32(H ** 0.5))
    bufs = wm.EmbedGradBuffers(n, V, H)
    bufs.grad, check = guarded((V, H), torch.float32)
    bufs.workspace.fill_(255)
    ref, bound = seq.embed_grad(tok, dy, V, scale)
    first = None
    for _ in range(2):
        bufs.grad.fill_(float("nan"))  # written whole
        wm.embed_grad(dev(tok), dev(dy, dtype), V, scale, bufs=bufs)
        check("embed_grad")
        within(host(bufs.grad), ref, bound, "fp32", "dtable")
        first = bufs.grad.clone() if first is None else first
    assert torch.equal(first, bufs.grad)  # the order of the sums is fixed


@pytest.mark.parametrize("n,V,H,dtype,how", [
    # one part, parts whose last is short or one position, the most parts; then one more, which sorts
    (512, 40, 300, "bf16", "any"), (513, 40, 300, "fp32", "any"), (7224, 50, 367, "fp32", "one"),
    (7224, 50, 700, "bf16", "any"), (32768, 3, 20, "fp32", "one"), (32768, 16, 1030, "bf16", "any"),
    (32769, 3, 20, "fp32", "one"), (100, 4096, 64, "fp32", "any"), (100, 4097, 64, "fp32", "any"),
    # short lists that are sorted: by one work-group, in one pass and in two
    (4000, 200, 700, "bf16", "any"), (4000, 200, 700, "fp32", "one"), (3000, 900, 300, "fp32", "any"),
    (3000, 900, 300, "bf16", "one"), (4096, 700, 520, "fp32", "rising"), (2500, 800, 600, "fp32", "none"),
])
def test_embed_grad_both_ways(n, V, H, dtype, how):
    test_embed_grad(n, V, H, dtype, how)


@pytest.mark.parametrize("n,V,H,dtype,how", [  # few positions of a large table, and one more than that way takes
    (1, 5000, 64, "fp32", "one"), (2, 9001, 3, "bf16", "any"), (64, 5000, 257, "fp32", "one"),
    (65, 5000, 8, "bf16", "rising"), (511, 4700, 100, "fp32", "any"), (513, 5000, 300, "bf16", "one"),
    (1000, 5003, 367, "fp32", "any"), (1024, 2500, 1024, "bf16", "any"), (1024, 5000, 130, "fp32", "one"),
    (1025, 5000, 130, "fp32", "one"), (700, 5000, 64, "bf16", "none"), (15, 40, 65536, "bf16", "any"),
    (17, 40, 65536, "fp32", "any")])
def test_embed_grad_of_few_positions(n, V, H, dtype, how):
    test_embed_grad(n, V, H, dtype, how)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strided_rows_and_shapes(dtype):
    rng = np.random.default_rng(5)
    T, B, V, H = 6, 35, 11, 50
    tok, wide = _tokens(rng, T * B, V, "any").reshape(T, B), rounded(rng, (T, B, H + 13), dtype)
    table = rounded(rng, (V, H), dtype)
    out = torch.full((T, B, H + 13), 7.0, dtype=TORCH[dtype], device="cuda")
    y = wm.embed(dev(table, dtype), dev(tok), 1.0, out=out[..., :H])
    np.testing.assert_array_equal(host(y), seq.embed(table, tok, 1.0))
    assert bool((out[..., H:] == 7.0).all())
    ref, bound = seq.embed_grad(tok, wide[..., 3:3 + H], V, 0.5)
    g = wm.embed_grad(dev(tok), dev(wide, dtype)[..., 3:3 + H], V, 0.5).grad
    within(host(g), ref, bound, "fp32", "dtable")


def test_no_tokens_and_buffers_of_a_larger_call():
    bufs = wm.EmbedGradBuffers(500, 40, 12)
    bufs.grad.fill_(3.0)
    wm.embed_grad(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 12, device="cuda"), 40, bufs=bufs)
    assert not bool(bufs.grad.any())
    rng = np.random.default_rng(6)
    tok, dy = _tokens(rng, 77, 40, "any"), rounded(rng, (77, 12), "fp32")
    ref, bound = seq.embed_grad(tok, dy, 40, 1.0)
    within(host(wm.embed_grad(dev(tok), dev(dy, "fp32"), 40, bufs=bufs).grad), ref, bound, "fp32", "dtable")


def test_non_finite_rows_stay_with_their_tokens():
    tok = np.array([0, 1, -1, 3, 1], np.int32)
    dy = np.ones((5, 3))
    dy[2], dy[3, 1] = np.nan, np.inf  # a code's row enters nothing
    g = host(wm.embed_grad(dev(tok), dev(dy, "fp32"), 4).grad)
    np.testing.assert_array_equal(g, [[1, 1, 1], [2, 2, 2], [0, 0, 0], [1, np.inf, 1]])
    table = np.ones((2, 3))
    table[0] = np.inf
    np.testing.assert_array_equal(host(wm.embed(dev(table, "fp32"), dev(np.array([-1, 1], np.int32)))),
                                  [[0, 0, 0], [1, 1, 1]])


def test_on_another_stream():
    rng = np.random.default_rng(7)
    tok, dy = _tokens(rng, 3000, 64, "any"), rounded(rng, (3000, 64), "bf16")
    ref, bound = seq.embed_grad(tok, dy, 64, 1.0)
    s = torch.cuda.Stream()
    d, t = dev(dy, "bf16"), dev(tok)
    bufs = wm.EmbedGradBuffers(3000, 64, 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        wm.embed_grad(t, d, 64, bufs=bufs)
    s.synchronize()
    within(host(bufs.grad), ref, bound, "fp32", "dtable")


def test_refusals():
    t = torch.zeros(4, 8, device="cuda")
    tok = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        wm.embed(t, tok.long())
    with pytest.raises(ValueError):
        wm.embed(t.half(), tok)
    with pytest.raises(ValueError):
        wm.embed(t, tok, out=torch.zeros(2, 8, device="cuda"))
    with pytest.raises(ValueError):
        wm.embed(t, tok, out=torch.zeros(3, 8, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        wm.embed(t, tok, out=torch.zeros(8, 3, device="cuda").t())
    with pytest.raises(ValueError):
        wm.embed_grad(tok, torch.zeros(4, 8, device="cuda"), 4)
    with pytest.raises(ValueError):
        wm.embed_grad(tok, torch.zeros(3, 8, device="cuda"), 4, bufs=wm.EmbedGradBuffers(3, 5, 8))
    with pytest.raises(wm.WmError) as e:  # a workspace for fewer tokens
        wm.embed_grad(torch.zeros(200000, dtype=torch.int32, device="cuda"), torch.zeros(200000, 8, device="cuda"), 4,
                      bufs=wm.EmbedGradBuffers(1, 4, 8))
    assert e.value.status == wm.WM_ERR_WORKSPACE
