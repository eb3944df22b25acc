"""Pins of the sequence-core operators' oracle: library routines, closed
forms, and every gradient against central differences of its forward form."""

import numpy as np
import pytest
import torch

from oracle import seq


def _num_grad(f, x, eps=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += eps
        b[i] -= eps
        g[i] = (f(a) - f(b)) / (2 * eps)
    return g


def test_embed_and_its_gradient():
    rng = np.random.default_rng(0)
    table, tok = rng.normal(size=(5, 3)), np.array([[4, -1, 0], [0, 5, 2]])
    y = seq.embed(table, tok, 2.5)
    assert y.shape == (2, 3, 3)
    np.testing.assert_array_equal(y[0, 0], 2.5 * table[4])
    assert not y[0, 1].any() and not y[1, 1].any()
    dy = rng.normal(size=y.shape)
    g, bound = seq.embed_grad(tok, dy, 5, 2.5)
    np.testing.assert_allclose(g, _num_grad(lambda w: (seq.embed(w, tok, 2.5) * dy).sum(), table), atol=1e-8)
    assert not g[1].any() and not bound[3].any() and (bound[0] > 0).all()


@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_is_the_library_routine(affine):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(4, 7)) * 3 + 1
    g, b = (rng.normal(size=7), rng.normal(size=7)) if affine else (None, None)
    t = lambda a: None if a is None else torch.from_numpy(a)  # noqa: E731
    y, _, _ = seq.layer_norm(x, g, b, 1e-5)
    np.testing.assert_allclose(y, torch.nn.functional.layer_norm(t(x), (7,), t(g), t(b), 1e-5).numpy(), atol=1e-12)
    dy = rng.normal(size=x.shape)
    dx, dg, db = seq.layer_norm_grad(x, dy, g, 1e-5)
    np.testing.assert_allclose(dx, _num_grad(lambda v: (seq.layer_norm(v, g, b, 1e-5)[0] * dy).sum(), x), atol=1e-7)
    if affine:
        np.testing.assert_allclose(dg, _num_grad(lambda v: (seq.layer_norm(x, v, b, 1e-5)[0] * dy).sum(), g), atol=1e-7)
        np.testing.assert_allclose(db, _num_grad(lambda v: (seq.layer_norm(x, g, v, 1e-5)[0] * dy).sum(), b), atol=1e-7)


def test_linrec_closed_forms():
    T, B, H = 6, 2, 3
    rng = np.random.default_rng(2)
    x = rng.normal(size=(T, B, H))
    h0 = rng.normal(size=(B, H))
    # a gate of 0 halves: h_T = 2^-T h0 + sum 2^-(T-t) x_t
    f = seq.linrec(x, np.zeros((T, B, H)), h0)
    w = 2.0 ** -np.arange(T, 0, -1)
    np.testing.assert_allclose(f["h_T"], 2.0 ** -T * h0 + np.tensordot(w, x, 1), atol=1e-14)
    # a gate of -inf copies x, one of +inf keeps h0
    np.testing.assert_array_equal(seq.linrec(x, np.full((T, B, H), -np.inf), h0)["y"], x)
    np.testing.assert_array_equal(seq.linrec(x, np.full((T, B, H), np.inf), h0)["h_T"], h0)


def test_linrec_resets_and_lengths():
    T, B, H = 9, 3, 2
    rng = np.random.default_rng(3)
    x, g, h0 = rng.normal(size=(T, B, H)), rng.normal(size=(T, B, H)), rng.normal(size=(B, H))
    resets = np.zeros((T, B), np.uint8)
    resets[4, 1] = 1
    lengths = np.array([9, 7, 0])
    f = seq.linrec(x, g, h0, resets, lengths)
    # each piece alone
    np.testing.assert_allclose(f["y"][:, 0], seq.linrec(x[:, :1], g[:, :1], h0[:1])["y"][:, 0])
    np.testing.assert_allclose(f["y"][:4, 1], seq.linrec(x[:4, 1:2], g[:4, 1:2], h0[1:2])["y"][:, 0])
    tail = seq.linrec(x[4:7, 1:2], g[4:7, 1:2])
    np.testing.assert_allclose(f["y"][4:7, 1], tail["y"][:, 0])
    np.testing.assert_allclose(f["h_T"][1], tail["h_T"][0])
    assert not f["y"][7:, 1].any() and not f["y"][:, 2].any()
    np.testing.assert_array_equal(f["h_T"][2], h0[2])
    # what lies in padding or before a reset does not matter
    x2, g2, h2 = x.copy(), g.copy(), h0.copy()
    x2[7:, 1], g2[:, 2], h2[1] = np.nan, np.inf, np.nan
    x2[3, 1] = np.inf
    f2 = seq.linrec(x2, g2, h2, resets, lengths)
    np.testing.assert_array_equal(f2["y"][4:, 1], f["y"][4:, 1])
    np.testing.assert_array_equal(f2["y"][:, 2], f["y"][:, 2])


@pytest.mark.parametrize("masks", [False, True])
def test_linrec_gradient_against_differences(masks):
    T, B, H = 7, 3, 2
    rng = np.random.default_rng(4)
    x, g, dy = (rng.normal(size=(T, B, H)) for _ in range(3))
    h0, dT = rng.normal(size=(B, H)), rng.normal(size=(B, H))
    resets = (rng.random((T, B)) < 0.3).astype(np.uint8) if masks else None
    lengths = np.array([7, 0, 4]) if masks else None

    def loss(x_, g_, h_):
        f = seq.linrec(x_, g_, h_, resets, lengths)
        return (f["y"] * dy).sum() + (f["h_T"] * dT).sum()

    o = seq.linrec_grad(x, g, dy, dT, h0, resets, lengths)
    np.testing.assert_allclose(o["dx"], _num_grad(lambda v: loss(v, g, h0), x), atol=1e-8)
    np.testing.assert_allclose(o["dgate"], _num_grad(lambda v: loss(x, v, h0), g), atol=1e-8)
    np.testing.assert_allclose(o["dh0"], _num_grad(lambda v: loss(x, g, v), h0), atol=1e-8)


def test_clip():
    grads = [np.array([3.0, 0.0]), np.array([[4.0]]), np.zeros(0)]
    n, f, out = seq.clip(grads, 1.0)
    assert n == 5.0 and f == 0.2
    np.testing.assert_allclose(out[0], [0.6, 0.0])
    assert seq.clip(grads, 5.0)[1] == 1.0 and seq.clip([np.array([np.inf])], 1.0)[1] == 1.0
