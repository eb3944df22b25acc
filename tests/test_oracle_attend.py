"""Pins of the attending-core operators' oracle: closed forms, automatic
differentiation of the same formulas written plainly, and differences."""

import math

import numpy as np
import pytest
import torch

from oracle import attend


def _t(a):
    return torch.from_numpy(np.ascontiguousarray(a)).double().requires_grad_(True)


@pytest.mark.parametrize("neighbours", [0, 1])
@pytest.mark.parametrize("D,R", [(8, 8), (7, 4), (5, 0), (2, 2)])
def test_qk_norm(D, R, neighbours):
    rng = np.random.default_rng(D + R)
    x, dy, g = rng.normal(size=(6, 3, D)), rng.normal(size=(6, 3, D)), rng.normal(size=D)
    pos = np.array([0, 1, -3, 7, 100, 12345])
    y, bound = attend.qk_norm(x, pos, g, 1e-6, R, 100.0, neighbours)
    assert (bound > 0).all()
    X, G = _t(x), _t(g)
    n = X / torch.sqrt((X * X).mean(-1, keepdim=True) + 1e-6) * G
    # a pair as a complex number times e^(i angle)
    out = n.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + R // 2)
        ang = torch.from_numpy(pos * 100.0 ** (-2 * i / R))[:, None]
        z = torch.complex(n[..., a], n[..., b]) * torch.polar(torch.ones_like(ang), ang)
        out[..., a], out[..., b] = z.real, z.imag
    np.testing.assert_allclose(y, out.detach().numpy(), atol=1e-11)
    (out * torch.from_numpy(dy)).sum().backward()
    r = attend.qk_norm_grad(x, dy, pos, g, 1e-6, R, 100.0, neighbours)
    np.testing.assert_allclose(r["dx"], X.grad.numpy(), atol=1e-10)
    np.testing.assert_allclose(r["dgamma"], G.grad.numpy(), atol=1e-9)


def _plain(q, k, v, a, scale, h0, resets, lengths):
    """y_t = scale sum_s a^(t-s) (q_t . k_s) v_s over the steps of t's trajectory, and the
    state's part, without a recurrence."""
    T, B, N, _ = q.shape
    y, h = [[None] * B for _ in range(T)], [None] * B
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        start = -1  # the state's part reaches the steps before the first reset
        for t in range(n):
            if resets is not None and resets[t, b]:
                start = t
            lo = max(start, 0)
            acc = sum(a[:, None] ** (t - s) * (q[t, b] * k[s, b]).sum(-1, keepdim=True) * v[s, b] for s in range(lo, t + 1))
            if start < 0:
                acc = acc + a[:, None] ** (t + 1) * (q[t, b][:, :, None] * h0[b]).sum(1)
            y[t][b] = scale * acc
        for t in range(n, T):
            y[t][b] = torch.zeros_like(v[0, 0])
        lo = max(start, 0)
        h[b] = sum((a[:, None, None] ** (n - 1 - s) * k[s, b][:, :, None] * v[s, b][:, None, :] for s in range(lo, n)),
                   torch.zeros_like(h0[b]))
        if start < 0:
            h[b] = h[b] + a[:, None, None] ** n * h0[b]
    return torch.stack([torch.stack(r) for r in y]), torch.stack(h)


@pytest.mark.parametrize("masks", [False, True])
def test_linattn(masks):
    rng = np.random.default_rng(3)
    T, B, N, K, V = 9, 4, 2, 3, 2
    q, k, v, dy = (rng.normal(size=(T, B, N, w)) for w in (K, K, V, V))
    h0, dh = rng.normal(size=(B, N, K, V)), rng.normal(size=(B, N, K, V))
    a = np.array([0.9, 0.4])
    resets = (rng.random((T, B)) < 0.3) if masks else None
    lengths = np.array([9, 0, 1, 5]) if masks else None
    f = attend.linattn(q, k, v, a, 0.7, h0, resets, lengths)
    ts = [_t(z) for z in (q, k, v, h0)]
    y, h = _plain(*ts[:3], torch.from_numpy(a), 0.7, ts[3], resets, lengths)
    np.testing.assert_allclose(f["y"], y.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(f["h_T"], h.detach().numpy(), atol=1e-12)
    ((y * torch.from_numpy(dy)).sum() + (h * torch.from_numpy(dh)).sum()).backward()
    g = attend.linattn_grad(q, k, v, dy, a, 0.7, h0, dh, resets, lengths)
    for n, t in zip(("dq", "dk", "dv", "dh0"), ts):
        np.testing.assert_allclose(g[n], np.zeros_like(g[n]) if t.grad is None else t.grad.numpy(), atol=1e-12, err_msg=n)


def test_linattn_closed_forms():
    # no decay and one key: the state counts; a decay of 0 forgets all but the step itself
    T = 5
    one = np.ones((T, 1, 2, 1))
    y = attend.linattn(one, one, one, np.array([1.0, 0.0]), 1.0)["y"][:, 0, :, 0]
    np.testing.assert_array_equal(y[:, 0], np.arange(1, T + 1))
    np.testing.assert_array_equal(y[:, 1], np.ones(T))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_glu(act):
    rng = np.random.default_rng(5)
    x, W, dh = rng.normal(size=(7, 5)), rng.normal(size=(8, 5)), rng.normal(size=(7, 4))
    X, Wt = _t(x), _t(W)
    pre = X @ Wt.t()
    f = torch.nn.functional.silu if act == "silu" else torch.nn.functional.gelu
    h = f(pre[:, :4]) * pre[:, 4:]
    np.testing.assert_allclose(attend.glu(x, W, act)["h"], h.detach().numpy(), atol=1e-12)
    (h * torch.from_numpy(dh)).sum().backward()
    g = attend.glu_grad(x, W, dh, act)
    np.testing.assert_allclose(g["dx"], X.grad.numpy(), atol=1e-11)
    np.testing.assert_allclose(g["dW"], Wt.grad.numpy(), atol=1e-11)
    assert (g["dx_err"] > 0).all() and (g["dW_err"] > 0).all()


def test_the_activations_slopes():
    # the bounds of the gradients' errors take a slope of 1.13 and a curvature of 1
    g = np.linspace(-12, 12, 4801)
    for act in ("silu", "gelu"):
        a, da = attend.activation(act, g)
        assert np.abs(da).max() <= 1.13
        assert np.abs(np.diff(da) / np.diff(g)).max() <= 1.0
        assert math.isclose(float(a[2400]), 0.0, abs_tol=1e-12)
