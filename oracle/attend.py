"""The attending-core operators in plain float64 numpy: the norm and rotation of
queries and keys, linear attention with one decay a head, the gated projection,
and their gradients, each from its definition.  Every function also gives what a
computation in float32 may be off, element by element, to first order (``*_err``);
the derivations stand at each."""

import math

import numpy as np

from .seq import U16, U32, _live

# --- norm and rotation of queries and keys -------------------------------------


def frequencies(R, base):
    return np.array([base ** (-2.0 * i / R) for i in range(R // 2)])


def _pairs(R, neighbours):
    i = np.arange(R // 2)
    return (2 * i, 2 * i + 1) if neighbours else (i, i + R // 2)


def rotate(v, positions, R, base, neighbours, sign=1.0):
    """v [rows, heads, D] with its pairs turned, and |first| + |second| of each
    pair in both places (what an error of a sine or cosine multiplies)."""
    out, mag = v.copy(), np.abs(v)
    if R:
        a, b = _pairs(R, neighbours)
        ang = sign * np.asarray(positions, np.float64)[:, None, None] * frequencies(R, base)
        c, s = np.cos(ang), np.sin(ang)
        out[..., a] = v[..., a] * c - v[..., b] * s
        out[..., b] = v[..., a] * s + v[..., b] * c
        mag[..., a] = mag[..., b] = np.abs(v[..., a]) + np.abs(v[..., b])
    return out, mag


def qk_norm(x, positions, gamma, eps, R, base, neighbours):
    """(y, bound).  The mean square is a sum of at most 16 terms in a lane and six
    levels over lanes (22 u, half of it in r), r itself a root and a quotient (4 u),
    two products (2 u), sine and cosine 4 u absolute, the turn 2 u."""
    x = x.astype(np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r * (1.0 if gamma is None else gamma.astype(np.float64))
    y, mag = rotate(n, positions, R, base, neighbours)
    # a double's own angle at far positions: half a unit in its last place
    far = np.abs(np.asarray(positions, np.float64))[:, None, None] * 2.0 ** -52
    return y, (24 * U32 + far) * mag


def qk_norm_grad(x, dy, positions, gamma, eps, R, base, neighbours):
    """dict(dx, dgamma, *_err): 6 u of a pair's magnitudes in d; r cubed, the sum over
    the head and the products around it within 64 u of the magnitudes they add; the
    weights' gradient adds rows x heads terms in some order."""
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    g = 1.0 if gamma is None else np.abs(gamma.astype(np.float64))
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh = x * r
    d, mag = rotate(dy, positions, R, base, neighbours, -1.0)
    e = d if gamma is None else d * gamma.astype(np.float64)
    dx = r * (e - xh * (e * xh).mean(-1, keepdims=True))
    far = np.abs(np.asarray(positions, np.float64))[:, None, None] * 2.0 ** -52
    m = mag * g
    n = x.shape[0] * x.shape[1]
    return dict(dx=dx, dx_err=(64 * U32 + far) * r * (m + np.abs(xh) * (m * np.abs(xh)).mean(-1, keepdims=True)),
                dgamma=(d * xh).sum((0, 1)), dgamma_err=(((n + 56) * U32 + far) * mag * np.abs(xh)).sum((0, 1)))


# --- linear attention -----------------------------------------------------------


def _scan(q, k, v, decay, scale, h0, resets, lengths):
    """y [T, B, N, V], the states after each step [T, B, N, K, V] and the last."""
    T, B, N, K = q.shape
    V = v.shape[-1]
    S = np.zeros((B, N, K, V)) if h0 is None else h0.astype(np.float64).copy()
    a = np.clip(decay.astype(np.float64), 0.0, 1.0)[:, None, None]
    live = _live(T, B, lengths)
    y, states = np.zeros((T, B, N, V)), np.zeros((T, B, N, K, V))
    for t in range(T):
        for b in range(B):
            if live[t, b]:
                old = np.zeros((N, K, V)) if resets is not None and resets[t, b] else S[b]
                S[b] = a * old + k[t, b].astype(np.float64)[:, :, None] * v[t, b].astype(np.float64)[:, None, :]
                y[t, b] = scale * np.einsum("nk,nkv->nv", q[t, b].astype(np.float64), S[b])
                states[t, b] = S[b]
    return y, states, S


def _ops(T, W):
    """Roundings on the way of one term: the two products' sums (W and 64 terms) and
    once more those of the state's part (W), a weight a^n = 2^-x within (2 + 1.4 x) u,
    60 u up to x = 40, beyond which it no longer counts, twice; and a factor, a sum
    of 64 terms and another factor for every 64 steps that the state passes."""
    return 2 * W + 64 + 120 + 32 + 8 * (T // 64 + 1)


# bf16 calls hold the weights of a chunk and the state that rows meet as two bf16
# terms each, which leave out 2^-17
def _terms(dtype):
    return 2 * 2.0 ** -17 if dtype == "bf16" else 0.0


def linattn(q, k, v, decay, scale, h0=None, resets=None, lengths=None, dtype="fp32"):
    """dict(y, h_T, *_err): errors relative to the same sums over magnitudes."""
    T, K = q.shape[0], q.shape[-1]
    y, states, S = _scan(q, k, v, decay, scale, h0, resets, lengths)
    ab = [np.abs(z) for z in (q, k, v)]
    ym, _, Sm = _scan(*ab, decay, abs(scale), None if h0 is None else np.abs(h0), resets, lengths)
    c = _ops(T, K) * U32
    return dict(y=y, h_T=S, y_err=(c + _terms(dtype)) * ym, h_T_err=c * Sm, states=states)


def _back(q, k, v, dy, decay, scale, h0, dh_T, resets, lengths):
    T, B, N, K = q.shape
    V = v.shape[-1]
    _, states, _ = _scan(q, k, v, decay, scale, h0, resets, lengths)
    a = np.clip(decay.astype(np.float64), 0.0, 1.0)[:, None, None]
    live = _live(T, B, lengths)
    G = np.zeros((B, N, K, V)) if dh_T is None else dh_T.astype(np.float64).copy()
    dq, dk, dv = np.zeros((T, B, N, K)), np.zeros((T, B, N, K)), np.zeros((T, B, N, V))
    for t in range(T - 1, -1, -1):
        for b in range(B):
            if not live[t, b]:
                continue
            d = dy[t, b].astype(np.float64)
            dq[t, b] = scale * np.einsum("nkv,nv->nk", states[t, b], d)
            F = G[b] + scale * q[t, b].astype(np.float64)[:, :, None] * d[:, None, :]
            dk[t, b] = np.einsum("nkv,nv->nk", F, v[t, b].astype(np.float64))
            dv[t, b] = np.einsum("nkv,nk->nv", F, k[t, b].astype(np.float64))
            G[b] = 0.0 if resets is not None and resets[t, b] else a * F
    return dict(dq=dq, dk=dk, dv=dv, dh0=G)


def linattn_grad(q, k, v, dy, decay, scale, h0=None, dh_T=None, resets=None, lengths=None, dtype="fp32"):
    out = _back(q, k, v, dy, decay, scale, h0, dh_T, resets, lengths)
    mag = _back(*(np.abs(z) for z in (q, k, v, dy)), decay, abs(scale), None if h0 is None else np.abs(h0),
                None if dh_T is None else np.abs(dh_T), resets, lengths)
    c = _ops(q.shape[0], max(q.shape[-1], v.shape[-1])) * U32
    out.update({n + "_err": (c + (0.0 if n == "dh0" else _terms(dtype))) * m for n, m in mag.items()})
    return out


# --- gated projection --------------------------------------------------------------

_erf = np.vectorize(math.erf)


def activation(act, g):
    """(act(g), act'(g))."""
    if act == "silu":
        s = np.where(g >= 0, 1.0, np.exp(-np.abs(g))) / (1.0 + np.exp(-np.abs(g)))
        return g * s, s * (1.0 + g * (1.0 - s))
    p = 0.5 * (1.0 + _erf(g / math.sqrt(2.0)))
    return g * p, p + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def glu(x, W, act):
    """dict(h, h_err, and what the gradient needs): a sum of D products is off by at
    most (D + 1) u of its magnitudes; the activation's slope is at most 1.13 and its
    own error 16 u of |g|, the product's 1 u."""
    x, W = x.astype(np.float64), W.astype(np.float64)
    F, D = W.shape[0] // 2, W.shape[1]
    pre, mag = x @ W.T, (D + 1) * U32 * (np.abs(x) @ np.abs(W).T)
    g, u = pre[:, :F], pre[:, F:]
    a, da = activation(act, g)
    err = (1.13 * mag[:, :F] + 16 * U32 * np.abs(g)) * np.abs(u) + np.abs(a) * mag[:, F:] + U32 * np.abs(a * u)
    return dict(h=a * u, h_err=err, g=g, u=u, a=a, da=da, pre_err=mag)


def glu_grad(x, W, dh, act, dtype="fp32"):
    """dict(dx, dW, *_err): g and u as the forward call saved them (bf16: cut to 16
    significant bits), curvatures of the activation at most 1, dg and du rounded once in bf16, and the
    products' sums over 2F and the rows."""
    f = glu(x, W, act)
    x, W, dh = x.astype(np.float64), W.astype(np.float64), dh.astype(np.float64)
    F = W.shape[0] // 2
    r = U16 if dtype == "bf16" else 0.0
    cut = 2.0 ** -15 if dtype == "bf16" else 0.0
    eg, eu = f["pre_err"][:, :F] + cut * np.abs(f["g"]), f["pre_err"][:, F:] + cut * np.abs(f["u"])
    dg, du = dh * f["u"] * f["da"], dh * f["a"]
    edg = np.abs(dh) * (np.abs(f["u"]) * (eg + 16 * U32) + np.abs(f["da"]) * eu) + (r + 2 * U32) * np.abs(dg)
    edu = np.abs(dh) * (1.13 * eg + 16 * U32 * np.abs(f["g"])) + (r + 2 * U32) * np.abs(du)
    d, e = np.concatenate([dg, du], 1), np.concatenate([edg, edu], 1)
    e = e * (1.0 + r)  # a rounding of what is off already
    return dict(dx=d @ W, dx_err=e @ np.abs(W) + (2 * F + 1) * U32 * (np.abs(d) @ np.abs(W)),
                dW=d.T @ x, dW_err=e.T @ np.abs(x) + (len(x) + 1) * U32 * (np.abs(d).T @ np.abs(x)))
