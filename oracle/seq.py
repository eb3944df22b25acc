"""The sequence-core operators in plain float64 numpy: scaled embedding, layer
norm, the gated linear recurrence, gradient clipping, and their gradients,
each from its definition.  ``*_bound`` give what a computation with unit
roundoff ``u`` in every operation may be off, element by element, to first
order; the derivations stand at each."""

import numpy as np

U32 = 2.0 ** -24   # unit roundoff of float32
U16 = 2.0 ** -8    # ... of bfloat16


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


# --- embedding --------------------------------------------------------------

def embed(table, tokens, scale):
    out = np.zeros(tokens.shape + (table.shape[1],))
    for i in np.ndindex(tokens.shape):
        if 0 <= tokens[i] < table.shape[0]:
            out[i] = scale * table[tokens[i]].astype(np.float64)
    return out


def embed_grad(tokens, dout, V, scale):
    """(gradient, bound): a sum of m terms in any order is off by at most m u
    times the sum of their magnitudes; one more rounding for the scale."""
    d = dout.reshape(-1, dout.shape[-1]).astype(np.float64)
    g, mag, m = np.zeros((V, d.shape[1])), np.zeros((V, d.shape[1])), np.zeros((V, 1))
    for t, row in zip(tokens.reshape(-1), d):
        if 0 <= t < V:
            g[t] += row
            mag[t] += np.abs(row)
            m[t] += 1
    return scale * g, (m + 2) * U32 * abs(scale) * mag


# --- layer norm ---------------------------------------------------------------

def layer_norm(x, gamma, beta, eps):
    """(y, mean, rstd) over the last axis."""
    x = x.astype(np.float64)
    mu = x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt(((x - mu) ** 2).mean(-1, keepdims=True) + eps)
    g = 1.0 if gamma is None else gamma.astype(np.float64)
    b = 0.0 if beta is None else beta.astype(np.float64)
    return (x - mu) * r * g + b, mu[..., 0], r[..., 0]


def norm_ops(H):
    """Roundings on the way of one term through a row's sum: H / 64 in a lane
    at the least parallel, the levels of the reduction, and the operations
    around it."""
    return H / 64 + 24


def layer_norm_bound(x, gamma, beta, eps):
    """The mean is off by c u mean|x|; so is every centred value, and the
    variance relatively by 2 c u and the square of the mean's error."""
    y, mu, r = layer_norm(x, gamma, beta, eps)
    x, r = x.astype(np.float64), r[..., None]
    c = norm_ops(x.shape[-1]) * U32
    g = 1.0 if gamma is None else np.abs(gamma.astype(np.float64))
    xh = np.abs(x - mu[..., None]) * r
    dxh = c * (2 * xh + np.abs(x).mean(-1, keepdims=True) * r)
    return g * dxh + c * np.abs(y), dxh


def layer_norm_grad(x, dy, gamma, eps):
    """(dx, dgamma, dbeta)."""
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    _, mu, r = layer_norm(x, None, None, eps)
    r = r[..., None]
    xh = (x - mu[..., None]) * r
    q = dy if gamma is None else dy * gamma.astype(np.float64)
    dx = r * (q - q.mean(-1, keepdims=True) - xh * (q * xh).mean(-1, keepdims=True))
    axes = tuple(range(x.ndim - 1))
    return dx, (dy * xh).sum(axes), dy.sum(axes)


def layer_norm_grad_bound(x, dy, gamma, eps):
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    _, mu, r = layer_norm(x, None, None, eps)
    _, dxh = layer_norm_bound(x, None, None, eps)
    r, c = r[..., None], norm_ops(x.shape[-1]) * U32
    xh = np.abs(x - mu[..., None]) * r
    q = np.abs(dy if gamma is None else dy * gamma.astype(np.float64))
    mean = lambda v: v.mean(-1, keepdims=True)  # noqa: E731
    bx = 2 * c * r * (q + mean(q) + xh * mean(q * xh)) + r * (dxh * mean(q * xh) + xh * mean(q * dxh))
    rel = mean(dxh * np.maximum(xh, 1e-30))  # the relative error of rstd, through the variance
    bx = bx + 2 * rel * r * (q + mean(q) + xh * mean(q * xh))
    axes = tuple(range(x.ndim - 1))
    R = float(np.prod([x.shape[i] for i in axes]))
    a = np.abs(dy)
    return bx, ((R + 32) * U32 * a * xh + a * dxh).sum(axes), ((R + 32) * U32 * a).sum(axes)


# --- gated linear recurrence -----------------------------------------------------

def _live(T, B, lengths):
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    return np.arange(T)[:, None] < n[None, :]


def linrec(x, gate, h0=None, resets=None, lengths=None):
    """dict(y, h_T, and the bounds y_err, h_T_err).  The bound follows the
    recurrence: a step multiplies the error before it by a, and adds 16 u of
    the magnitudes it sums (the gate's and its complement's errors of a few u,
    the products, the sum, and the same operations once more where the step's
    map is composed with others before it is applied)."""
    T, B, H = x.shape
    live = _live(T, B, lengths)
    h = np.zeros((B, H)) if h0 is None else h0.astype(np.float64).copy()
    mag, err = np.abs(h), np.zeros((B, H))
    y, ye = np.zeros((T, B, H)), np.zeros((T, B, H))
    before, be = np.zeros((T, B, H)), np.zeros((T, B, H))
    for t in range(T):
        on = live[t]
        if resets is not None:
            cut = on & (resets[t] != 0)
            h[cut], mag[cut], err[cut] = 0.0, 0.0, 0.0
        g, v = gate[t, on].astype(np.float64), x[t, on].astype(np.float64)
        a, om = sigmoid(g), sigmoid(-g)
        before[t], be[t] = np.where(on[:, None], h, 0), np.where(on[:, None], err, 0)
        h[on] = a * h[on] + om * v
        mag[on] = a * mag[on] + om * np.abs(v)
        err[on] = a * err[on] + 16 * U32 * mag[on]
        y[t, on], ye[t, on] = h[on], err[on]
    return dict(y=y, y_err=ye, h_T=h, h_T_err=err, before=before, before_err=be)


def linrec_grad(x, gate, dy, dh_T=None, h0=None, resets=None, lengths=None):
    """dict(dx, dgate, dh0 and their bounds *_err): the reverse recurrence with
    the same kind of bound, and the error of h_{t-1} on its way into dgate."""
    T, B, H = x.shape
    live = _live(T, B, lengths)
    f = linrec(x, gate, h0, resets, lengths)
    R = np.zeros((B, H)) if dh_T is None else dh_T.astype(np.float64).copy()
    mag, err = np.abs(R), np.zeros((B, H))
    out = {k: np.zeros((T, B, H)) for k in ("dx", "dgate", "dx_err", "dgate_err")}
    for t in range(T - 1, -1, -1):
        on = live[t]
        g, v, d = (q[t, on].astype(np.float64) for q in (gate, x, dy))
        a, om = sigmoid(g), sigmoid(-g)
        D, m, e = R[on] + d, mag[on] + np.abs(d), err[on]
        e = e + 16 * U32 * m
        p, pe = f["before"][t, on], f["before_err"][t, on]
        out["dx"][t, on], out["dx_err"][t, on] = om * D, om * e
        out["dgate"][t, on] = a * om * (p - v) * D
        out["dgate_err"][t, on] = a * om * ((np.abs(p) + np.abs(v)) * (e + 16 * U32 * m) + pe * m)
        R[on], mag[on], err[on] = a * D, a * m, a * e
        if resets is not None:
            cut = on & (resets[t] != 0)
            R[cut], mag[cut], err[cut] = 0.0, 0.0, 0.0
    return dict(out, dh0=R, dh0_err=err + 16 * U32 * mag)


# --- clipping ---------------------------------------------------------------

def clip(grads, max_norm):
    """(norm, factor, outs)."""
    norm = float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))
    with np.errstate(over="ignore"):
        seen = np.float32(norm)  # what the caller gets: infinite where fp32 cannot hold the norm
    f = max_norm / norm if norm > max_norm and np.isfinite(seen) else 1.0
    return norm, f, [g.astype(np.float64) * f for g in grads]
