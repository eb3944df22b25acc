"""Performance cases of the sequence-core operators: what a recurrent core
that trains in parallel over logged sequences consists of besides its matrix
products.

Kinds of case:
  embed  scaled rows of an action table for n logged actions (codes outside
         the table, as a frozen step logs them, give zero rows); with ``grad``
         also the table's gradient;
  norm   layer norm over rows; with ``grad`` also dx, dgamma, dbeta;
  rec    the gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) x_t,
         a = sigmoid(gate), over [T, B, H], with resets and lengths; with
         ``grad`` also dx, dgate, dh0;
  clip   the global norm of a model's gradient tensors, and their clipped
         values in the flat buffer that the optimiser step takes.

``packed``: x and gate are the halves of one projection's rows [T, B, 2H]
(rec), or the rows lie in a wider matrix (norm).
"""

from __future__ import annotations

import math

import torch

DEV = "cuda"
EPS = 1e-5

own = False


def listed():
    return [
        # the agent acting in its environment: one action's row, launch latency
        dict(name="embed_one", kind="embed", n=1, V=64, H=256, dtype="fp32", grad=False),
        # a training step's actions on padded sequences, sizes off every tile edge
        dict(name="embed_ragged", kind="embed", n=7224, V=50, H=367, dtype="fp32", grad=True),
        # the widest two-level action space (288 x 200) on the large model's batch
        dict(name="embed_two_level", kind="embed", n=81920, V=57600, H=1024, dtype="bf16", grad=True),
        # the agent acting: a few rows
        dict(name="norm_few", kind="norm", rows=16, H=1024, dtype="bf16", packed=False, grad=False),
        # a training step on padded sequences, rows of odd width inside a wider matrix
        dict(name="norm_ragged", kind="norm", rows=7224, H=367, dtype="fp32", packed=True, grad=True),
        # every step of the large dream batch
        dict(name="norm_large", kind="norm", rows=204800, H=1024, dtype="bf16", packed=False, grad=True),
        # the agents of the middle workload acting: one step from a kept state
        dict(name="rec_step", kind="rec", T=1, B=256, H=512, dtype="fp32", packed=True, masks=True, grad=False),
        # a training step on a few padded sequences of odd sizes
        dict(name="rec_ragged", kind="rec", T=45, B=100, H=367, dtype="bf16", packed=False, masks=True, grad=True),
        # the likelihood workload's sequences
        dict(name="rec_train", kind="rec", T=128, B=512, H=512, dtype="fp32", packed=True, masks=True, grad=True),
        # one long episode
        dict(name="rec_long", kind="rec", T=32768, B=1, H=1024, dtype="bf16", packed=True, masks=False, grad=True),
        # the gradient of a one-layer core at the smallest workload's width
        dict(name="clip_small", kind="clip", layers=1, H=256, Z=32, A=32, bf16=False, big=0.5),
        # a deep core with the widest action table: hundreds of millions of values, large and small tensors
        dict(name="clip_large", kind="clip", layers=24, H=1024, Z=64, A=57600, bf16=True, big=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "norm", "rec", "rec", "clip"])
    # the model widths in use, and any width around them
    H = rng.choice([256, 512, 1024, rng.randint(16, 1024), rng.randint(16, 1024)])
    c = dict(kind=kind, H=H, dtype=rng.choice(["fp32", "bf16"]), grad=rng.random() < 0.7)
    if kind == "embed":
        c["n"], c["V"] = _log(rng, 1, 120000), _log(rng, 8, 57600)
    elif kind == "norm":
        c["H"] = rng.choice([H, _log(rng, 16, 8192)])
        c["rows"] = max(1, min(_log(rng, 1, 200000), (90 if c["dtype"] == "fp32" else 180) * 1000000 // c["H"]))
        c["packed"] = rng.random() < 0.5
    elif kind == "rec":
        c["T"] = _log(rng, 1, 32768)
        c["B"] = max(1, min(_log(rng, 1, 4096), 30000000 // (c["T"] * H)))
        c["packed"], c["masks"] = rng.random() < 0.5, rng.random() < 0.5
    else:
        c = dict(kind=kind, H=H, layers=rng.randint(1, 24), Z=8 * _log(rng, 2, 16), A=_log(rng, 8, 57600),
                 bf16=rng.random() < 0.5, big=rng.choice([0.5, 2.0]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _clip_shapes(c):
    """The tensors of a core: the action table, the latent's projection, per
    layer two norms, the gate / candidate projection and the output one, and
    the reward and done heads."""
    H, Z, A = c["H"], c["Z"], c["A"]
    layer = [(H,), (H,), (2 * H, H), (2 * H,), (H, H), (H,)]
    return [(A, H), (H, Z), (H,)] + layer * c["layers"] + [(Z, H), (Z,), (H,), (1,), (H,), (1,)]


def _inputs(c, seed):
    """Everything random of a case, from the seed alone (device tensors)."""
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt = torch.bfloat16 if c.get("dtype") == "bf16" else torch.float32

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=g, device=DEV, dtype=dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    H = c["H"]
    if c["kind"] == "embed":
        n, V = c["n"], c["V"]
        # a learned policy prefers some actions; one step in twenty is frozen
        tok = (V * uniform(n) ** 2).long().clamp(max=V - 1)
        tok = torch.where(uniform(n) < 0.05, -1, (tok * 7919 + 13) % V).to(torch.int32)
        x = dict(tokens=tok, table=normal(V, H), scale=math.sqrt(H))
        if c["grad"]:
            x["dy"] = normal(n, H)
        return x
    if c["kind"] == "norm":
        rows, wide = c["rows"], H + (H // 2 if c["packed"] else 0)
        x = dict(x=normal(rows, wide)[:, :H], gamma=1 + 0.1 * normal(H, dtype=torch.float32),
                 beta=0.1 * normal(H, dtype=torch.float32))
        if c["grad"]:
            x["dy"] = normal(rows, wide)[:, :H]
        return x
    if c["kind"] == "rec":
        T, B = c["T"], c["B"]
        xg = normal(T, B, 2 * H)
        xg[..., H:] += 2  # gates that remember tens of steps, as a trained core's
        x = dict(x=xg[..., :H], gate=xg[..., H:]) if c["packed"] else dict(x=xg[..., :H].contiguous(), gate=xg[..., H:].contiguous())
        x["h0"] = normal(B, H, dtype=torch.float32)
        x["resets"] = (uniform(T, B) < 1.0 / max(T, 8)).to(torch.uint8) if c["masks"] else None
        x["lengths"] = (torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32).clamp(min=T // 4)
                        if c["masks"] and T > 1 else None)
        if c["grad"]:
            x["dy"], x["dh_T"] = normal(T, B, H), normal(B, H, dtype=torch.float32)
        return x
    shapes = _clip_shapes(c)
    # matrices in bf16 where asked, vectors always fp32, at the sizes of a mean loss's gradient
    grads = [1e-3 * normal(*s, dtype=torch.bfloat16 if c["bf16"] and len(s) > 1 else torch.float32) for s in shapes]
    norm = 1e-3 * math.sqrt(sum(math.prod(s) for s in shapes))
    return dict(grads=grads, max_norm=norm / c["big"])  # big 2: the norm is over the limit, 0.5: under it


def prepare(case, seed):
    c = dict(case)
    s = dict(c=c, x=_inputs(c, seed))
    if c["kind"] == "clip":
        # one flat buffer for each type, as the optimiser's step takes them, and its views in the tensors' shapes
        s["flats"], s["views"], at = {}, [], {}
        for dt in (torch.float32, torch.bfloat16):
            s["flats"][dt] = torch.empty(sum(g.numel() for g in s["x"]["grads"] if g.dtype == dt), dtype=dt, device=DEV)
        for g in s["x"]["grads"]:
            i = at.get(g.dtype, 0)
            at[g.dtype] = i + g.numel()
            s["views"].append(s["flats"][g.dtype][i:i + g.numel()].view(g.shape))
    if own:
        from paper_2205_01435_amd import _lib as wm

        s["wm"] = wm
        dt = torch.bfloat16 if c.get("dtype") == "bf16" else torch.float32
        if c["kind"] == "embed":
            s["out"] = torch.empty(c["n"], c["H"], dtype=dt, device=DEV)
            s["bufs"] = wm.EmbedGradBuffers(c["n"], c["V"], c["H"]) if c["grad"] else None
        elif c["kind"] == "norm":
            s["bufs"] = wm.LayerNormBuffers(c["rows"], c["H"], dt, grad=c["grad"])
        elif c["kind"] == "rec":
            s["bufs"] = wm.LinrecBuffers(c["T"], c["B"], c["H"], dt, grad=c["grad"])
        else:
            s["bufs"] = wm.ClipPlan(s["x"]["grads"], s["views"])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    c, x = s["c"], s["x"]
    if not own:
        return _PLAIN[c["kind"]](c, x)
    wm = s["wm"]
    if c["kind"] == "embed":
        r = dict(y=wm.embed(x["table"], x["tokens"], x["scale"], out=s["out"]))
        if c["grad"]:
            r["dtable"] = wm.embed_grad(x["tokens"], x["dy"], c["V"], x["scale"], bufs=s["bufs"]).grad
        return r
    b = s["bufs"]
    if c["kind"] == "norm":
        wm.layer_norm(x["x"], x["gamma"], x["beta"], EPS, bufs=b)
        r = dict(y=b.y)
        if c["grad"]:
            wm.layer_norm_grad(x["x"], x["dy"], x["gamma"], bufs=b)
            r.update(dx=b.dx, dgamma=b.dgamma, dbeta=b.dbeta)
        return r
    if c["kind"] == "rec":
        wm.linrec(x["x"], x["gate"], h0=x["h0"], resets=x["resets"], lengths=x["lengths"], bufs=b)
        r = dict(y=b.y, h_T=b.h_T)
        if c["grad"]:
            wm.linrec_grad(x["x"], x["gate"], x["dy"], dh_T=x["dh_T"], resets=x["resets"], lengths=x["lengths"], bufs=b)
            r.update(dx=b.dx, dgate=b.dgate, dh0=b.dh0)
        return r
    wm.clip_grads(b, x["max_norm"])
    return dict(norm=b.norm, fp32=s["flats"][torch.float32], bf16=s["flats"][torch.bfloat16])


def _plain_embed(c, x):
    tok, V, dt = x["tokens"].long(), c["V"], x["table"].dtype
    ok = (tok >= 0) & (tok < V)
    rows = x["table"].index_select(0, tok.clamp(0, V - 1)).float() * x["scale"]
    r = dict(y=torch.where(ok[:, None], rows, torch.zeros_like(rows)).to(dt))
    if c["grad"]:
        # the codes add into a row past the table's end
        d = torch.zeros(V + 1, c["H"], device=DEV).index_add_(0, torch.where(ok, tok, V), x["dy"].float() * x["scale"])
        r["dtable"] = d[:V]
    return r


def _plain_norm(c, x):
    v, dt = x["x"].float(), x["x"].dtype
    d = v - v.mean(-1, keepdim=True)
    rstd = (d.square().mean(-1, keepdim=True) + EPS).rsqrt()
    xh = d * rstd
    r = dict(y=(xh * x["gamma"] + x["beta"]).to(dt))
    if c["grad"]:
        dy = x["dy"].float()
        q = dy * x["gamma"]
        r["dx"] = (rstd * (q - q.mean(-1, keepdim=True) - xh * (q * xh).mean(-1, keepdim=True))).to(dt)
        r["dgamma"], r["dbeta"] = (dy * xh).sum(0), dy.sum(0)
    return r


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t from h_{-1} = 0 over the first axis, by doubling:
    after k rounds (a, u) are the maps over the last 2^k steps."""
    k = 1
    while k < u.shape[0]:
        u = torch.cat([u[:k], u[k:] + a[k:] * u[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return u


def _masks(c, x):
    """[T, B, 1] truth values: the step lies in its sequence, and starts a new one."""
    T, B = c["T"], c["B"]
    t = torch.arange(T, device=DEV)[:, None, None]
    live = t < (x["lengths"][None, :, None] if x["lengths"] is not None else T)
    live = live.expand(T, B, 1)
    start = live & (x["resets"][..., None] != 0) if x["resets"] is not None else torch.zeros_like(live)
    return live, start


def _plain_rec(c, x):
    dt, h0 = x["x"].dtype, x["h0"][None]
    v, g = x["x"].float(), x["gate"].float()
    live, start = _masks(c, x)
    sig, off = torch.sigmoid(g), torch.sigmoid(-g)
    a = torch.where(start, 0.0, torch.where(live, sig, 1.0))
    u = torch.where(live, off * v, 0.0)
    h = _scan(a, torch.cat([u[:1] + a[:1] * h0, u[1:]]))
    r = dict(y=torch.where(live, h, 0.0).to(dt), h_T=h[-1])
    if c["grad"]:
        D = torch.where(live, x["dy"].float(), 0.0)
        D = torch.cat([D[:-1], D[-1:] + x["dh_T"][None]])
        nxt = torch.cat([a[1:], torch.zeros_like(a[:1])])  # what step t + 1 takes of h_t
        D = _scan(nxt.flip(0), D.flip(0)).flip(0)
        prev = torch.where(start, 0.0, torch.cat([h0, h[:-1]]))
        r["dx"] = torch.where(live, D * off, 0.0).to(dt)
        r["dgate"] = torch.where(live, D * (prev - v) * sig * off, 0.0).to(dt)
        r["dh0"] = (a * D)[0]
    return r


def _plain_clip(c, x):
    norm = torch.stack([g.float().square().sum() for g in x["grads"]]).sum().sqrt()
    k = torch.where(norm > x["max_norm"], x["max_norm"] / norm, 1.0)
    out = [(g.float() * k).to(g.dtype).reshape(-1) for g in x["grads"]]
    none = [torch.empty(0, device=DEV)]
    return dict(norm=norm.reshape(1), fp32=torch.cat([o for o in out if o.dtype == torch.float32]),
                bf16=torch.cat([o for o in out if o.dtype == torch.bfloat16] or [t.to(torch.bfloat16) for t in none]))


_PLAIN = dict(embed=_plain_embed, norm=_plain_norm, rec=_plain_rec, clip=_plain_clip)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c, H, e = case, case["H"], 2 if case.get("dtype") == "bf16" else 4
    if c["kind"] == "embed":
        n, V = c["n"], c["V"]
        b, f = 4 * n + min(n, V) * H * e + n * H * e, n * H
        if c["grad"]:
            b, f = b + n * H * e + 4 * V * H, f + n * H
        return dict(bytes=float(b), flops=float(f))
    if c["kind"] == "norm":
        m = c["rows"] * H
        b, f = 2 * m * e + 8 * H, 8 * m
        if c["grad"]:
            b, f = b + 2 * m * e + 8 * H, f + 14 * m  # x counts once for the pass
        return dict(bytes=float(b), flops=float(f))
    if c["kind"] == "rec":
        T, B = c["T"], c["B"]
        m = T * B * H
        b, f = 3 * m * e + 8 * B * H + (T * B + 4 * B if c["masks"] else 0), 8 * m
        if c["grad"]:
            b, f = b + 3 * m * e + 8 * B * H, f + 14 * m  # x and the gate count once
        return dict(bytes=float(b), flops=float(f))
    n = [(math.prod(s), 2 if c["bf16"] and len(s) > 1 else 4) for s in _clip_shapes(c)]
    return dict(bytes=float(sum(2 * k * w for k, w in n) + 4), flops=3.0 * sum(k for k, _ in n))


# ---------------------------------------------------------------------------
# the same in 64 bits, step by step
# ---------------------------------------------------------------------------

def exact(case, seed):
    c = dict(case)
    x = _inputs(c, seed)

    def embed():
        V, H, n = c["V"], c["H"], c["n"]
        # a table with a row of zeros at its end, where every code outside it points
        table = torch.cat([x["table"].double(), torch.zeros(1, H, dtype=torch.float64, device=DEV)])
        tok = x["tokens"].long()
        tok[(tok < 0) | (tok >= V)] = V
        r = dict(y=table[tok] * x["scale"])
        if c["grad"]:
            # sums of runs of equal tokens: differences of the running sum over the sorted rows
            order = torch.argsort(tok, stable=True)
            end = torch.searchsorted(tok[order].contiguous(), torch.arange(V + 1, device=DEV))
            cols = []
            for h in range(0, H, 64):
                run_sum = torch.zeros(n + 1, min(64, H - h), dtype=torch.float64, device=DEV)
                run_sum[1:] = x["dy"][order, h:h + 64].double().cumsum(0)
                cols.append((run_sum[end[1:]] - run_sum[end[:-1]]) * x["scale"])
            r["dtable"] = torch.cat(cols, 1)
        return r

    def norm():
        n, H, out = c["rows"], c["H"], dict(y=[], dx=[])
        gamma, beta = x["gamma"].double(), x["beta"].double()
        dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
        for i in range(0, n, 1 << 14):
            v = x["x"][i:i + (1 << 14)].double()
            var, mean = torch.var_mean(v, -1, unbiased=False, keepdim=True)
            s = torch.sqrt(var + EPS)
            out["y"].append((v - mean) / s * gamma + beta)
            if c["grad"]:
                d = x["dy"][i:i + (1 << 14)].double()
                dgamma += (d * (v - mean) / s).sum(0)
                dbeta += d.sum(0)
                q = d * gamma
                along = (q * (v - mean)).sum(-1, keepdim=True) / (H * s * s)
                out["dx"].append((q - q.mean(-1, keepdim=True) - (v - mean) * along) / s)
        r = dict(y=torch.cat(out["y"]))
        if c["grad"]:
            r.update(dx=torch.cat(out["dx"]), dgamma=dgamma, dbeta=dbeta)
        return r

    def rec():
        T, B, H = c["T"], c["B"], c["H"]
        n = x["lengths"].long() if x["lengths"] is not None else torch.full((B,), T, device=DEV)
        rs = x["resets"] if x["resets"] is not None else torch.zeros(T, B, dtype=torch.uint8, device=DEV)
        keep = (rs == 0).double()[..., None]
        live = (torch.arange(T, device=DEV)[:, None] < n[None]).double()[..., None]
        h = x["h0"].double()
        y, before = (torch.empty(T, B, H, dtype=torch.float64, device=DEV) for _ in range(2))
        for t in range(T):
            p, v = h * keep[t], x["x"][t].double()
            before[t] = p
            new = v + (p - v) * torch.sigmoid(x["gate"][t].double())
            y[t] = new * live[t]
            h = h + (new - h) * live[t]
        r = dict(y=y, h_T=h)
        if c["grad"]:
            d = x["dh_T"].double()
            dx, dg = torch.empty_like(y), torch.empty_like(y)
            for t in range(T - 1, -1, -1):
                a = torch.sigmoid(x["gate"][t].double())
                m = (d + x["dy"][t].double()) * live[t]
                dx[t] = m * (1 - a)
                dg[t] = m * (before[t] - x["x"][t].double()) * a * (1 - a)
                d = d * (1 - live[t]) + m * a * keep[t]
            r.update(dx=dx, dgate=dg, dh0=d)
        return r

    def clip():
        total = sum(float(g.double().square().sum()) for g in x["grads"])
        k = min(1.0, x["max_norm"] / math.sqrt(total))
        out = {torch.float32: [], torch.bfloat16: [torch.empty(0, dtype=torch.float64, device=DEV)]}
        for g in x["grads"]:
            out[g.dtype].append(g.double().reshape(-1) * k)
        return dict(norm=torch.full((1,), math.sqrt(total), dtype=torch.float64, device=DEV),
                    fp32=torch.cat(out[torch.float32]), bf16=torch.cat(out[torch.bfloat16]))

    return dict(embed=embed, norm=norm, rec=rec, clip=clip)[c["kind"]]()
