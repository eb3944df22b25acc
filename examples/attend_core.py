"""A core that mixes the steps of logged sequences by linear attention, on the
library's operators:

    e_t = s E[a_t] + W_z z_t                     embed, and a product
    [q, k, v] = W_qkv norm(e)                    layer_norm, one product, its parts
    q, k = rotated norms of their heads          qk_norm, by the step's position
    m = linattn(q, k, v)                         every head with its own decay
    f = e + W_o norm_head(m)                     layer_norm of each head's output
    g = f + W_2 (silu(W_g n) * (W_u n)), n = norm(f)     layer_norm, glu, a product
    [z_{t+1}, r_t] ~ W_out norm(g) + b_out

fitted by the mean squared error over the steps inside each sequence: the
gradient of every weight, clipping, Adam.  ``act`` is the same core one step at a
time; what it keeps of the past is each head's state, whatever the length.

    python examples/attend_core.py [steps]
"""

from __future__ import annotations

import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for _p in (ROOT, os.path.join(ROOT, "examples")):
    if _p not in sys.path:
        sys.path.insert(0, _p)

from paper_2205_01435_amd import _lib as wm  # noqa: E402
from seq_core import logged  # noqa: E402


class AttendCore:
    """Weights (views of one flat buffer), and the buffers of one batch shape.  The
    core has N heads of width H / N, and F columns in its feed-forward block."""

    def __init__(self, A: int, Z: int, H: int, N: int, F: int, T: int, B: int, seed: int = 0, device="cuda"):
        self.A, self.Z, self.H, self.N, self.D, self.F, self.T, self.B = A, Z, H, N, H // N, F, T, B
        D = self.D
        shapes = {"E": (A, H), "W_z": (H, Z), "n1_g": (H,), "n1_b": (H,), "W_qkv": (3 * H, H), "g_q": (D,), "g_k": (D,),
                  "nh_g": (D,), "nh_b": (D,), "W_o": (H, H), "n2_g": (H,), "n2_b": (H,), "W_gu": (2 * F, H), "W_2": (H, F),
                  "n3_g": (H,), "n3_b": (H,), "W_out": (Z + 1, H), "b_out": (Z + 1,)}
        sizes = {k: (math.prod(s) + 3) // 4 * 4 for k, s in shapes.items()}  # 16-byte boundaries for the optimiser
        new = lambda: torch.zeros(sum(sizes.values()), device=device)  # noqa: E731
        self.flat, self.flat_grad, self.m, self.v = new(), new(), new(), new()
        self.w, self.clipped, self.grads, at = {}, {}, {}, 0
        gen = torch.Generator(device=device).manual_seed(seed)
        for k, s in shapes.items():
            n = math.prod(s)
            self.w[k] = self.flat[at:at + n].view(s)
            self.clipped[k] = self.flat_grad[at:at + n].view(s)
            self.grads[k] = torch.zeros(s, device=device)
            at += sizes[k]
            if len(s) == 2:
                self.w[k].copy_(torch.randn(s, generator=gen, device=device) / math.sqrt(s[1]))
            elif k.endswith("_g") or k.startswith("g_"):
                self.w[k].fill_(1.0)
        self.scale, self.attn_scale = math.sqrt(H), D ** -0.5
        self.w["E"].mul_(1.0 / math.sqrt(H))
        # heads that remember from 4 to 256 steps
        self.decay = torch.tensor([1 - 2.0 ** -(2 + 6 * n / max(N - 1, 1)) for n in range(N)], device=device)
        self.rotary = wm.Rotary(D // 2 * 2, device=device)
        R = T * B
        self.e_bufs = wm.EmbedGradBuffers(R, A, H, device)
        self.n1, self.n2, self.n3 = (wm.LayerNormBuffers(R, H, device=device) for _ in range(3))
        self.nh = wm.LayerNormBuffers(R * N, D, device=device)
        self.qk = wm.QkNormBuffers(R, N, N, D, device=device)
        self.mix = wm.LinattnBuffers(T, B, N, D, D, device=device)
        self.ff = wm.GluBuffers(R, H, F, device=device)
        g = self.grads
        # the gradients of q, k and v as the parts of their projection's
        self.dqkv = torch.empty(T, B, 3, N, D, device=device)
        self.qk.dq, self.qk.dk, self.mix.dv = (self.dqkv[:, :, i] for i in range(3))
        self.e_bufs.grad, self.qk.dgamma_q, self.qk.dgamma_k, self.ff.dW = g["E"], g["g_q"], g["g_k"], g["W_gu"]
        for b, n in ((self.n1, "n1"), (self.n2, "n2"), (self.n3, "n3"), (self.nh, "nh")):
            b.dgamma, b.dbeta = g[n + "_g"], g[n + "_b"]
        self.clip = wm.ClipPlan(list(g.values()), [self.clipped[k] for k in g])
        self.positions = torch.arange(T, dtype=torch.int32, device=device)[:, None].expand(T, B).contiguous()
        self.steps = 0

    def forward(self, z, actions, resets=None, lengths=None, positions=None):
        """Predictions [T, B, Z + 1] for latents z [T, B, Z] and int32 actions
        [T, B] (``positions`` [T, B] int32: the steps' own, counted from 0 without)."""
        w, (T, B, H, N, D) = self.w, (self.T, self.B, self.H, self.N, self.D)
        pos = self.positions if positions is None else positions
        e = wm.embed(w["E"], actions, self.scale).view(T * B, H)
        e.addmm_(z.view(T * B, -1), w["W_z"].t())
        wm.layer_norm(e, w["n1_g"], w["n1_b"], bufs=self.n1)
        qkv = torch.mm(self.n1.y, w["W_qkv"].t()).view(T, B, 3, N, D)
        wm.qk_norm(qkv[:, :, 0], qkv[:, :, 1], pos, self.rotary, w["g_q"], w["g_k"], bufs=self.qk)
        q, k = (x.view(T, B, N, D) for x in (self.qk.q, self.qk.k))
        wm.linattn(q, k, qkv[:, :, 2], self.decay, self.attn_scale, resets=resets, lengths=lengths, bufs=self.mix)
        wm.layer_norm(self.mix.y, w["nh_g"], w["nh_b"], bufs=self.nh)
        f = torch.addmm(e, self.nh.y.view(T * B, H), w["W_o"].t())
        wm.layer_norm(f, w["n2_g"], w["n2_b"], bufs=self.n2)
        wm.glu(self.n2.y, w["W_gu"], bufs=self.ff)
        g = torch.addmm(f, self.ff.h, w["W_2"].t())
        wm.layer_norm(g, w["n3_g"], w["n3_b"], bufs=self.n3)
        self.kept = (z, actions, resets, lengths, pos, e, qkv, f, g)
        return torch.addmm(w["b_out"], self.n3.y, w["W_out"].t()).view(T, B, -1)

    def backward(self, dpred):
        """Every weight's gradient (self.grads) from that of the predictions."""
        w, gr, (T, B, H, N, D) = self.w, self.grads, (self.T, self.B, self.H, self.N, self.D)
        z, actions, resets, lengths, pos, e, qkv, f, g = self.kept
        d = dpred.reshape(T * B, -1)
        torch.mm(d.t(), self.n3.y, out=gr["W_out"])
        torch.sum(d, 0, out=gr["b_out"])
        wm.layer_norm_grad(g, d @ w["W_out"], w["n3_g"], bufs=self.n3)
        dg = self.n3.dx
        torch.mm(dg.t(), self.ff.h, out=gr["W_2"])
        wm.glu_grad(self.n2.y, w["W_gu"], dg @ w["W_2"], bufs=self.ff)
        wm.layer_norm_grad(f, self.ff.dx, w["n2_g"], bufs=self.n2)
        df = dg + self.n2.dx
        torch.mm(df.t(), self.nh.y.view(T * B, H), out=gr["W_o"])
        wm.layer_norm_grad(self.mix.y, (df @ w["W_o"]).view(T * B * N, D), w["nh_g"], bufs=self.nh)
        q, k = (x.view(T, B, N, D) for x in (self.qk.q, self.qk.k))
        wm.linattn_grad(q, k, qkv[:, :, 2], self.decay, self.nh.dx.view(T, B, N, D), self.attn_scale, resets=resets,
                        lengths=lengths, bufs=self.mix)
        wm.qk_norm_grad(qkv[:, :, 0], qkv[:, :, 1], self.mix.dq, self.mix.dk, pos, self.rotary, w["g_q"], w["g_k"], bufs=self.qk)
        dqkv = self.dqkv.view(T * B, 3 * H)
        torch.mm(dqkv.t(), self.n1.y, out=gr["W_qkv"])
        wm.layer_norm_grad(e, dqkv @ w["W_qkv"], w["n1_g"], bufs=self.n1)
        de = df + self.n1.dx
        torch.mm(de.t(), z.reshape(T * B, -1), out=gr["W_z"])
        wm.embed_grad(actions, de.view(T, B, H), self.A, self.scale, bufs=self.e_bufs)

    def train_step(self, z, actions, rewards, resets=None, lengths=None, lr: float = 1e-3, max_norm: float = 1.0):
        """One step on logged latents z [T + 1, B, Z], actions and rewards [T, B];
        returns the loss and the gradient's norm (device tensors)."""
        T, B = self.T, self.B
        pred = self.forward(z[:T].contiguous(), actions, resets, lengths)
        live = torch.ones(T, B, 1, device=z.device)
        if lengths is not None:
            live = (torch.arange(T, device=z.device)[:, None] < lengths[None, :]).float()[..., None]
        err = (pred - torch.cat([z[1:], rewards[..., None]], -1)) * live
        n = live.sum() * (self.Z + 1)
        self.backward(err * (2.0 / n))
        norm = wm.clip_grads(self.clip, max_norm)
        self.steps += 1
        wm.adam_step(self.flat, self.flat_grad, self.m, self.v, self.steps, lr)
        return (err * err).sum() / n, norm

    def act(self, z, action, position, state, reset=None):
        """One step for rows of any number: the prediction [B, Z + 1] and the new
        state [B, N, D, D] (from z [B, Z], action and position [B] int32)."""
        w, H, N, D, B = self.w, self.H, self.N, self.D, len(z)
        norm = lambda x, n: wm.layer_norm(x, w[n + "_g"], w[n + "_b"],  # noqa: E731
                                          bufs=wm.LayerNormBuffers(x.numel() // x.shape[-1], x.shape[-1], grad=False)).y
        e = wm.embed(w["E"], action, self.scale)
        e.addmm_(z, w["W_z"].t())
        qkv = torch.mm(norm(e, "n1"), w["W_qkv"].t()).view(B, 3, N, D)
        qk = wm.qk_norm(qkv[:, 0], qkv[:, 1], position, self.rotary, w["g_q"], w["g_k"])
        mix = wm.linattn(qk.q[None], qk.k[None], qkv[None, :, 2], self.decay, self.attn_scale, h0=state,
                         resets=None if reset is None else reset[None], bufs=wm.LinattnBuffers(1, B, N, D, D, grad=False))
        f = torch.addmm(e, norm(mix.y[0], "nh").view(B, H), w["W_o"].t())
        ff = wm.glu(norm(f, "n2"), w["W_gu"], bufs=wm.GluBuffers(B, H, self.F, grad=False))
        g = torch.addmm(f, ff.h, w["W_2"].t())
        return torch.addmm(w["b_out"], norm(g, "n3"), w["W_out"].t()), mix.h_T


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 200
    A, Z, H, N, F, T, B = 64, 64, 512, 8, 1408, 128, 128
    core, (z, actions, rewards, resets, lengths) = AttendCore(A, Z, H, N, F, T, B), logged(A, Z, T, B)
    for k in range(steps):
        loss, norm = core.train_step(z, actions, rewards, resets, lengths, lr=wm.poly_lr(k, 1e-3, 1e-5, steps))
        if k % 20 == 0 or k == steps - 1:
            print(f"step {k:4d}  loss {float(loss):.4f}  gradient norm {float(norm):.3f}", flush=True)
    state = torch.zeros(B, N, H // N, H // N, device="cuda")
    for t in range(3):
        pred, state = core.act(z[t], actions[t], core.positions[t], state, resets[t])
    print(f"one step at a time: predicted reward of row 0 {float(pred[0, -1]):.3f}, logged {float(rewards[2, 0]):.3f}")


if __name__ == "__main__":
    main()
