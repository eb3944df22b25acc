"""A recurrent core that trains in parallel over logged sequences, on the
library's sequence-core operators.

It predicts the next latent and the reward from the latents and actions so far:

    e_t = s E[a_t] + W_z z_t          embed, and a product
    n_t = norm(e_t)                   layer_norm
    [x_t, g_t] = W_in n_t + b_in      one product, its halves
    h_t = linrec(x_t, g_t)            over all steps at once
    o_t = norm(h_t)                   layer_norm
    [z_{t+1}, r_t] ~ W_out o_t + b_out

and is fitted by the mean squared error over the steps inside each sequence:
the gradient of every weight, their global norm, clipping into the flat buffer
that the optimiser takes, Adam.  ``act`` is the same core one step at a time,
its state kept between calls.

    python examples/seq_core.py [steps]
"""

from __future__ import annotations

import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2205_01435_amd import _lib as wm  # noqa: E402


class SeqCore:
    """Weights (views of one flat buffer), and the buffers of one batch shape."""

    def __init__(self, A: int, Z: int, H: int, T: int, B: int, seed: int = 0, device="cuda"):
        self.A, self.Z, self.H, self.T, self.B = A, Z, H, T, B
        shapes = {"E": (A, H), "W_z": (H, Z), "n1_g": (H,), "n1_b": (H,), "W_in": (2 * H, H), "b_in": (2 * H,),
                  "n2_g": (H,), "n2_b": (H,), "W_out": (Z + 1, H), "b_out": (Z + 1,)}
        # the optimiser's arrays start on 16-byte boundaries
        sizes = {k: (math.prod(s) + 3) // 4 * 4 for k, s in shapes.items()}
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
        self.w["n1_g"].fill_(1.0)
        self.w["n2_g"].fill_(1.0)
        self.w["b_in"][H:] = 2.0  # gates that remember some ten steps at first
        self.scale = math.sqrt(H)
        self.w["E"].mul_(1.0 / math.sqrt(H))
        self.e_bufs = wm.EmbedGradBuffers(T * B, A, H, device)
        self.n1, self.n2 = (wm.LayerNormBuffers(T * B, H, device=device) for _ in range(2))
        self.rec = wm.LinrecBuffers(T, B, H, device=device)
        self.e_bufs.grad, self.n1.dgamma, self.n1.dbeta = self.grads["E"], self.grads["n1_g"], self.grads["n1_b"]
        self.n2.dgamma, self.n2.dbeta = self.grads["n2_g"], self.grads["n2_b"]
        self.clip = wm.ClipPlan(list(self.grads.values()), [self.clipped[k] for k in self.grads])
        self.steps = 0

    def forward(self, z, actions, resets=None, lengths=None):
        """Predictions [T, B, Z + 1] for latents z [T, B, Z] and int32 actions
        [T, B]."""
        w, (T, B, H) = self.w, (self.T, self.B, self.H)
        e = wm.embed(w["E"], actions, self.scale).view(T * B, H)
        e.addmm_(z.view(T * B, -1), w["W_z"].t())
        wm.layer_norm(e, w["n1_g"], w["n1_b"], bufs=self.n1)
        xg = torch.addmm(w["b_in"], self.n1.y, w["W_in"].t()).view(T, B, 2 * H)
        wm.linrec(xg[..., :H], xg[..., H:], resets=resets, lengths=lengths, bufs=self.rec)
        wm.layer_norm(self.rec.y, w["n2_g"], w["n2_b"], bufs=self.n2)
        self.kept = (z, actions, resets, lengths, e, xg)
        return torch.addmm(w["b_out"], self.n2.y, w["W_out"].t()).view(T, B, -1)

    def backward(self, dpred):
        """Every weight's gradient (self.grads) from that of the predictions."""
        w, g, (T, B, H) = self.w, self.grads, (self.T, self.B, self.H)
        z, actions, resets, lengths, e, xg = self.kept
        d = dpred.reshape(T * B, -1)
        torch.mm(d.t(), self.n2.y, out=g["W_out"])
        torch.sum(d, 0, out=g["b_out"])
        wm.layer_norm_grad(self.rec.y, d @ w["W_out"], w["n2_g"], bufs=self.n2)
        wm.linrec_grad(xg[..., :H], xg[..., H:], self.n2.dx.view(T, B, H), resets=resets, lengths=lengths, bufs=self.rec)
        dxg = self.rec.dxg.view(T * B, 2 * H)
        torch.mm(dxg.t(), self.n1.y, out=g["W_in"])
        torch.sum(dxg, 0, out=g["b_in"])
        wm.layer_norm_grad(e, dxg @ w["W_in"], w["n1_g"], bufs=self.n1)
        torch.mm(self.n1.dx.t(), z.reshape(T * B, -1), out=g["W_z"])
        wm.embed_grad(actions, self.n1.dx.view(T, B, H), self.A, self.scale, bufs=self.e_bufs)

    def train_step(self, z, actions, rewards, resets=None, lengths=None, lr: float = 1e-3, max_norm: float = 1.0):
        """One step on logged latents z [T + 1, B, Z], actions and rewards
        [T, B]; returns the loss and the gradient's norm (device tensors)."""
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

    def act(self, z, action, state, reset=None):
        """One step for rows of any number: the prediction [B, Z + 1] and the
        new state [B, H] (from z [B, Z], action [B] int32, state [B, H])."""
        w, H = self.w, self.H
        e = wm.embed(w["E"], action, self.scale)
        e.addmm_(z, w["W_z"].t())
        n1 = wm.layer_norm(e, w["n1_g"], w["n1_b"], bufs=wm.LayerNormBuffers(len(z), H, grad=False))
        xg = torch.addmm(w["b_in"], n1.y, w["W_in"].t())[None]
        rec = wm.linrec(xg[..., :H], xg[..., H:], state, None if reset is None else reset[None],
                        bufs=wm.LinrecBuffers(1, len(z), H, grad=False))
        n2 = wm.layer_norm(rec.y[0], w["n2_g"], w["n2_b"], bufs=wm.LayerNormBuffers(len(z), H, grad=False))
        return torch.addmm(w["b_out"], n2.y, w["W_out"].t()), rec.h_T


def logged(A: int, Z: int, T: int, B: int, seed: int = 0, device="cuda"):
    """Logged sequences whose next latent and reward depend on the action:
    z [T + 1, B, Z], actions, rewards, resets [T, B], lengths [B]."""
    g = torch.Generator(device=device).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=device)  # noqa: E731
    effect, z = 0.5 * r(A, Z), r(T + 1, B, Z)
    actions = torch.randint(0, A, (T, B), generator=g, device=device, dtype=torch.int32)
    resets = (torch.rand(T, B, generator=g, device=device) < 1.0 / T).to(torch.uint8)
    for t in range(T):
        z[t + 1] = 0.9 * z[t] + effect[actions[t].long()] + 0.1 * z[t + 1]
    rewards = z[:T, :, 0] * 0.3 + 0.1 * r(T, B)
    lengths = torch.randint(T // 2, T + 1, (B,), generator=g, device=device, dtype=torch.int32)
    return z, actions, rewards, resets, lengths


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 200
    A, Z, H, T, B = 64, 64, 512, 128, 128
    core, (z, actions, rewards, resets, lengths) = SeqCore(A, Z, H, T, B), logged(A, Z, T, B)
    for k in range(steps):
        loss, norm = core.train_step(z, actions, rewards, resets, lengths, lr=wm.poly_lr(k, 1e-3, 1e-5, steps))
        if k % 20 == 0 or k == steps - 1:
            print(f"step {k:4d}  loss {float(loss):.4f}  gradient norm {float(norm):.3f}", flush=True)
    state = torch.zeros(B, H, device="cuda")
    for t in range(3):
        pred, state = core.act(z[t], actions[t], state, resets[t])
    print(f"one step at a time: predicted reward of row 0 {float(pred[0, -1]):.3f}, logged {float(rewards[2, 0]):.3f}")


if __name__ == "__main__":
    main()
