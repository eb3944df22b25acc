"""GPU test of the sequence core built on the operators (examples/seq_core.py):
every weight's gradient against automatic differentiation of the same model
written plainly in 64 bits on the CPU, the loss going down, and the one-step
form against the pass over all steps."""

import os
import sys

import numpy as np
import pytest
import torch

from seqcheck import say

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
SIZES = dict(A=11, Z=8, H=37, T=21, B=6)


@pytest.fixture(scope="module")
def sc():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import seq_core
    return seq_core


def _plain(core, z, actions, rewards, resets, lengths):
    """Loss and gradients by automatic differentiation in float64, CPU."""
    w = {k: v.detach().double().cpu().requires_grad_(True) for k, v in core.w.items()}
    z, rewards = z.double().cpu(), rewards.double().cpu()
    actions, resets, lengths = actions.long().cpu(), resets.cpu(), lengths.cpu()
    T, B, H = core.T, core.B, core.H

    def norm(x, g, b):
        d = x - x.mean(-1, keepdim=True)
        return d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5) * g + b

    e = core.scale * w["E"][actions] + z[:T] @ w["W_z"].t()
    xg = norm(e, w["n1_g"], w["n1_b"]) @ w["W_in"].t() + w["b_in"]
    h, ys = torch.zeros(B, H, dtype=torch.float64), []
    for t in range(T):
        a = torch.sigmoid(xg[t, :, H:])
        live = (t < lengths)[:, None]
        new = a * torch.where(resets[t][:, None] != 0, torch.zeros_like(h), h) + (1 - a) * xg[t, :, :H]
        h = torch.where(live, new, h)
        ys.append(torch.where(live, new, torch.zeros_like(new)))
    pred = norm(torch.stack(ys), w["n2_g"], w["n2_b"]) @ w["W_out"].t() + w["b_out"]
    live = (torch.arange(T)[:, None] < lengths[None]).double()[..., None]
    err = (pred - torch.cat([z[1:], rewards[..., None]], -1)) * live
    loss = (err * err).sum() / (live.sum() * (core.Z + 1))
    loss.backward()
    return loss.detach(), {k: v.grad for k, v in w.items()}


def test_gradients_of_every_weight(sc):
    core = sc.SeqCore(**SIZES)
    data = sc.logged(SIZES["A"], SIZES["Z"], SIZES["T"], SIZES["B"])
    ref_loss, ref = _plain(core, *data)
    before = core.flat.clone()
    loss, norm = core.train_step(*data, lr=1e-3, max_norm=0.1)
    say("seq core", float(loss), float(norm))
    # fp32 throughout: some hundred roundings a value through two norms and the
    # recurrence, a condition of a few; no gradient is a difference of larger ones
    assert abs(float(loss) - float(ref_loss)) <= 1e-5 * float(ref_loss)
    total = np.sqrt(sum(float((g ** 2).sum()) for g in ref.values()))
    assert abs(float(norm) - total) <= 1e-4 * total
    for k, g in ref.items():
        got = core.grads[k].double().cpu()
        assert float((got - g).norm()) <= 1e-4 * float(g.norm()) + 1e-5 * total, k
        clipped = core.clipped[k].double().cpu()
        assert float((clipped - got * min(1.0, 0.1 / total)).norm()) <= 1e-4 * 0.1, k
    assert not torch.equal(before, core.flat)


def test_the_loss_goes_down_and_steps_agree(sc):
    A, Z, H, T, B = 16, 16, 128, 40, 24
    core = sc.SeqCore(A, Z, H, T, B, seed=1)
    z, actions, rewards, resets, lengths = sc.logged(A, Z, T, B, seed=2)
    losses = [float(core.train_step(z, actions, rewards, resets, lengths, lr=3e-3)[0]) for _ in range(60)]
    say("losses", losses[0], losses[-1])
    assert losses[-1] < 0.5 * losses[0] and np.isfinite(losses).all()
    pred = core.forward(z[:T].contiguous(), actions, resets)
    state = torch.zeros(B, H, device="cuda")
    for t in range(T):
        p, state = core.act(z[t], actions[t], state, resets[t])
        torch.testing.assert_close(p, pred[t], rtol=1e-4, atol=1e-4)
