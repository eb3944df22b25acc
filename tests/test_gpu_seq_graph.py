"""GPU test of the sequence-core operators under a captured graph: every kernel
that embedding, layer norm and clipping can launch, replayed with new inputs
and eager work in between, bit for bit."""

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from seqcheck import say

pytestmark = pytest.mark.gpu


def _embed(n, V, H, dtype):
    table = torch.empty(V, H, device="cuda", dtype=dtype)
    tok, dy = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, H, device="cuda", dtype=dtype)
    bufs, out = wm.EmbedGradBuffers(n, V, H), torch.empty(n, H, device="cuda", dtype=dtype)

    def fill(gen):
        table.normal_(generator=gen)
        dy.normal_(generator=gen)
        tok.random_(-1, V + 1, generator=gen)

    def run():
        wm.embed(table, tok, 2.0, out=out)
        wm.embed_grad(tok, dy, V, 2.0, bufs=bufs)
        return [out, bufs.grad]

    return fill, run


def _norm(rows, H, dtype):
    x, dy = (torch.empty(rows, H, device="cuda", dtype=dtype) for _ in range(2))
    gamma, beta = (torch.empty(H, device="cuda") for _ in range(2))
    bufs = wm.LayerNormBuffers(rows, H, dtype)

    def fill(gen):
        for t in (x, dy, gamma, beta):
            t.normal_(generator=gen)

    def run():
        wm.layer_norm(x, gamma, beta, bufs=bufs)
        wm.layer_norm_grad(x, dy, gamma, bufs=bufs)
        return [bufs.y, bufs.dx, bufs.dgamma, bufs.dbeta]

    return fill, run


def _clip(sizes):
    grads = [torch.empty(n, device="cuda", dtype=torch.bfloat16 if i % 3 else torch.float32) for i, n in enumerate(sizes)]
    plan = wm.ClipPlan(grads, [torch.empty_like(g) for g in grads])

    def fill(gen):
        for g in grads:
            g.normal_(generator=gen)

    def run():
        wm.clip_grads(plan, 1.0)
        return [plan.norm, *plan.outs]

    return fill, run


@pytest.mark.parametrize("what", [
    (_embed, 300, 40, 70, torch.float32), (_embed, 3000, 40, 70, torch.bfloat16), (_embed, 3000, 900, 300, torch.float32),
    (_embed, 20000, 900, 300, torch.bfloat16), (_norm, 33, 50, torch.float32), (_norm, 3000, 1003, torch.bfloat16),
    (_clip, [5000 + i for i in range(200)]), (_clip, [3, 100001]),
], ids=str)
def test_replays(what):
    say("graph", what)
    fill, run = what[0](*what[1:])
    gen = torch.Generator(device="cuda").manual_seed(3)
    s = torch.cuda.Stream()
    fill(gen)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        outs = run()
    for i in range(4):
        fill(gen)
        eager = [t.clone() for t in run()]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b), i
