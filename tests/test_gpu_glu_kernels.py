"""GPU tests of which kernel each product of the gated projection takes, by the
names of its launches: on both sides of the rows, tiles, types and alignments that
decide, so that the tests of values at these sizes are tests of these kernels."""

import pytest
import torch

from paper_2205_01435_amd import _lib as wm
from seqcheck import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


CASES = [  # rows, D, F, dtype, columns behind the rows of x, kernels of outputs, dx and dW
    (256, 64, 96, "bf16", 0, "few", "128", "128"), (257, 64, 96, "bf16", 0, "128", "128", "128"),
    (256, 64, 96, "fp32", 0, "few", "128", "128"), (257, 64, 96, "fp32", 0, "128", "128", "128"),
    (4200, 1000, 2100, "bf16", 0, "256", "256", "256"), (4200, 1000, 2100, "fp32", 0, "128", "128", "128"),
    (4352, 1024, 2304, "bf16", 0, "256", "256", "256"),
    # 10 and 9 x 16 tiles of outputs
    (2305, 256, 2048, "bf16", 0, "256", "128", "128"), (2304, 256, 2048, "bf16", 0, "128", "128", "128"),
    # 4 x 16 and 4 x 15 tiles of dx
    (3841, 1024, 256, "bf16", 0, "128", "256", "128"), (3840, 1024, 256, "bf16", 0, "128", "128", "128"),
    # 16 x 4 tiles of dW, and 15 x 4; rows of x that are no multiple of 8, off and on 16-byte boundaries
    (2048, 1024, 1921, "bf16", 0, "128", "128", "128"), (2048, 1024, 1924, "bf16", 0, "128", "128", "256"),
    (2048, 1024, 1920, "bf16", 0, "128", "128", "128"), (2047, 1024, 1924, "bf16", 0, "128", "128", "128"),
    (4096, 1001, 4012, "bf16", 0, "128", "128", "128"), (4096, 1001, 4012, "bf16", 7, "128", "128", "256"),
]


@pytest.mark.parametrize("rows,D,F,dtype,wide,out,dx,dW", CASES)
def test_kernels(rows, D, F, dtype, wide, out, dx, dW):
    say("glu kernels", rows, D, F, dtype, wide)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, W = torch.randn(rows, D + wide, device="cuda").to(dt)[:, :D], torch.randn(2 * F, D, device="cuda").to(dt)
    bufs = wm.GluBuffers(rows, D, F, dt)
    wm.profile_reset()
    wm.profile_enable("glu")
    wm.glu(x, W, bufs=bufs)
    wm.glu_grad(x, W, bufs.h.clone(), bufs=bufs)
    torch.cuda.synchronize()
    got = {n: [k for k in ("few", "128", "256") if wm.profile_read(f"{n}/{k}")[1] == 1] for n in ("glu", "glu_dx", "glu_dw")}
    total = sum(wm.profile_read(n)[1] for n in ("glu/", "glu_dx/", "glu_dw/"))
    wm.profile_enable(None)
    wm.profile_reset()
    assert got == {"glu": [out], "glu_dx": [dx], "glu_dw": [dW]} and total == 3, got
