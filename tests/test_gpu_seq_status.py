"""GPU tests of the device-side status for buffers without status words."""

import pytest
import torch

from paper_2205_01435_amd import _lib as wm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [0, 1, 16, 200, 256])
def test_a_recurrence_without_a_workspace(T):
    """Nothing is read for it: what lies beyond its (one) byte is another's."""
    bufs = wm.LinrecBuffers(T, 2, 70)
    assert bufs.ws_bytes == 0
    whole = torch.full((8192,), 255, dtype=torch.uint8, device="cuda")  # no status that a call left
    bufs.workspace = whole[:1]
    x = torch.ones(T, 2, 70, device="cuda")
    wm.linrec(x, x, bufs=bufs)
    wm.status(bufs)
    wm.linrec_grad(x, x, x, bufs=bufs)
    wm.status(bufs)
    assert bool((whole == 255).all())


def test_buffers_that_hold_no_status():
    for bufs in (wm.EmbedGradBuffers(9000, 5, 8), wm.LayerNormBuffers(100, 8), wm.ClipPlan([torch.ones(9, device="cuda")])):
        bufs.workspace.fill_(255)
        with pytest.raises(ValueError):
            wm.status(bufs)
