"""GPU tests of a clipping plan whose tensors change after it was made."""

import pytest
import torch

from paper_2205_01435_amd import _lib as wm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    wm.load()
    yield


@pytest.mark.parametrize("which", ["grads", "outs"])
def test_a_refused_plan_stays_refused(which):
    """A tensor that no longer fits is refused at every call, and the others
    are as they were: not clipped by a list without it."""
    grads = [torch.full((60,), float(i + 1), device="cuda") for i in range(5)]
    outs = [torch.full_like(g, 7.0) for g in grads]
    plan = wm.ClipPlan(grads, outs)
    good = (grads if which == "grads" else outs)[2].data
    (grads if which == "grads" else outs)[2].data = torch.ones(60, 2, device="cuda")[:, 0]  # not contiguous
    for _ in range(3):
        with pytest.raises(ValueError):
            wm.clip_grads(plan, 1e9)
    assert all(bool((o == 7.0).all()) for i, o in enumerate(outs) if i != 2)
    (grads if which == "grads" else outs)[2].data = good
    assert abs(float(wm.clip_grads(plan, 1e9)) - (60 * 55) ** 0.5) < 1e-4
    assert all(torch.equal(o, g) for o, g in zip(outs, grads))


def _guarded_pair(n):
    """A buffer with known values around a tensor of n, and the tensor."""
    whole = torch.full((n + 200,), 3.0, device="cuda")
    return whole, whole[100:100 + n]


@pytest.mark.parametrize("in_place", [True, False])
def test_a_shorter_tensor_at_the_same_address(in_place):
    whole, g = _guarded_pair(4000)
    out_whole, out = _guarded_pair(4000)
    plan = wm.ClipPlan([g], None if in_place else [out])
    wm.clip_grads(plan, 1e9)
    g.data = whole[100:1100]
    out.data = out_whole[100:1100]
    before = whole.clone()
    norm = wm.clip_grads(plan, 1.0)
    assert abs(float(norm) - 3 * 1000 ** 0.5) < 1e-4
    written = whole if in_place else out_whole
    assert bool((written[100:1100] < 1.0).all()) and bool((written[1100:] == 3.0).all()) and bool((written[:100] == 3.0).all())
    if not in_place:
        assert torch.equal(whole, before)


def test_another_type_at_the_same_address():
    whole = torch.full((1000,), 3.0, device="cuda")
    g = whole[:500]
    plan = wm.ClipPlan([g])
    halves = whole.view(torch.bfloat16)
    halves.fill_(2.0)
    g.data = halves[:500]  # as many values, half the bytes
    norm = wm.clip_grads(plan, 1.0)
    assert abs(float(norm) - 2 * 500 ** 0.5) < 1e-4
    assert bool((halves[:500] < 1.0).all()) and bool((halves[500:] == 2.0).all())


@pytest.mark.parametrize("which", ["grads", "outs"])
def test_other_strides_at_the_same_address(which):
    a, b = torch.ones(4, 6, device="cuda"), torch.zeros(4, 6, device="cuda")
    plan = wm.ClipPlan([a], [b])
    t = a if which == "grads" else b
    t.data = torch.as_strided(t, (4, 6), (1, 4))
    with pytest.raises(ValueError):
        wm.clip_grads(plan, 1.0)


def test_larger_tensors_than_the_plan_was_made_for():
    grads = [torch.ones(10, device="cuda") for _ in range(3)]
    plan = wm.ClipPlan(grads)
    for g in grads:
        g.data = torch.full((3000000,), 0.5, device="cuda")
    with pytest.raises(wm.WmError) as e:
        wm.clip_grads(plan, 1.0)
    assert e.value.status == wm.WM_ERR_WORKSPACE
    assert all(bool((g == 0.5).all()) for g in grads)


def test_more_and_fewer_tensors():
    grads = [torch.ones(50, device="cuda") for _ in range(4)]
    plan = wm.ClipPlan(grads)
    plan.grads.append(torch.ones(50, device="cuda"))
    with pytest.raises(wm.WmError) as e:  # more than the workspace serves
        wm.clip_grads(plan, 1e9)
    assert e.value.status == wm.WM_ERR_WORKSPACE
    del plan.grads[1:]
    assert abs(float(wm.clip_grads(plan, 1e9)) - 50 ** 0.5) < 1e-4
    plan = wm.ClipPlan([grads[0], grads[1]], [torch.zeros(50, device="cuda"), torch.zeros(50, device="cuda")])
    plan.grads.append(plan.outs.pop(0))  # the same tensors, other roles
    with pytest.raises(ValueError):
        wm.clip_grads(plan, 1e9)
    plan.outs = [torch.ones(50, device="cuda") for _ in range(2)]
    with pytest.raises(ValueError):
        wm.clip_grads(plan, 1e9)
    plan.outs = plan.grads
    plan.grads[0] = None
    with pytest.raises(ValueError):
        wm.clip_grads(plan, 1e9)
    del plan.grads[:]
    with pytest.raises(ValueError):
        wm.clip_grads(plan, 1e9)
