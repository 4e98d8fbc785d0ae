"""moe_muon where updates are next to nothing: experts that get no rows any more, whose momentum falls by a factor every step until it is 0.

Tolerances are those of test_gpu_muon. (u of elements of 1e-39 is rounded by 2^-150, 7e-7 of them.)"""
import pytest
import torch

import training_reference as R
from block_reference import U, within
from paper_1701_06538_b200 import binding as B
from test_gpu_muon import DECAY, LR, MU, check, copies, step, tensor

pytestmark = pytest.mark.gpu
LEAST = 1.2e-38  # of eps
# by one block from beginning to end, by tiles of one SM, by tiles of two; rows in eights and not
SHAPES = [(2, 72, 96), (3, 13, 37), (1, 16, 4096), (2, 264, 200), (2, 300, 131)]


@pytest.mark.parametrize("types", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32")], ids=lambda t: "-".join(t))
@pytest.mark.parametrize("factor", [1e-12, 1e-16, 1e-18, 1e-21, 1e-27, 1e-32, 1e-36])
def test_small_gradients(factor, types):
    """1e-15 to 1e-39: their squares lose bits, are 0, and are the least numbers themselves."""
    t = [tensor(shape, *types, momentum=False, seed=sum(shape)) for shape in SHAPES]
    for one in t:
        one["g"] = (one["g"].double() * factor).to(one["g"].dtype)
    before = copies(t)
    step(t, eps=LEAST)
    check(before, t, eps=LEAST)


def test_elements_of_all_sizes():
    """Some columns of a matrix 1e-30 of the others: the large ones make the norm."""
    t = [tensor(shape, momentum=False, seed=3) for shape in SHAPES]
    for one in t:
        one["g"][..., ::3] *= 1e-30
        one["g"][..., 8:] *= 1e-10
    before = copies(t)
    step(t, eps=LEAST)
    # five columns are left. Directions that u has next to nothing in: as in test_low_rank, 0.15 of the norm that X begins with, beside five singular values of 0.7 or more at its end
    check(before, t, eps=LEAST, off=4e-3 + 0.15 / (0.7 * 5 ** 0.5))


@pytest.mark.parametrize("eps", [LEAST, 1e-36, 3e-36, 1e-30, 1e-7])
@pytest.mark.parametrize("nesterov", [True, False])
def test_zeros(eps, nesterov):
    """A matrix whose u is zero keeps its weights but for the decay, whatever eps is; its neighbours know nothing of it."""
    t = [tensor(tuple([3] + list(shape[1:])), seed=sum(shape)) for shape in SHAPES]
    want = copies(t)
    step(want, eps=eps, nesterov=nesterov)
    for one in t:
        one["g"][1], one["m"][1] = 0.0, 0.0
    before = copies(t)
    step(t, eps=eps, nesterov=nesterov)
    for a, b, w in zip(t, before, want):
        within(a["w"][1], R.f64(b["w"][1]) * (1 - LR * DECAY), 4 * U * R.f64(b["w"][1]).abs(), "decay alone")
        assert not a["m"][1].any()
        assert torch.equal(a["w"][::2], w["w"][::2]) and torch.equal(a["m"][::2], w["m"][::2])


def test_an_expert_that_gets_no_rows():
    """A thousand steps' worth of decay in eighty: momentum from 1e-3 to nothing."""
    t = [tensor((2, 72, 96), seed=5), tensor((1, 264, 200), seed=6)]
    for one in t:
        one["g"].zero_()
    L = B.moe_muon_list(t)
    ws = B.empty_bytes(B.moe_muon_workspace_bytes(L))
    for turn in range(80):
        for one in t:
            one["m"] *= 0.25
        before = copies(t)
        B.moe_muon(L, LR, MU, LEAST, 5, True, ws)
        assert all(one["w"].isfinite().all() for one in t), turn
        if float(before[0]["m"].abs().max()) > 1e-28:  # (below, small elements are no normal numbers)
            check(before, t, eps=LEAST)
    assert not any(one["m"].any() for one in t)
