"""moe_muon of lists whose shapes have segments of different lengths: what a matrix comes to does not depend on what it is taken together with."""
import pytest
import torch

from test_gpu_muon import check, copies, step, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shapes", [((3, 256, 1024), (8, 512, 512)), ((1, 1024, 1024), (8, 1024, 4096)), ((2, 256, 272), (5, 512, 1024), (4, 1200, 300), (2, 300, 330)),
                                    ((200, 160, 150), (30, 136, 600), (7, 800, 140))], ids=str)
@pytest.mark.parametrize("steps", [1, 4, 5, 7])
def test_alone_and_together(shapes, steps):
    t = [tensor(shape, seed=sum(shape)) for shape in shapes]
    before, alone = copies(t), copies(t)
    step(t, steps)
    for one in alone:
        step([one], steps)
    assert all(torch.equal(a[q], b[q]) for a, b in zip(t, alone) for q in ("w", "m"))
    if steps == 5 and shapes[0][1] < 1024:
        check(before, t)


def test_a_square_matrix_beside_wide_ones():
    """Off by what it is off alone: in segments of two and three steps it would be 2.8 times as much (8.9e-4 and 2.5e-3 of X, every rounding simulated in 64 bits)."""
    t = [tensor((2, 512, 512), seed=1), tensor((20, 512, 2048), seed=2)]
    before, alone = copies(t), copies(t[:1])
    step(t)
    step(alone)
    check(before, t)
    assert torch.equal(alone[0]["w"], t[0]["w"])
