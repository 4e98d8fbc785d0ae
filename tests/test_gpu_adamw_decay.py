"""Weight decay of rates far below a unit of the weight's last place, summed over steps: what a schedule's end has."""
import pytest
import torch

import test_gpu_adamw as A
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
COUNT, STEPS, DECAY = 1 << 18, 50, 0.1


def held(t, q):
    """Moments as numbers, in 64 bits."""
    if t[q].element_size() == 4:
        return t[q].double()
    pad = t[q].view(torch.float8_e4m3fn).double().view(-1, 128)
    return (pad * t[q + "_scale"].double()[:, None]).view(-1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w,master", [("f32", False), ("bf16", True)])
@pytest.mark.parametrize("lr", [1e-5, 1e-6, 2.5e-7])
def test_decay_adds_up(bits, w, master, lr):
    """Every step's weight against its 64-bit value from the same weight and moments, rounded once to float as the formula has it (steps of less than half a unit of the weight's last place are
    lost in that rounding, whoever does it). What is off, along the weight, is decay that is lost or too much. The step s is off by some eight roundings of its own, 8 u |s| with u = 2^-24; that turns
    the rounding of the weight over, by a unit of its last place, for a share of 2 x 8 u |s| / unit of the elements: 16 u |s| |w| on average. |s| is 0.1 to 1 times lr here, and the mean of |w|
    over that of w^2 is 1.6: 16 u x 1e-5 x 1.6 = 1.5e-11 of the weight a step at most, 8e-10 in fifty. Allowed is ten times that; the smallest decay of fifty steps is 1.25e-6."""
    t = A.tensor(COUNT, w, "f32", master, bits, decay=DECAY, seed=11)
    gen = torch.Generator(device="cuda").manual_seed(12)
    opt = B.moe_adamw_list([t])
    off, decayed = 0.0, 0.0
    for step in range(1, STEPS + 1):
        t["g"].copy_(torch.randn(COUNT, device="cuda", generator=gen) * 1e-2)
        at = t["master"] if master else t["w"]
        before, g = at.double().clone(), t["g"].double()
        m, v = A.B1 * held(t, "m") + (1 - A.B1) * g, held(t, "v")
        v = A.B2 * (v * v if bits == 8 else v) + (1 - A.B2) * g * g
        part = lr * (m / (1 - A.B1 ** (100 + step))) / ((v / (1 - A.B2 ** (100 + step))).sqrt() + A.EPS)
        decay = lr * float(torch.tensor(DECAY)) * before
        B.moe_adamw(opt, lr, A.B1, A.B2, A.EPS, 100 + step, step)
        size = float(before.square().sum())
        off += float(((at.double() - (before - part - decay).float().double()) * before).sum()) / size
        decayed += float((decay * before).sum()) / size
    assert abs(off) <= 8e-9 and decayed >= 1.2e-6
