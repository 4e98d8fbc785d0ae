"""moe_muon with up to sixteen steps, on updates for which the number of steps can be told from the result. The polynomial has a cycle of four values that singular values near it fall into,
0.682, 1.134, 0.753, 1.047: errors of them shrink to a sixth every four steps. With orthogonal rows all singular values are one, s, which eps puts where s comes to that cycle soon: then
X is a multiple of u whose factor says how many steps were taken, and a step too many or too few, two or three, are off by 4 % at least.

Tolerance: four roundings a step are 5.7e-4 of X (see test_gpu_muon); what a step is off by is, n - j steps later, that times the product of |s p'(s) / p(s)| on the way where it is along s, and
itself in all other directions, which neither grow nor shrink. The sum of all steps', one by one."""
import pytest
import torch

import training_reference as R
from test_gpu_muon import MU, step

pytestmark = pytest.mark.gpu
A, B3, C5 = R.NS
ROUNDINGS = 5.7e-4


def p(s):
    return s * (A + B3 * s ** 2 + C5 * s ** 4)


def growth(s):
    return abs(s * (A + 3 * B3 * s ** 2 + 5 * C5 * s ** 4) / p(s))


def tolerance(s, steps):
    at = [s]
    for _ in range(steps):
        at.append(p(at[-1]))
    total = 0.0
    for j in range(steps):
        along = 1.0
        for i in range(j, steps):
            along *= growth(at[i])
        total += ROUNDINGS * max(1.0, along)
    return total, at


def start(M):
    """Singular values of u over its norm are M^-1/2; eps can make them less."""
    return min((M ** -0.5 * (1.0 - i / 400) for i in range(1, 200)), key=lambda s: max(tolerance(s, n)[0] for n in (8, 13, 16)))


def test_the_cycle():
    s = 1.047
    for _ in range(8):
        s = p(s)
    ring = [s, p(s), p(p(s)), p(p(p(s)))]
    assert abs(p(ring[3]) - s) < 1e-5 and [round(v, 2) for v in sorted(ring)] == [0.68, 0.75, 1.05, 1.13]
    assert growth(ring[0]) * growth(ring[1]) * growth(ring[2]) * growth(ring[3]) < 1 / 5


@pytest.mark.parametrize("shape", [(2, 256, 1024), (1, 1024, 256), (2, 96, 200), (1, 16, 4096), (1, 300, 330), (1, 150, 1200)], ids=str)
@pytest.mark.parametrize("steps", [5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16])
def test_steps(shape, steps):
    count, rows, cols = shape
    M, gen = min(rows, cols), torch.Generator().manual_seed(rows + steps)
    q = torch.linalg.qr(torch.randn(count, max(rows, cols), M, generator=gen, dtype=torch.float64))[0]
    q = q.mT if rows <= cols else q
    s = start(M)
    tol, at = tolerance(s, steps)
    g = (1e-3 * q).float().contiguous()
    norm = 1e-3 * (1 + MU) * M ** 0.5
    w = torch.zeros(shape, device="cuda")
    step([dict(w=w, g=g.cuda(), m=torch.zeros(shape, device="cuda"), scale=1.0, weight_decay=0.0)], steps, lr=1.0, eps=norm * (M ** -0.5 / s - 1))
    off = lambda n: float((R.f64(-w) - at[n] * q).norm() / (at[n] * q).norm())
    assert off(steps) < tol < 0.03
    at.append(p(at[-1]))
    for other in range(max(steps - 3, 0), steps + 2):
        if other != steps:
            assert off(other) > 2 * tol, other
    # and the formula itself says so
    x = R.muon(torch.zeros(shape), g, torch.zeros(shape), 1.0, MU, norm * (M ** -0.5 / s - 1), steps, True, 1.0, 0.0, 1.0, torch.float32)[2]
    assert float((x - at[steps] * q).norm() / x.norm()) < 1e-4
