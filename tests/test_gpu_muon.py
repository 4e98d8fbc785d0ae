"""moe_muon against the formulas in 64 bits.

Tolerances. Momentum and weights: a handful of float roundings of their terms. The orthogonalised update: a step's operands (X twice, A', B') are rounded to fp16, by 2^-11 / sqrt(3) at most in
root mean square, so 4 roundings are 5.7e-4 of X and, in quadrature, 2.8e-4; a later step multiplies an error of a singular value relative to it by |s p'(s) / p(s)|, at most 5 near s = 1.2
and below 2 from there on, so all of them together by less than 10: 4e-3 of X (2-norm), times scale and rate in the weights.
Steps in segments round powers of A instead of X: with every rounding simulated in 64 bits, normal matrices of 256 x 1024, 300 x 1200, 256 x 272 and 256 x 256 are off by 1.1e-3, 1.1e-3, 2.9e-3 and
3.2e-3 at most, over segments of 1, 2, 3, 1 + 3, 2 + 3, 3 + 3 and 1 + 3 + 3 steps."""
import pytest
import torch

import training_reference as R
from block_reference import U, half_step, within
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, MU, EPS, DECAY = 0.02, 0.95, 1e-7, 0.1
OFF = 4e-3


def tensor(shape, w="f32", g="f32", m="f32", master=False, seed=0, rank=None, scale=None, decay=DECAY, momentum=True):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen)
    rows, cols = shape[-2:]
    base = n(*shape) * 0.05
    grad = n(*shape) if rank is None else n(*shape[:-1], rank) @ n(*shape[:-2], rank, cols)
    t = dict(w=base.to(DT[w]).cuda(), g=(grad * 1e-3).to(DT[g]).cuda(), m=(n(*shape) * 1e-3 * momentum).to(DT[m]).cuda(), weight_decay=decay,
             scale=0.2 * max(rows, cols) ** 0.5 if scale is None else scale)
    if master:
        t["master"] = base.cuda()
    return t


def step(tensors, steps=5, nesterov=True, grad_scale=1.0, rates=None, lr=LR, mu=MU, eps=EPS, ws=None):
    L = B.moe_muon_list(tensors)
    if ws is None:
        ws = B.empty_bytes(B.moe_muon_workspace_bytes(L))
        ws.fill_(0xff)
    B.moe_muon(L, lr, mu, eps, steps, nesterov, ws, grad_scale, rates)
    assert B.moe_check_status(ws) == 0


def copies(tensors):
    return [{q: v.clone() if torch.is_tensor(v) else v for q, v in t.items()} for t in tensors]


def check(before, after, steps=5, nesterov=True, grad_scale=1.0, lr=LR, off=OFF, mu=MU, eps=EPS):
    for b, a in zip(before, after):
        three = lambda v: v if v.dim() == 3 else v[None]
        base = three(b.get("master", b["w"]))
        w, m, x = R.muon(base, three(b["g"]), three(b["m"]), lr, mu, eps, steps, nesterov, b["scale"], b["weight_decay"], grad_scale, b["m"].dtype)
        within(three(a["m"]), m, 4 * U * (R.f64(three(b["m"])).abs() + (R.f64(three(b["g"])) * grad_scale).abs()), "m")
        assert torch.equal(a["g"], b["g"])
        for q in ("w", "master"):
            if q not in a:
                continue
            got, size = three(a[q]).double().cpu(), lr * b["scale"] * x.flatten(1).norm(dim=1)
            # a half step of the type, four of float in the sum, and the products' error
            allowed = off * size + (half_step(a[q].dtype) + 4 * U) * (w.flatten(1).norm(dim=1) + size)
            worst = ((got - w).flatten(1).norm(dim=1) / allowed.clamp(min=1e-300)).max()
            assert float(worst) <= 1.0, (q, tuple(b["w"].shape), float(worst))
        if "master" in a:
            assert torch.equal(a["w"], a["master"].bfloat16())


SHAPES = [(1, 1, 1), (3, 1, 5), (2, 7, 1), (4, 2, 3), (5, 8, 8), (2, 13, 9), (3, 64, 64), (8, 64, 128), (3, 128, 64), (2, 72, 520), (2, 520, 72), (1, 128, 128), (2, 100, 1000), (2, 129, 129), (2, 130, 257),
          (3, 257, 130), (1, 192, 448), (2, 448, 192), (1, 320, 832), (1, 832, 320), (1, 256, 256), (1, 512, 1024), (1, 1024, 512), (1, 600, 650), (1, 1000, 1001), (1, 16, 4096), (1, 4096, 16), (40, 24, 40), (2, 65, 127), (2, 128, 768), (2, 768, 128), (3, 100, 769), (2, 385, 90), (150, 16, 200), (2, 513, 17), (2, 64, 768), (2, 768, 64), (2, 96, 512), (2, 512, 96), (2, 384, 128)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(shape):
    t = [tensor(shape, seed=sum(shape))]
    before = copies(t)
    step(t)
    check(before, t)


@pytest.mark.parametrize("w,g,m,master", [("f32", "f32", "f32", False), ("f32", "bf16", "bf16", False), ("bf16", "f32", "f32", False), ("bf16", "bf16", "bf16", False), ("bf16", "f32", "bf16", True),
                                          ("bf16", "bf16", "f32", True)])
@pytest.mark.parametrize("shape", [(3, 72, 136), (2, 264, 200), (2, 13, 37), (2, 300, 131)], ids=str)
def test_types(shape, w, g, m, master):
    t = [tensor(shape, w, g, m, master, seed=1)]
    before = copies(t)
    for nesterov in (True, False):
        now = copies(t)
        step(now, nesterov=nesterov, grad_scale=0.5)
        check(before, now, nesterov=nesterov, grad_scale=0.5)


@pytest.mark.parametrize("steps", [1, 2, 3, 8, 16])
def test_steps(steps):
    t = [tensor((2, 96, 200), seed=2), tensor((2, 300, 270), seed=3)]
    before = copies(t)
    step(t, steps=steps)
    # further steps keep singular values within 0.7 and 1.2 and multiply errors on as they go round there: by about 1.6 a step on average
    check(before, t, steps=steps, off=OFF * max(1.0, 1.6 ** (steps - 5)))


@pytest.mark.parametrize("shape", [(2, 8, 16), (2, 64, 128), (1, 16, 4096), (1, 192, 448), (1, 448, 192)], ids=str)
@pytest.mark.parametrize("w,g,m,master", [("f32", "f32", "f32", False), ("bf16", "bf16", "bf16", False), ("bf16", "f32", "bf16", True)])
def test_tensors_at_16_bytes(shape, w, g, m, master):
    """Slices of a model's layers begin where the layers before end."""
    t = [tensor(shape, w, g, m, master, seed=5)]
    whole = {}
    for q in [q for q, v in t[0].items() if torch.is_tensor(v)]:
        v = t[0][q]
        lead = 16 // v.element_size()
        whole[q] = torch.full((v.numel() + 2 * lead,), 7.0, dtype=v.dtype, device="cuda")
        whole[q][lead:-lead] = v.reshape(-1)
        t[0][q] = whole[q][lead:-lead].view(shape)
        assert t[0][q].data_ptr() % 32 == 16
    before = copies(t)
    step(t)
    check(before, t)
    for v in whole.values():
        lead = 16 // v.element_size()
        assert (v[:lead] == 7.0).all() and (v[-lead:] == 7.0).all()


def test_a_models_list():
    """Tensors of several layers, shapes mixed, some of no matrices; what is taken together does not change a result."""
    t = []
    for layer in range(3):
        t += [tensor((4, 72, 264), "bf16", "bf16", "f32", True, seed=10 * layer), tensor((4, 264, 72), "bf16", "bf16", "bf16", seed=10 * layer + 1), tensor((72, 4), seed=10 * layer + 2),
              tensor((0, 72, 264), seed=3), tensor((1, 300, 264), seed=10 * layer + 4, decay=0.0, scale=1.0)]
    before = copies(t)
    alone = copies(t)
    step(t)
    check([b for b in before if b["w"].numel()], [a for a in t if a["w"].numel()])
    for one in alone:
        if one["w"].numel():
            step([one])
    assert all(torch.equal(a[q], b[q]) for a, b in zip(t, alone) for q in ("w", "m"))


def test_more_tensors_than_a_launch_takes():
    t = [tensor((1 + i % 3, 24, 40), seed=i) for i in range(150)]
    before = copies(t)
    step(t)
    check(before, t)


def test_many_matrices_in_a_ring_of_scratch():
    """More matrices than the scratch has slots for, a few of them compared."""
    t = [tensor((900, 136, 152), "bf16", "bf16", "bf16", seed=4)]
    before = copies(t)
    step(t)
    pick = [0, 1, 447, 448, 898, 899]
    part = lambda l: [{q: v[pick] if torch.is_tensor(v) else v for q, v in l[0].items()}]
    check(part(before), part(t))
    again = copies(before)
    step(again)
    assert torch.equal(again[0]["w"], t[0]["w"])


def test_low_rank():
    """Experts with few rows. Directions that u has nothing in: rounding of every step leaves 2^-12.8 of X there, which the others multiply by 3.4 each until it meets 1, about 485 in all:
    root of five of them, 485 * 1.4e-4 * sqrt(5) = 0.15 of the norm |u| = 1 that X begins with, against sqrt(rank) = 4 at its end."""
    t = [tensor((2, 128, 256), rank=16, momentum=False, seed=5), tensor((2, 512, 256), rank=16, momentum=False, seed=6)]
    before = copies(t)
    step(t)
    check(before, t, off=OFF + 0.15 / 4)


def test_sizes_of_the_gradient():
    """The update does not know the gradient's size, as long as it is well above eps and its squares are floats."""
    for factor in (1e-15, 1e-3, 1e12):
        t = [tensor((2, 72, 96), momentum=False, seed=7)]
        t[0]["g"] *= factor
        before = copies(t)
        step(t, eps=1e-30)
        check(before, t, eps=1e-30)


def test_zeros_and_no_numbers():
    t = [tensor((6, 72, 200), seed=8), tensor((2, 300, 264), seed=9)]
    want = copies(t)
    step(want)
    t[0]["g"][1], t[0]["m"][1] = 0.0, 0.0
    t[0]["g"][3, 5, 7], t[0]["g"][4, 0, 0] = float("nan"), float("inf")
    t[1]["m"][1, 299, 263] = -float("inf")
    before = copies(t)
    step(t)
    within(t[0]["w"][1], R.f64(before[0]["w"][1]) * (1 - LR * DECAY), 4 * U * R.f64(before[0]["w"][1]).abs(), "decay alone")
    assert not t[0]["m"][1].any()
    for i in (0, 2, 5):
        assert torch.equal(t[0]["w"][i], want[0]["w"][i])
    assert torch.equal(t[1]["w"][0], want[1]["w"][0])
    for v in (t[0]["w"][3], t[0]["w"][4], t[1]["w"][1]):
        assert v.isnan().all()


def test_singular_values():
    """Of the step alone: between 0.7 and 1.2 (the coefficients' range) whatever they were between 1 and 1/500 of the largest."""
    gen = torch.Generator().manual_seed(11)
    u, v = torch.linalg.qr(torch.randn(256, 256, generator=gen))[0], torch.linalg.qr(torch.randn(320, 256, generator=gen))[0]
    s = torch.logspace(0, -1.3, 256)
    g = (u * s) @ v.T
    t = [dict(w=torch.zeros(256, 320, device="cuda"), g=g.cuda(), m=torch.zeros(256, 320, device="cuda"), scale=1.0, weight_decay=0.0)]
    step(t, lr=1.0)
    got = torch.linalg.svdvals(-t[0]["w"].double().cpu())
    assert 0.65 < float(got.min()) and float(got.max()) < 1.25


def test_rates_and_a_recorded_step():
    """Two recorded steps with workspaces of their own, replayed at once, read their rates when they run."""
    make = lambda: [tensor((5, 72, 136), "bf16", "bf16", "f32", True, seed=20), tensor((2, 264, 200), seed=21)]
    rates = torch.zeros(2, device="cuda")
    sets = [make(), make()]
    eager = make()
    lists = [B.moe_muon_list(t) for t in sets]
    spaces = [B.empty_bytes(B.moe_muon_workspace_bytes(l)) for l in lists]
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    step(make())
    torch.cuda.synchronize()
    for l, ws, s in zip(lists, spaces, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            g.capture_begin()
            B.moe_muon(l, 0.0, MU, EPS, 5, True, ws, 1.0, rates)
            g.capture_end()
        graphs.append(g)
    for lr, grad_scale in ((0.02, 1.0), (0.01, 0.25)):
        rates.copy_(torch.tensor([lr, grad_scale]))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        step(eager, lr=lr, grad_scale=grad_scale)
        torch.cuda.synchronize()
        for t in sets:
            for a, b in zip(t, eager):
                assert torch.equal(a["w"], b["w"]) and torch.equal(a["m"], b["m"])
        assert all(B.moe_check_status(ws) == 0 for ws in spaces)


def test_nothing_is_written_outside():
    for shape in ((2, 13, 37), (2, 130, 200), (1, 200, 132)):
        pad, n = 64, shape[0] * shape[1] * shape[2]
        src = tensor(shape, "bf16", "bf16", "bf16", True, seed=30)
        big = {q: torch.full((n + 2 * pad,), 7.0, device="cuda", dtype=src[q].dtype) for q in ("w", "m", "master")}
        for q, b in big.items():
            b[pad:-pad] = src[q].view(-1)
        t = dict(src, **{q: b[pad:-pad].view(shape) for q, b in big.items()})
        step([t])
        for q, b in big.items():
            assert bool((b[:pad] == 7.0).all()) and bool((b[-pad:] == 7.0).all()), (q, shape)
        L = B.moe_muon_list([t])
        need = B.moe_muon_workspace_bytes(L)
        room = torch.full((need + 4096,), 0x5a, device="cuda", dtype=torch.uint8)
        B.moe_muon(L, LR, MU, EPS, 5, True, room[:need])
        torch.cuda.synchronize()
        assert bool((room[need:] == 0x5a).all())


def test_lists_without_matrices():
    t = [tensor((0, 8, 16)), tensor((0, 200, 300))]
    before = copies(t)
    for tensors in ([], t):
        L = B.moe_muon_list(tensors)
        ws = B.empty_bytes(B.moe_muon_workspace_bytes(L))
        ws.fill_(0xff)
        B.moe_muon(L, LR, MU, EPS, 5, True, ws)
        assert bool((ws == 0xff).all())
    assert all(torch.equal(a["w"], b["w"]) for a, b in zip(t, before))


def test_steps_of_lists_with_wide_matrices():
    """Segments of every length, a rest of one or two steps before them, near-square matrices beside wide ones."""
    for steps in (1, 2, 3, 4, 6, 7):
        t = [tensor((3, 256, 1024), seed=steps), tensor((2, 1200, 300), seed=steps + 1), tensor((1, 256, 272), seed=steps + 2), tensor((1, 64, 256), seed=steps + 3)]
        before = copies(t)
        step(t, steps)
        check(before, t, steps)


def test_two_calls_at_once():
    """Two lists on two streams, each with its workspace."""
    lists = [[tensor((4, 256, 1024), seed=1), tensor((3, 64, 128), seed=2)], [tensor((3, 520, 200), seed=3), tensor((2, 72, 520), seed=4)]]
    before = [copies(t) for t in lists]
    made = [B.moe_muon_list(t) for t in lists]
    ws = [B.empty_bytes(B.moe_muon_workspace_bytes(L)) for L in made]
    streams = [torch.cuda.Stream() for _ in lists]
    torch.cuda.synchronize()
    for L, w, s in zip(made, ws, streams):
        with torch.cuda.stream(s):
            B.moe_muon(L, LR, MU, EPS, 5, True, w)
    torch.cuda.synchronize()
    for b, t, w in zip(before, lists, ws):
        assert B.moe_check_status(w) == 0
        check(b, t)


def test_a_workspace_that_is_too_small():
    t = [tensor((2, 200, 300))]
    L = B.moe_muon_list(t)
    with pytest.raises(ValueError):
        B.moe_muon(L, LR, MU, EPS, 5, True, torch.empty(1024, device="cuda", dtype=torch.uint8))
