"""Every place that the outputs of the norms may take among the inputs."""
import itertools

import pytest
import torch

import test_gpu_norms as N
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
# rows of a warp (with and without its gate in the ring) and of several; one row and more than a block's
SHAPES = [(1, 64, "bf16"), (300, 72, "bf16"), (700, 512, "f32"), (150, 2056, "bf16"), (70, 8200, "f32")]


@pytest.mark.parametrize("T,d,act", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_norm_in_bwd(T, d, act, residual):
    cfg, t = N.config(T, d, act), N.tensors(T, d, act, 21)
    r = torch.empty(T, device="cuda")
    B.moe_norm_in(cfg, t["x"], t["w"], N.EPS, N.empty(t["x"]), r)
    ws = B.empty_bytes(B.moe_norm_workspace_bytes(cfg))

    def run(place):
        u = {q: t[q].clone() for q in ("dNext", "x", "dOut")}
        dX, dw = u.get(place, N.empty(t["x"])), torch.full((d,), 7.0, device="cuda")
        ws.fill_(0xff)
        B.moe_norm_in_bwd(cfg, u["dNext"], u["x"], t["w"], r, u["dOut"] if residual else None, dX, dw, ws)
        for q, v in u.items():
            assert q == place or torch.equal(v, t[q]), q  # the others are only read
        return dX, dw

    want = run(None)
    for place in ("dNext", "x") + (("dOut",) if residual else ()):
        got = run(place)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), place


@pytest.mark.parametrize("T,d,act", SHAPES)
@pytest.mark.parametrize("with_next", [True, False])
@pytest.mark.parametrize("per", [0, 1, 40, -1])
def test_norm_out_bwd(T, d, act, with_next, per):
    per = T if per < 0 else per
    cfg, t = N.config(T, d, act), N.tensors(T, d, act, 22, -(-T // per) if per else 0)
    f = N.forward(cfg, t, per, 0.7, with_next)
    want = N.backward(cfg, t, f, per, 0.7, with_next)
    places = ["dOut", "y"] + (["dNext", "out"] if with_next else [])
    for a, b in itertools.product([None] + places, repeat=2):
        if a is not None and a == b:
            continue
        u = {q: v.clone() if torch.is_tensor(v) else v for q, v in t.items()}
        u["out"] = f[0].clone()
        got = N.backward(cfg, u, (u["out"],) + f[1:], per, 0.7, with_next, dX=u.get(a), dY=u.get(b))
        for q, v in want.items():
            assert v is None or torch.equal(got[q], v), (a, b, q)
        for q in places:
            assert q in (a, b) or torch.equal(u[q], f[0] if q == "out" else t[q]), (a, b, q)


@pytest.mark.parametrize("T,d,act", SHAPES)
@pytest.mark.parametrize("per", [0, 1, -1])
def test_norm_out(T, d, act, per):
    per = T if per < 0 else per
    cfg, t = N.config(T, d, act), N.tensors(T, d, act, 23, -(-T // per) if per else 0)
    want = N.forward(cfg, t, per)
    for a, b in itertools.product([None, "x", "y"], repeat=2):
        if a is not None and a == b:
            continue
        u = dict(t, x=t["x"].clone(), y=t["y"].clone())
        got = N.forward(cfg, u, per, out=u.get(a), nxt=u.get(b))
        for g, v in zip(got, want):
            assert torch.equal(g, v), (a, b)
        for q in ("x", "y"):
            assert q in (a, b) or torch.equal(u[q], t[q]), (a, b)
