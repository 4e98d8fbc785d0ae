"""moe_norm_in / moe_norm_out and their backward passes against the same in 64 bits.

Tolerance: an element is half a step of its type off, and float arithmetic: a row's sums go through at most 32 elements in a thread, five steps of a warp and 16
warps, the products and square root around them make it less than 64 roundings; values made from two such sums 128; sums over rows add eight rows of
a thread and eight teams. 160 u times the magnitudes of the terms covers each."""
import pytest
import torch

import block_reference as R
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-6
K = 160 * R.U
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# from one token and one vector a row to rows of several warps, odd numbers of vectors, more rows than a wave of blocks
SHAPES = [(1, 8, "bf16"), (1, 4, "f32"), (3, 512, "bf16"), (37, 72, "bf16"), (64, 264, "f32"), (131, 1032, "bf16"), (9, 1028, "f32"), (33, 4104, "bf16"), (5, 16384, "bf16"),
          (5, 16384, "f32"), (2, 8200, "f32"), (700, 320, "f32"), (2085, 256, "bf16")]


def tensors(T, d, act, seed=0, groups=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T + d)
    f = lambda *s, std=1.0, mean=0.0, dt=DT[act]: (torch.randn(*s, device="cuda", generator=g) * std + mean).to(dt)
    t = dict(x=f(T, d), y=f(T, d, std=0.5), dOut=f(T, d), dNext=f(T, d), w=f(d, std=0.3, mean=1.0, dt=torch.float32), w_next=f(d, std=0.3, mean=1.0, dt=torch.float32))
    t["gate"] = f(groups, d, std=0.5, mean=0.5) if groups else None
    return t


def config(T, d, act):
    return B.make_config(T, d, d, 1, 1, act)


def empty(like):
    return torch.full_like(like, 7.0)


def forward(cfg, t, per=0, scale=0.7, with_next=True, out=None, nxt=None):
    T = cfg.T
    out = empty(t["x"]) if out is None else out
    nxt = (empty(t["x"]) if nxt is None else nxt) if with_next else None
    r, r2 = torch.empty(T, device="cuda"), torch.empty(T, device="cuda") if with_next else None
    B.moe_norm_out(cfg, t["x"], t["y"], t["w"], t["gate"], per, scale, t["w_next"] if with_next else None, EPS, out, nxt, r, r2)
    return out, nxt, r, r2


@pytest.mark.parametrize("T,d,act", SHAPES)
def test_norm_in(T, d, act):
    t, cfg = tensors(T, d, act), config(T, d, act)
    xn, r = empty(t["x"]), torch.empty(T, device="cuda")
    B.moe_norm_in(cfg, t["x"], t["w"], EPS, xn, r)
    want, rstd = R.norm_in(t["x"], t["w"], EPS)
    R.within(xn, want, K * want.abs(), "xn")
    R.within(r, rstd, K * rstd, "rstd")
    again = t["x"].clone()
    B.moe_norm_in(cfg, again, t["w"], EPS, again, None)  # in place, no rstd
    assert torch.equal(again, xn)


@pytest.mark.parametrize("T,d,act", SHAPES)
@pytest.mark.parametrize("with_next", [True, False])
@pytest.mark.parametrize("per", [0, 1, 3, -1])
def test_norm_out(T, d, act, with_next, per):
    per = T if per < 0 else per
    t, cfg = tensors(T, d, act, 1, -(-T // per) if per else 0), config(T, d, act)
    out, nxt, r, r2 = forward(cfg, t, per, 0.7, with_next)
    want, want_next, rstd, rstd_next, terms = R.norm_out(t["x"], t["y"], t["w"], t["gate"], per, 0.7, t["w_next"] if with_next else None, EPS)
    R.within(out, want, K * terms, "out")
    R.within(r, rstd, K * rstd, "rstd")
    if with_next:
        ratio = (terms.norm(dim=1) / want.norm(dim=1))[:, None].clamp(min=1.0)  # of what the sum of squares is made of to what it is
        R.within(r2, rstd_next, 2 * K * rstd_next * ratio[:, 0], "rstd_next")
        R.within(nxt, want_next, 2 * K * terms * rstd_next[:, None] * t["w_next"].double().cpu().abs() * ratio, "next")
    x, y = t["x"].clone(), t["y"].clone()  # results in the place of the inputs
    u = dict(t, x=x, y=y)
    a, b, _, _ = forward(cfg, u, per, 0.7, with_next, out=y, nxt=x)
    assert torch.equal(a, out) and (not with_next or torch.equal(b, nxt))


def backward(cfg, t, f, per=0, scale=0.7, with_next=True, dX=None, dY=None):
    d = cfg.d
    o = dict(dX=empty(t["x"]) if dX is None else dX, dY=empty(t["x"]) if dY is None else dY, dw=torch.full((d,), 7.0, device="cuda"))
    o["dgate"] = empty(t["gate"]) if t["gate"] is not None else None
    o["dw_next"] = torch.full((d,), 7.0, device="cuda") if with_next else None
    ws = B.empty_bytes(B.moe_norm_workspace_bytes(cfg))
    ws.fill_(0xff)
    out, _, r, r2 = f
    B.moe_norm_out_bwd(cfg, t["dOut"], t["dNext"] if with_next else None, out if with_next else None, t["y"], t["w"], t["gate"], per, scale, t["w_next"] if with_next else None,
                       r, r2, o["dX"], o["dY"], o["dw"], o["dgate"], o["dw_next"], ws)
    return o


@pytest.mark.parametrize("T,d,act", SHAPES)
@pytest.mark.parametrize("with_next", [True, False])
@pytest.mark.parametrize("per", [0, 1, 3, 20, 100, -1])
def test_norm_out_bwd(T, d, act, with_next, per):
    per = T if per < 0 else per
    t, cfg = tensors(T, d, act, 2, -(-T // per) if per else 0), config(T, d, act)
    f = forward(cfg, t, per, 0.7, with_next)
    o = backward(cfg, t, f, per, 0.7, with_next)
    want = R.norm_out_bwd(t["dOut"], t["dNext"] if with_next else None, f[0], t["y"], t["w"], t["gate"], per, 0.7, t["w_next"] if with_next else None, f[2], f[3])
    for q, (value, terms) in want.items():
        R.within(o[q], value, K * terms, q)
    again = backward(cfg, t, f, per, 0.7, with_next)  # fixed orders of all sums
    for q in want:
        assert torch.equal(o[q], again[q]), q
    u = {q: v.clone() if torch.is_tensor(v) else v for q, v in t.items()}  # results in the place of the inputs
    third = backward(cfg, u, f, per, 0.7, with_next, dX=u["dOut"], dY=u["y"])
    for q in want:
        assert torch.equal(o[q], third[q]), q


@pytest.mark.parametrize("T,d,act", SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_norm_in_bwd(T, d, act, residual):
    t, cfg = tensors(T, d, act, 3), config(T, d, act)
    xn, r = empty(t["x"]), torch.empty(T, device="cuda")
    B.moe_norm_in(cfg, t["x"], t["w_next"], EPS, xn, r)
    dX, dw, ws = empty(t["x"]), torch.full((d,), 7.0, device="cuda"), B.empty_bytes(B.moe_norm_workspace_bytes(cfg))
    dres = t["dOut"] if residual else None
    B.moe_norm_in_bwd(cfg, t["dNext"], t["x"], t["w_next"], r, dres, dX, dw, ws)
    want = R.norm_out_bwd(t["dOut"] if residual else torch.zeros_like(t["dOut"]), t["dNext"], t["x"], None, t["w"], None, 0, 1.0, t["w_next"], None, r)
    R.within(dX, want["dX"][0], K * want["dX"][1], "dX")
    R.within(dw, want["dw_next"][0], K * want["dw_next"][1], "dw")


@pytest.mark.parametrize("per", [0, 2, 6])
def test_gradients_against_differences(per):
    """The derivative along a random direction of all inputs: (f(+s) - f(-s)) / 2s in 64 bits against the kernel's gradients. With s = 1e-4 the difference is off by s^2 of the
    third derivative, 1e-7 or so of the value's terms; the gradients carry K of theirs."""
    T, d = 6, 64
    t, cfg = tensors(T, d, "f32", 4, -(-T // per) if per else 0), config(T, d, "f32")
    f = forward(cfg, t, per, 0.7)
    o = backward(cfg, t, f, per, 0.7)
    names = dict(x="dX", y="dY", w="dw", w_next="dw_next", **({"gate": "dgate"} if per else {}))
    g = torch.Generator().manual_seed(5)
    way = {q: torch.randn(t[q].shape, generator=g, dtype=torch.float64) for q in names}

    def loss(s):
        v = {q: t[q].double().cpu() + s * way[q] if q in way else None for q in ("x", "y", "w", "w_next", "gate")}
        out, nxt, *_ = R.norm_out(v["x"], v["y"], v["w"], v["gate"], per, 0.7, v["w_next"], EPS)
        return float((out * t["dOut"].double().cpu()).sum() + (nxt * t["dNext"].double().cpu()).sum())

    s = 1e-4
    want = (loss(s) - loss(-s)) / (2 * s)
    parts = [float((o[n].double().cpu() * way[q]).sum()) for q, n in names.items()]
    terms = sum(float((o[n].double().cpu() * way[q]).abs().sum()) for q, n in names.items())
    assert abs(sum(parts) - want) <= (10 * K + 1e-6) * terms


def test_rows_that_are_all_zero_or_not_finite():
    """A row of zeros has rstd 1 / sqrt(eps) and stays 0; a row with an infinity or NaN is its own affair."""
    T, d = 5, 512
    t, cfg = tensors(T, d, "bf16", 6), config(T, d, "bf16")
    clean = forward(cfg, t)
    t["x"][1], t["y"][1] = 0.0, 0.0
    t["y"][3, 7], t["x"][4, 9] = float("inf"), float("nan")
    out, nxt, r, r2 = forward(cfg, t)
    assert not out[1].any() and not nxt[1].any() and torch.isfinite(r[1]) and torch.isfinite(r2[1])
    assert abs(float(r[1]) - EPS ** -0.5) <= 4 * R.U * EPS ** -0.5
    assert torch.isnan(nxt[4]).all()
    for row in (0, 2):
        assert torch.equal(out[row], clean[0][row]) and torch.equal(nxt[row], clean[1][row])


def test_rows_behind_the_last_are_left():
    T, d = 7, 72
    t, cfg = tensors(T, d, "bf16", 7, 3), config(T, d, "bf16")
    big = torch.full((T + 3, d), 5.0, device="cuda", dtype=torch.bfloat16)
    forward(cfg, t, 3, out=big[:T])
    assert (big[T:] == 5.0).all()


def test_recorded_in_a_graph_and_on_another_stream():
    T, d = 260, 512
    t, cfg = tensors(T, d, "bf16", 8, 1), config(T, d, "bf16")
    f = forward(cfg, t, T)
    want = backward(cfg, t, f, T)
    ws = B.empty_bytes(B.moe_norm_workspace_bytes(cfg))
    got = {q: torch.zeros_like(v) for q, v in want.items()}
    out, nxt, r, r2 = (torch.zeros_like(v) for v in f)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        B.moe_norm_out(cfg, t["x"], t["y"], t["w"], t["gate"], T, 0.7, t["w_next"], EPS, out, nxt, r, r2)
        B.moe_norm_out_bwd(cfg, t["dOut"], t["dNext"], out, t["y"], t["w"], t["gate"], T, 0.7, t["w_next"], r, r2, got["dX"], got["dY"], got["dw"], got["dgate"], got["dw_next"], ws)
        graph.capture_end()
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, f[0]) and torch.equal(nxt, f[1])
    for q in want:
        assert torch.equal(want[q], got[q]), q


def test_no_rows():
    cfg, d = config(0, 64, "f32"), 64
    t = tensors(1, d, "f32", 9)
    dX, dw, r, ws = empty(t["x"]), torch.full((d,), 7.0, device="cuda"), torch.ones(1, device="cuda"), B.empty_bytes(B.moe_norm_workspace_bytes(cfg))
    B.moe_norm_in(cfg, t["x"], t["w"], EPS, dX, r)
    B.moe_norm_in_bwd(cfg, t["dNext"], t["x"], t["w"], r, None, dX, dw, ws)
    assert (dX == 7.0).all() and not dw.any()


# Shares of many rows: groups whole in a team (one or several, blocks of fewer teams), in a block, in chunks; several waves; rows of one and of several warps. A thread adds up to some 400
# rows one by one: 600 u instead of 160
@pytest.mark.parametrize("T,d,act,per", [(40000, 72, "bf16", 1), (40000, 72, "bf16", 5), (40000, 72, "bf16", 37), (40000, 72, "bf16", 64), (40000, 72, "bf16", 301), (40000, 72, "bf16", 5000),
                                         (40000, 72, "bf16", 0), (20000, 512, "f32", 1), (20000, 512, "f32", 67), (20000, 1024, "bf16", 33), (20000, 1024, "bf16", 200), (20000, 1024, "bf16", 1000),
                                         (6000, 1544, "bf16", 70), (6000, 1544, "bf16", 1), (6000, 1544, "bf16", 0), (3000, 2064, "f32", 13), (2000, 8200, "bf16", 40)])
def test_shares_of_many_rows(T, d, act, per):
    t, cfg = tensors(T, d, act, 5, -(-T // per) if per else 0), config(T, d, act)
    f = forward(cfg, t, per, 0.7)
    o = backward(cfg, t, f, per, 0.7)
    want = R.norm_out_bwd(t["dOut"], t["dNext"], f[0], t["y"], t["w"], t["gate"], per, 0.7, t["w_next"], f[2], f[3])
    for q, (value, terms) in want.items():
        R.within(o[q], value, 600 * R.U * terms, q)
    again = backward(cfg, t, f, per, 0.7)
    for q in want:
        assert torch.equal(o[q], again[q]), q


@pytest.mark.parametrize("T,d,act", [(9001, 72, "bf16"), (7000, 512, "bf16"), (5003, 1024, "bf16"), (1201, 4096, "bf16"), (900, 2056, "bf16"), (9001, 320, "f32"), (1500, 2048, "f32"), (700, 8192, "bf16")])
def test_several_rows_a_team(T, d, act):
    cfg = config(T, d, act)
    for per in (0, 1, 100):
        test_norm_out(T, d, act, True, per)
    test_norm_out(T, d, act, False, 7)
    test_norm_in(T, d, act)
    # rows behind the last are left
    t = tensors(T, d, act)
    big = torch.full((T + 3, d), 3.0, device="cuda", dtype=DT[act])
    B.moe_norm_in(cfg, t["x"], t["w"], EPS, big[:T], None)
    assert (big[T:] == 3.0).all()
