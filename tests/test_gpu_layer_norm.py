"""moe_layer_norm and moe_layer_norm_bwd against a plain 64-bit form, and their gradients against differences.

Tolerances: a sum of d or of T terms in threads and teams takes at most 40 roundings one behind the other and what follows 8 more, each of half a step of float of the magnitudes of the terms."""
import pytest
import torch

import training_reference as R
from block_reference import U, within
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
K = 48 * U


def data(T, d, act, seed=0, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)
    t = dict(x=(n(T, d) + mean).to(DT[act]), w=1 + 0.2 * n(d), b=0.3 * n(d), dxn=n(T, d).to(DT[act]), dres=n(T, d).to(DT[act]))
    return {q: v.cuda() for q, v in t.items()}


def forward(c, t, b=True, xn=None):
    T, d = t["x"].shape
    xn = torch.full_like(t["x"], 7.0) if xn is None else xn
    mean, rstd = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    B.moe_layer_norm(c, t["x"], t["w"], t["b"] if b else None, EPS, xn, mean, rstd)
    return xn, mean, rstd


def check_forward(t, b, got):
    xn, mean, rstd = got
    want, m, r = R.layer_norm(t["x"], t["w"], t["b"] if b else None, EPS)
    x, w = R.f64(t["x"]), R.f64(t["w"])
    row = x.abs().mean(1)
    within(mean, m, K * row, "mean")
    off = K * (x.abs() + row[:, None])                       # of a difference from the mean
    spread = (off * (x - m[:, None]).abs()).mean(1)          # of half the variance
    r_slack = r * (K + spread * r.square())
    within(rstd, r, r_slack, "rstd")
    slack = w.abs() * (off * r[:, None] + (x - m[:, None]).abs() * r_slack[:, None]) + K * want.abs()
    within(xn, want, slack + (K * R.f64(t["b"]).abs() if b else 0.0), "xn")


SIZES = [(1, 8, "bf16"), (1, 4, "f32"), (3, 64, "bf16"), (5, 72, "bf16"), (7, 68, "f32"), (33, 512, "bf16"), (130, 320, "f32"), (1000, 1024, "bf16"), (37, 1288, "f32"), (29, 2048, "bf16"),
         (19, 2056, "bf16"), (17, 2752, "bf16"), (9, 4096, "f32"), (11, 4104, "bf16"), (5, 8192, "bf16"), (6, 8196, "f32"), (4, 16384, "bf16"), (5, 16384, "f32"), (3001, 104, "f32")]


@pytest.mark.parametrize("T,d,act", SIZES)
def test_forward(T, d, act):
    t, c = data(T, d, act), B.make_config(T, d, d, 1, 1, act)
    check_forward(t, True, forward(c, t))
    check_forward(t, False, forward(c, t, b=False))
    bare = torch.full_like(t["x"], 7.0)
    B.moe_layer_norm(c, t["x"], t["w"], t["b"], EPS, bare, None, None)
    assert torch.equal(bare, forward(c, t)[0])


@pytest.mark.parametrize("T,d,act", SIZES + [(20000, 64, "bf16"), (9001, 512, "bf16"), (4000, 2048, "f32")])
@pytest.mark.parametrize("res", [False, True])
def test_backward(T, d, act, res):
    t, c = data(T, d, act), B.make_config(T, d, d, 1, 1, act)
    _, mean, rstd = forward(c, t)
    ws = B.empty_bytes(B.moe_layer_norm_workspace_bytes(c))
    ws.fill_(0xff)
    o = dict(dX=torch.full_like(t["x"], 7.0), dw=torch.full((d,), 7.0, device="cuda"), db=torch.full((d,), 7.0, device="cuda"))
    call = lambda o, db=True: B.moe_layer_norm_bwd(c, t["dxn"], t["x"], t["w"], mean, rstd, t["dres"] if res else None, o["dX"], o["dw"], o["db"] if db else None, ws)
    call(o)
    want = R.layer_norm_bwd(t["dxn"], t["x"], t["w"], mean, rstd, t["dres"] if res else None)
    for q, v in o.items():
        # a thread adds up the rows of one block and team: at most T / 100 of them beyond the 40
        within(v, want[q][0], (K + (T / 100) * U) * want[q][1], q)
    again = {q: torch.zeros_like(v) for q, v in o.items()}
    call(again)
    assert all(torch.equal(o[q], again[q]) for q in o)  # always the same sums
    again["db"].fill_(5.0)
    call(again, db=False)
    assert torch.equal(again["dw"], o["dw"]) and torch.equal(again["dX"], o["dX"]) and bool((again["db"] == 5.0).all())


def test_gradient_against_differences():
    T, d = 6, 40
    t, c = data(T, d, "f32", seed=3), B.make_config(T, d, d, 1, 1, "f32")
    _, mean, rstd = forward(c, t)
    o = [torch.zeros_like(t["x"]), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")]
    B.moe_layer_norm_bwd(c, t["dxn"], t["x"], t["w"], mean, rstd, None, *o, B.empty_bytes(B.moe_layer_norm_workspace_bytes(c)))
    loss = lambda x, w, b: (R.layer_norm(x, w, b, EPS)[0] * R.f64(t["dxn"])).sum()
    h = 1e-5
    args = [R.f64(t[q]) for q in ("x", "w", "b")]
    for i, got in enumerate(o):
        flat = args[i].view(-1)
        for j in range(0, flat.numel(), 7):
            keep = float(flat[j])
            flat[j] = keep + h
            up = loss(*args)
            flat[j] = keep - h
            down = loss(*args)
            flat[j] = keep
            # third derivatives of order 10 times h^2, differences of 64-bit sums over h, and the kernel's own roundings
            assert abs(float(got.view(-1)[j]) - float(up - down) / (2 * h)) < 1e-5, (i, j)


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_rows_far_from_zero(act):
    """A mean a thousand times the spread: the variance is that of the differences."""
    T, d = 40, 512
    t, c = data(T, d, act, mean=1000.0), B.make_config(T, d, d, 1, 1, act)
    check_forward(t, True, forward(c, t))


def test_constant_rows_and_rows_that_are_no_numbers():
    T, d = 16, 256
    t, c = data(T, d, "bf16"), B.make_config(T, d, d, 1, 1, "bf16")
    want = forward(c, t)
    t["x"][3] = 2.5
    t["x"][5] = 0.0
    t["x"][7, 9], t["x"][8, 100], t["x"][9, 255] = float("nan"), float("inf"), -float("inf")
    xn, mean, rstd = forward(c, t)
    other = [i for i in range(T) if i not in (3, 5, 7, 8, 9)]
    assert all(torch.equal(a[other], b[other]) for a, b in zip((xn, mean, rstd), want))
    for i, v in ((3, 2.5), (5, 0.0)):  # no spread: the bias alone
        assert torch.equal(xn[i], t["b"].bfloat16()) and float(mean[i]) == v
        within(rstd[i:i + 1], torch.tensor([EPS ** -0.5]), K * EPS ** -0.5, "rstd")
    assert xn[7].isnan().all() and xn[8].isnan().all() and xn[9].isnan().all()
    # such a row's gradient keeps to itself but for the weights'
    o = [torch.zeros_like(t["x"]), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")]
    B.moe_layer_norm_bwd(c, t["dxn"], t["x"], t["w"], mean, rstd, t["dres"], *o, B.empty_bytes(B.moe_layer_norm_workspace_bytes(c)))
    assert o[0][other].isfinite().all() and o[0][7].isnan().all() and o[1].isnan().all() and o[2].isfinite().all()


@pytest.mark.parametrize("T,d,act", [(37, 512, "bf16"), (50, 96, "f32"), (9, 4104, "bf16")])
def test_in_place(T, d, act):
    c = B.make_config(T, d, d, 1, 1, act)
    t = data(T, d, act)
    want, mean, rstd = forward(c, t)
    x = t["x"].clone()
    forward(c, t, xn=t["x"])
    assert torch.equal(t["x"], want)
    t["x"] = x
    ws = B.empty_bytes(B.moe_layer_norm_workspace_bytes(c))
    o = [torch.zeros_like(x), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")]
    B.moe_layer_norm_bwd(c, t["dxn"], x, t["w"], mean, rstd, t["dres"], *o, ws)
    for q in ("dxn", "x", "dres"):
        s = {k: v.clone() for k, v in t.items()}
        p = [s[q], torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")]
        B.moe_layer_norm_bwd(c, s["dxn"], s["x"], s["w"], mean, rstd, s["dres"], *p, ws)
        assert all(torch.equal(a, b) for a, b in zip(o, p)), q


def test_no_rows():
    c = B.make_config(0, 64, 64, 1, 1, "bf16")
    some = torch.zeros(64, 64, device="cuda", dtype=torch.bfloat16)  # (an empty tensor has no address)
    w, dw, db = torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    B.moe_layer_norm(c, some, w, None, EPS, some, None, None)
    B.moe_layer_norm_bwd(c, some, some, w, w, w, None, some, dw, db, B.empty_bytes(B.moe_layer_norm_workspace_bytes(c)))
    assert not dw.any() and not db.any()


def test_recorded_on_another_stream():
    T, d = 300, 512
    t, c = data(T, d, "bf16"), B.make_config(T, d, d, 1, 1, "bf16")
    xn, mean, rstd = forward(c, t)
    ws = B.empty_bytes(B.moe_layer_norm_workspace_bytes(c))
    o = [torch.zeros_like(xn), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")]

    def step():
        B.moe_layer_norm(c, t["x"], t["w"], t["b"], EPS, xn, mean, rstd)
        B.moe_layer_norm_bwd(c, t["dxn"], t["x"], t["w"], mean, rstd, t["dres"], *o, ws)

    step()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        step()
        graph.capture_end()
    for factor in (-1.5, 0.5):
        t["x"].mul_(factor)
        step()
        torch.cuda.synchronize()
        want = [v.clone() for v in (xn, mean, rstd, *o)]
        for v in (xn, mean, rstd, *o):
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((xn, mean, rstd, *o), want))


def test_nothing_is_written_outside():
    """Outputs in the middle of larger buffers."""
    for T, d, act in ((5, 72, "bf16"), (9, 1028, "f32"), (3, 4104, "bf16")):
        t, c = data(T, d, act), B.make_config(T, d, d, 1, 1, act)
        pad = 64
        big = {q: torch.full((n + 2 * pad,), 7.0, device="cuda", dtype=dt) for q, n, dt in (("xn", T * d, DT[act]), ("mean", T, torch.float32), ("rstd", T, torch.float32),
                                                                                           ("dX", T * d, DT[act]), ("dw", d, torch.float32), ("db", d, torch.float32))}
        v = {q: b[pad:-pad] for q, b in big.items()}
        B.moe_layer_norm(c, t["x"], t["w"], t["b"], EPS, v["xn"].view(T, d), v["mean"], v["rstd"])
        B.moe_layer_norm_bwd(c, t["dxn"], t["x"], t["w"], v["mean"], v["rstd"], t["dres"], v["dX"].view(T, d), v["dw"], v["db"], B.empty_bytes(B.moe_layer_norm_workspace_bytes(c)))
        for q, b in big.items():
            assert bool((b[:pad] == 7.0).all()) and bool((b[-pad:] == 7.0).all()), q
