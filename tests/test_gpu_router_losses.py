"""moe_router_losses against a plain 64-bit form, its gradient against that form's and against differences, and the way of the gradient through the gate.

Tolerances: a probability takes about ten roundings (the difference from the largest, exponential, sum over at most 40 roundings, quotient), sums of them over a block's rows a rounding a row at
most (T / 500 and eight), each half a step of float; a gradient is p times a difference of terms of the size of the largest c and of the z loss' factor."""
import math

import pytest
import torch

import training_reference as R
from block_reference import U, within
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
WB, WZ = 0.02, 0.003
K = 64 * U


def data(T, n, k, S=0, keep=False, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    logits = spread * torch.randn(T, n, generator=g) + 0.5 * torch.randn(n, generator=g)
    idx = (logits + 0.3 * torch.randn(T, n, generator=g)).topk(k, dim=1).indices.int()
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8) if keep else None
    offsets = None
    if S:
        offsets = torch.cat([torch.randint(0, 3, (1,), generator=g), torch.randint(0, T + 1, (S,), generator=g)]).sort().values.int()
    return logits, idx, mask, offsets


def run(logits, idx, keep, offsets, grad=True, sums=True, k=None):
    T, n = logits.shape
    S = 1 if offsets is None else len(offsets) - 1
    c = B.make_config(T, 64, 64, n, idx.shape[1], "bf16")
    cu = lambda t: None if t is None else t.cuda()
    o = dict(losses=torch.full((2,), 7.0, device="cuda"), counts=torch.full((S, n), -7, dtype=torch.int32, device="cuda"), prob_sums=torch.full((S, n), 7.0, device="cuda") if sums else None,
             dlogits=torch.full((T, n), 7.0, device="cuda") if grad else None)
    ws = B.empty_bytes(B.moe_router_losses_workspace_bytes(c, S))
    ws.fill_(0xff)
    B.moe_router_losses(c, cu(logits), cu(idx), cu(keep), cu(offsets), S, WB, WZ, o["losses"], o["counts"], o["prob_sums"], o["dlogits"], ws)
    return o


def check(logits, idx, keep, offsets, o):
    T, n = logits.shape
    x = logits.double().requires_grad_(True)
    losses, counts, sums, live = R.router_losses(x, idx, keep, offsets, WB, WZ)
    assert torch.equal(o["counts"].cpu().long(), counts)
    within(o["prob_sums"], sums, (K + (T / 500) * U) * sums, "prob_sums")
    within(o["losses"], losses.detach(), (K + (T / 500) * U) * losses.detach(), "losses")
    if o["dlogits"] is None:
        return
    want, = torch.autograd.grad(losses.sum() + 0.0 * x[0, 0], x)  # (where nothing is live the losses are no function of x)
    want = torch.nan_to_num(want)  # (rows of nothing but -inf)
    p = torch.nan_to_num(torch.softmax(x.detach(), 1))
    L = max(int(live.sum()), 1)
    per = counts.sum(1).clamp(min=1).double() / idx.shape[1]
    largest = (WB * n / (idx.shape[1] * L) * counts.max(1).values / per).max()
    z = 2 * WZ / L * torch.nan_to_num(torch.logsumexp(x.detach(), 1).abs(), posinf=0.0, neginf=0.0)
    within(o["dlogits"], want, K * p * (2 * largest + 2 * z[:, None]), "dlogits")
    assert not o["dlogits"].cpu()[~live].any()


CASES = [(1, 1, 1, 0, False), (1, 2, 2, 0, False), (24, 32, 4, 0, False), (5, 7, 3, 2, True), (64, 16, 2, 0, True), (300, 8, 1, 4, False), (257, 33, 8, 5, True), (500, 64, 2, 0, False),
         (333, 100, 4, 3, True), (700, 128, 2, 9, True), (129, 130, 2, 0, False), (200, 256, 4, 20, False), (65, 500, 8, 0, True), (40, 515, 4, 3, False), (33, 1000, 2, 0, False), (17, 1023, 3, 2, True),
         (21, 1028, 4, 0, False), (9, 2047, 8, 3, False), (13, 2048, 2, 0, True), (7, 4099, 4, 2, False), (6, 8192, 8, 0, False), (5000, 20, 3, 37, True), (6000, 128, 2, 0, False), (900, 4, 4, 300, False)]


@pytest.mark.parametrize("T,n,k,S,keep", CASES)
def test_against_the_formula(T, n, k, S, keep):
    a = data(T, n, k, S, keep)
    o = run(*a)
    check(*a, o)
    again = run(*a)
    assert all(torch.equal(o[q], again[q]) for q in o)
    bare = run(*a, grad=False, sums=False)
    assert torch.equal(bare["losses"], o["losses"]) and torch.equal(bare["counts"], o["counts"])


def test_sequences_are_batches():
    """Every sequence by itself, weighted by its tokens."""
    logits, idx, keep, _ = data(400, 48, 3, 0, True, seed=4)
    ends = [0, 100, 100, 130, 400]
    o = run(logits, idx, keep, torch.tensor(ends, dtype=torch.int32))
    total = 0.0
    for s in range(4):
        a, b = ends[s], ends[s + 1]
        if a == b:
            assert not o["counts"][s].any() and not o["prob_sums"][s].any()
            continue
        one = run(logits[a:b].contiguous(), idx[a:b].contiguous(), keep[a:b].contiguous(), None)
        assert torch.equal(one["counts"][0], o["counts"][s])
        total += float(one["losses"][0]) * int(keep[a:b].sum())
    assert abs(total / int(keep.sum()) - float(o["losses"][0])) < 100 * U * float(o["losses"][0])


def test_even_loads_cost_their_weight():
    n, k = 16, 2
    logits = torch.zeros(64, n)
    idx = torch.stack([torch.arange(64) % n, (torch.arange(64) + 1) % n], 1).int()
    o = run(logits, idx, None, None)
    assert abs(float(o["losses"][0]) - WB) < 100 * U * WB
    z = 2 * WZ * math.log(n) / 64  # a row's sum: of the z loss alone, lse being log n
    assert float((o["dlogits"].sum(1) - z).abs().max()) < 100 * U * z
    assert bool((o["counts"] == 64 * k // n).all())


def test_padding_sequences_and_masks_that_leave_nothing():
    logits, idx, _, _ = data(90, 24, 2, seed=7)
    for offsets in ([0, 90], [10, 40, 40, 70], [0, 0, 0], [90, 90], [0, 60, 30], [5, 5, 80]):
        off = torch.tensor(offsets, dtype=torch.int32)
        for keep in (None, torch.zeros(90, dtype=torch.uint8), (torch.arange(90) % 3 == 0).to(torch.uint8) * 255):
            a = (logits.clone(), idx, keep, off)
            o = run(*a)
            check(*a, o)
            # what is not live is not read
            _, _, _, live = R.router_losses(logits.double(), idx, keep, off, WB, WZ)
            a[0][~live] = float("nan")
            dead = idx.clone()
            dead[~live] = 1 << 30
            other = run(a[0], dead, keep, off)
            assert all(torch.equal(o[q], other[q]) for q in o)
            if not live.any():
                assert not o["losses"].any() and not o["dlogits"].any()


def test_offsets_outside_the_batch():
    logits, idx, _, _ = data(50, 12, 2, seed=8)
    o = run(logits, idx, None, torch.tensor([-5, 20, 900], dtype=torch.int32))
    want = run(logits, idx, None, torch.tensor([0, 20, 50], dtype=torch.int32))
    assert all(torch.equal(o[q], want[q]) for q in o)


@pytest.mark.parametrize("n", [12, 33, 160, 2048])
def test_shut_experts(n):
    logits, idx, _, _ = data(70, n, 2, seed=9)
    logits[:, 3] = -float("inf")
    logits[5] = -float("inf")        # nothing left
    logits[6, 1:] = -float("inf")    # one expert left
    logits[7] = torch.finfo(torch.float32).min
    idx[8, 0], idx[9, 1] = -1, n     # dropped choices
    o = run(logits, idx, None, None)
    x = logits.double()
    losses, counts, sums, _ = R.router_losses(x, idx, None, None, WB, WZ)
    assert torch.equal(o["counts"].cpu().long(), counts)
    within(o["prob_sums"], sums, 2 * K * sums, "prob_sums")
    assert not o["dlogits"][5].any() and not o["dlogits"][torch.arange(70) != 7, 3].any()
    assert o["dlogits"][torch.arange(70) != 7].isfinite().all()
    within(o["losses"][:1], losses[:1], 2 * K * losses[:1], "balance")


def test_rows_that_are_no_numbers():
    logits, idx, _, _ = data(30, 40, 2, seed=10)
    want = run(logits, idx, None, None)
    logits[4, 7], logits[11, 0] = float("nan"), float("inf")
    o = run(logits, idx, None, None)
    other = [i for i in range(30) if i not in (4, 11)]
    assert torch.equal(o["dlogits"][other], want["dlogits"][other]) and torch.equal(o["counts"], want["counts"])
    assert o["dlogits"][4].isnan().all() and o["dlogits"][11].isnan().any() and o["losses"].isnan().all()


def test_large_logits():
    """Differences of logits of some hundred: probabilities of one and of almost nothing."""
    a = data(60, 48, 2, spread=150.0, seed=11)
    o = run(*a)
    assert o["dlogits"].isfinite().all()
    # x - top is exact to half a step of 300, and exp turns that into as much of p: 2^-24 * 300 relative
    x = a[0].double().requires_grad_(True)
    losses, counts, sums, _ = R.router_losses(x, a[1], None, None, WB, WZ)
    within(o["losses"], losses.detach(), 400 * 2 * U * losses.detach(), "losses")
    want, = torch.autograd.grad(losses.sum(), x)
    lse = torch.logsumexp(x.detach(), 1)[:, None]
    size = torch.softmax(x.detach(), 1) * (2 * WZ / 60 * lse.abs() + 2 * WB * 48 / 120 * counts.max() / 60)
    # (what is below float's smallest normal number may be 0)
    within(o["dlogits"], want, 800 * 2 * U * size + 2.0 ** -126, "dlogits")


def test_gradient_against_differences():
    logits, idx, keep, offsets = data(12, 10, 2, 2, True, seed=12)
    o = run(logits, idx, keep, offsets)
    x, h = logits.double(), 1e-5
    for t in range(12):
        for j in range(10):
            up, down = x.clone(), x.clone()
            up[t, j] += h
            down[t, j] -= h
            f = lambda v: float(R.router_losses(v, idx, keep, offsets, WB, WZ)[0].sum())
            # third derivatives times h^2 and 64-bit differences over h are below 1e-10; the rest is float's
            assert abs(float(o["dlogits"][t, j]) - (f(up) - f(down)) / (2 * h)) < 1e-9 + 1e-6 * abs(float(o["dlogits"][t, j]))


def test_recorded_with_a_workspace_of_its_own():
    T, n, k = 1000, 64, 4
    logits, idx, keep, offsets = [None if v is None else v.cuda() for v in data(T, n, k, 7, True, seed=13)]
    c = B.make_config(T, 64, 64, n, k, "bf16")
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    run(logits.cpu(), idx.cpu(), keep.cpu(), offsets.cpu())
    torch.cuda.synchronize()
    for s in streams:
        o = dict(losses=torch.zeros(2, device="cuda"), counts=torch.zeros(7, n, dtype=torch.int32, device="cuda"), prob_sums=torch.zeros(7, n, device="cuda"), dlogits=torch.zeros(T, n, device="cuda"))
        ws = B.empty_bytes(B.moe_router_losses_workspace_bytes(c, 7))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            g.capture_begin()
            B.moe_router_losses(c, logits, idx, keep, offsets, 7, WB, WZ, o["losses"], o["counts"], o["prob_sums"], o["dlogits"], ws)
            g.capture_end()
        graphs.append((g, ws))
        outs.append(o)
    for turn in range(3):
        logits.mul_(0.9)
        torch.cuda.synchronize()
        for (g, _), s in zip(graphs, streams):  # both at once
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = run(logits.cpu(), idx.cpu(), keep.cpu(), offsets.cpu())
        for o in outs:
            assert all(torch.equal(o[q], want[q]) for q in o), turn


# ------------------------------------------------------------------------------------------ the gradient's way through the gate
def gate_inputs(T, d, n, k, act, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[act]
    x = torch.randn(T, d, generator=g).to(dt).cuda()
    Wg, Wn = [(torch.randn(d, n, generator=g) * d ** -0.5 * s).cuda() for s in (1.0, 0.3)]
    noise = torch.randn(T, n, generator=g).cuda()
    return x, Wg, Wn, noise


@pytest.mark.parametrize("T,d,n,k,act", [(40, 64, 8, 2, "f32"), (300, 128, 20, 3, "bf16"), (500, 64, 64, 2, "bf16"), (2500, 128, 128, 4, "bf16"), (260, 64, 256, 8, "bf16"), (100, 64, 300, 2, "f32"),
                                         (5000, 64, 32, 2, "bf16"), (700, 64, 96, 2, "bf16")])
def test_gate_bwd_added(T, d, n, k, act):
    x, Wg, Wn, noise = gate_inputs(T, d, n, k, act)
    c = B.make_config(T, d, 64, n, k, act)
    S = B.moe_query_sizes(c)
    ws = B.empty_bytes(S.ws_bytes)
    e = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)
    idx, gates, clean, raw, kv, ki = e(T, k, dt=torch.int32), e(T, k), e(T, n), e(T, n), e(T, 2), e(T, 2, dt=torch.int32)
    B.moe_gate(c, x, Wg, Wn, noise, idx, gates, clean, raw, kv, ki, ws)
    gen = torch.Generator().manual_seed(5)
    dgates, dload = torch.randn(T, k, generator=gen).cuda(), (0.1 * torch.randn(n, generator=gen)).cuda()
    more = torch.randn(T, n, generator=gen).cuda()

    def bwd(added, plain=False):
        o = dict(dWg=e(d, n), dWn=e(d, n), dX=e(T, d))
        args = (c, x, Wg, Wn, noise, clean, raw, idx, gates, kv, ki, dgates.clone(), dload)
        if plain:
            B.moe_gate_bwd(*args, o["dWg"], o["dWn"], o["dX"], ws)
        else:
            B.moe_gate_bwd_added(*args, added, o["dWg"], o["dWn"], o["dX"], ws)
        return o

    plain, none, both = bwd(None, plain=True), bwd(None), bwd(more)
    assert all(torch.equal(plain[q], none[q]) for q in plain)
    assert torch.equal(both["dWn"], plain["dWn"])  # of the clean logits alone
    dx, dw = more.double() @ Wg.double().T, x.double().T @ more.double()
    # the products of the gate's backward pass are held to 1e-5 of their size; here the difference of two of them
    for q, want in (("dX", dx), ("dWg", dw)):
        off = (both[q].double() - plain[q].double() - want).norm() / (plain[q].double().norm() + want.norm())
        assert float(off) < 3e-5, q


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("T,d,h,n,k,act", [(48, 64, 72, 6, 2, "f32"), (700, 64, 128, 16, 2, "bf16")])
def test_backward_added(T, d, h, n, k, act, layer):
    """The fused call adds what the losses over its own context's logits give."""
    x, Wg, Wn, noise = gate_inputs(T, d, n, k, act, seed=1)
    g = torch.Generator().manual_seed(2)
    W1, b1, W2, b2 = [(torch.randn(*s, generator=g) * f).to(x.dtype).cuda() for s, f in (((n, d, h), d ** -0.5), ((n, h), 0.1), ((n, h, d), h ** -0.5), ((n, d), 0.1))]
    dY = torch.randn(T, d, generator=g).to(x.dtype).cuda()
    keep = torch.randint(0, 256, (T, d // 8), generator=g, dtype=torch.uint8).cuda()
    c = B.make_config(T, d, h, n, k, act)
    S = B.moe_query_sizes(c)
    ctx, ws = B.empty_bytes(S.ctx_bytes), B.empty_bytes(max(S.ws_fwd_bytes, S.ws_bwd_bytes))
    e = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)
    y, losses, imp, load, counts = torch.zeros_like(x), e(2), e(n), e(n), e(n, dt=torch.int32)
    if layer:
        B.moe_layer_forward(c, x, Wg, Wn, noise, W1, b1, W2, b2, keep, 0.3, y, losses, imp, load, counts, ctx, ws)
    else:
        B.moe_forward(c, x, Wg, Wn, noise, W1, b1, W2, b2, y, losses, imp, load, counts, ctx, ws)
    v = B.ctx_views(c, ctx)
    r = dict(losses=e(2), counts=e(1, n, dt=torch.int32), prob_sums=e(1, n), dlogits=e(T, n))
    clean = v["clean"].view(T, n)
    B.moe_router_losses(c, clean, v["topk_idx"], None, None, 1, 3.0, 1.0, r["losses"], r["counts"], r["prob_sums"], r["dlogits"], B.empty_bytes(B.moe_router_losses_workspace_bytes(c)))
    assert torch.equal(r["counts"][0], counts)  # the dispatch's

    def bwd(added):
        o = [torch.zeros_like(x), e(d, n), e(d, n)] + [torch.zeros_like(t) for t in (W1, b1, W2, b2)]
        a = (c, dY, x, Wg, Wn, noise, W1, b1, W2, b2)
        if layer:
            B.moe_layer_backward_added(*a, keep, 0.3, ctx, added, *o, ws)
        else:
            B.moe_backward_added(*a, ctx, added, *o, ws)
        return o

    plain, both = bwd(None), bwd(r["dlogits"])
    for i in range(2, 7):
        assert torch.equal(plain[i], both[i])
    want = x.double().T @ r["dlogits"].double()
    assert float((both[1].double() - plain[1].double() - want).norm() / (want.norm() + plain[1].double().norm())) < 3e-5
    dx = r["dlogits"].double() @ Wg.double().T
    off = (both[0].double() - plain[0].double() - dx).abs()
    step = torch.finfo(x.dtype).eps / 2 * (both[0].double().abs() + plain[0].double().abs())
    assert bool((off <= step * 1.01 + 3e-5 * (dx.abs().max() + plain[0].double().abs().max())).all())
