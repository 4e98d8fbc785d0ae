"""The block's operators one behind the other, as a program uses them: norm, layer for a few tokens, output norm with the next block's; and a training step of norm, layer, output norm,
their backward passes and AdamW."""
import numpy as np
import pytest
import torch

import block_reference as R
import test_gpu_adamw as A
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS, SCALE = 1e-6, 0.8
K = 160 * R.U  # as in test_gpu_norms.py


def make(rng, *shape, std=1.0, mean=0.0, dt=torch.float32):
    return torch.from_numpy(rng.standard_normal(shape) * std + mean).to(dt)


def weights(d, h, n, act, seed, gate_rows):
    """On the host, so that the same numbers go into every form."""
    rng, dt = np.random.default_rng(seed), DT[act]
    return dict(w_in=make(rng, d, std=0.2, mean=1.0), Wg=make(rng, d, n, std=d ** -0.5), W1=make(rng, n, d, h, std=d ** -0.5, dt=dt), b1=make(rng, n, h, std=0.3, dt=dt),
                W2=make(rng, n, h, d, std=h ** -0.5, dt=dt), b2=make(rng, n, d, std=0.3, dt=dt), w=make(rng, d, std=0.2, mean=1.0), gate=make(rng, gate_rows, d, std=0.4, mean=0.6, dt=dt),
                w_next=make(rng, d, std=0.2, mean=1.0))


# ------------------------------------------------------------------------------------------ serving
class Server:
    """Two blocks; a block's output norm gives the next one's input."""

    def __init__(self, T, d, h, n, k, act):
        self.cfg = B.make_config(T, d, h, n, k, act)
        self.blocks = [{q: v.cuda() for q, v in weights(d, h, n, act, seed, T).items()} for seed in (1, 2)]
        self.x = make(np.random.default_rng(T), T, d, dt=DT[act]).cuda()
        e = lambda: torch.full_like(self.x, 7.0)
        f = lambda: torch.full((T,), 7.0, device="cuda")
        self.xn, self.r = e(), f()
        self.o = [dict(y=e(), out=e(), next=e(), rstd=f(), rstd_next=f(), idx=torch.full((T, k), -1, dtype=torch.int32, device="cuda"), gates=torch.zeros(T, k, device="cuda"))
                  for _ in self.blocks]
        self.ws = B.empty_bytes(B.moe_few_workspace_bytes(self.cfg))
        self.ws.fill_(0xff)

    def step(self):
        c = self.cfg
        x, xn = self.x, self.xn
        B.moe_norm_in(c, x, self.blocks[0]["w_in"], EPS, xn, self.r)
        for w, o in zip(self.blocks, self.o):
            B.moe_forward_few(c, xn, w["Wg"], w["W1"], w["b1"], w["W2"], w["b2"], o["y"], o["idx"], o["gates"], self.ws)
            B.moe_norm_out(c, x, o["y"], w["w"], w["gate"], 1, SCALE, w["w_next"], EPS, o["out"], o["next"], o["rstd"], o["rstd_next"])
            x, xn = o["out"], o["next"]

    def outputs(self):
        return [self.xn, self.r] + [o[q] for o in self.o for q in sorted(o)]


@pytest.mark.parametrize("T,d,h,n,k,act", [(1, 512, 256, 32, 4, "bf16"), (24, 264, 136, 9, 3, "bf16"), (64, 128, 256, 20, 2, "bf16"), (7, 68, 100, 5, 2, "f32")])
def test_blocks_that_serve(T, d, h, n, k, act):
    s = Server(T, d, h, n, k, act)
    s.step()
    assert B.moe_check_status(s.ws) == 0
    want, rstd = R.norm_in(s.x, s.blocks[0]["w_in"], EPS)
    R.within(s.xn, want, K * want.abs(), "xn")
    x, xn = s.x, s.xn
    for w, o in zip(s.blocks, s.o):  # every call against its own inputs
        y, slack, gates, gate_slack = R.few(xn, w["Wg"], w["W1"], w["b1"], w["W2"], w["b2"], k, o["idx"])
        R.within(o["gates"], gates, gate_slack, "gates")
        R.within(o["y"], y, slack, "y")
        out, nxt, r, r2, terms = R.norm_out(x, o["y"], w["w"], w["gate"], 1, SCALE, w["w_next"], EPS)
        R.within(o["out"], out, K * terms, "out")
        ratio = (terms.norm(dim=1) / out.norm(dim=1))[:, None].clamp(min=1.0)
        R.within(o["next"], nxt, 2 * K * terms * r2[:, None] * w["w_next"].double().cpu().abs() * ratio, "next")
        x, xn = o["out"], o["next"]

    # recorded, on another stream, and replayed on other inputs
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        s.step()
        graph.capture_end()
    for factor in (-1.5, 0.25):
        s.x.mul_(factor)
        s.step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in s.outputs()]
        for t in s.outputs():
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert B.moe_check_status(s.ws) == 0
        for a, b in zip(s.outputs(), eager):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------ training
class Trainer:
    def __init__(self, T, d, h, n, k, act, per, seed=3):
        self.T, self.per = T, per
        self.cfg = B.make_config(T, d, h, n, k, act, w_importance=0.0, w_load=0.0, flags=B.MOE_FLAG_GATE_SCREEN_OFF)
        rng, dt = np.random.default_rng(seed + 100), DT[act]
        self.host = weights(d, h, n, act, seed, -(-T // per))
        self.w = {q: v.cuda() for q, v in self.host.items()}
        self.io = {q: make(rng, T, d, dt=dt) for q in ("x", "dOut", "dNext")}
        self.t = {q: v.cuda() for q, v in self.io.items()}
        S = B.moe_query_sizes(self.cfg)
        self.ctx = B.empty_bytes(S.ctx_bytes)
        self.ws = B.empty_bytes(max(S.ws_fwd_bytes, S.ws_bwd_bytes, B.moe_norm_workspace_bytes(self.cfg)))  # in turn by all calls of the stream
        e = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)
        self.zero, self.no_noise = e(d, n), e(T, n)
        self.o = {q: torch.zeros_like(self.t["x"]) for q in ("xn", "y", "out", "next", "dX", "dY", "dxn")}
        self.o.update(losses=e(2), importance=e(n), load=e(n), counts=e(n, dt=torch.int32), r_in=e(T), rstd=e(T), rstd_next=e(T), dWnoise=e(d, n))
        self.g = {q: torch.zeros_like(v) for q, v in self.w.items()}

    def forward(self):
        c, w, o = self.cfg, self.w, self.o
        B.moe_norm_in(c, self.t["x"], w["w_in"], EPS, o["xn"], o["r_in"])
        B.moe_forward(c, o["xn"], w["Wg"], self.zero, self.no_noise, w["W1"], w["b1"], w["W2"], w["b2"], o["y"], o["losses"], o["importance"], o["load"], o["counts"], self.ctx, self.ws)
        B.moe_norm_out(c, self.t["x"], o["y"], w["w"], w["gate"], self.per, SCALE, w["w_next"], EPS, o["out"], o["next"], o["rstd"], o["rstd_next"])

    def backward(self):
        c, w, o, g = self.cfg, self.w, self.o, self.g
        B.moe_norm_out_bwd(c, self.t["dOut"], self.t["dNext"], o["out"], o["y"], w["w"], w["gate"], self.per, SCALE, w["w_next"], o["rstd"], o["rstd_next"], o["dX"], o["dY"], g["w"],
                           g["gate"], g["w_next"], self.ws)
        B.moe_backward(c, o["dY"], o["xn"], w["Wg"], self.zero, self.no_noise, w["W1"], w["b1"], w["W2"], w["b2"], self.ctx, o["dxn"], g["Wg"], o["dWnoise"], g["W1"], g["b1"], g["W2"],
                       g["b2"], self.ws)
        B.moe_norm_in_bwd(c, o["dxn"], self.t["x"], w["w_in"], o["r_in"], o["dX"], o["dX"], g["w_in"], self.ws)

    def loss(self):
        return float(sum((self.o[a].double() * self.t[b].double()).sum() for a, b in (("out", "dOut"), ("next", "dNext"))))


def in_64_bits(tr, k):
    """The same block by torch's own derivatives: gradients, the routing, and the smallest distances to another routing and to a unit's border."""
    leaf = {q: v.double().requires_grad_() for q, v in {**tr.host, "x": tr.io["x"]}.items()}
    norm = lambda x, w: x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * w
    T = tr.T
    xn = norm(leaf["x"], leaf["w_in"])
    logits = xn @ leaf["Wg"]
    top = logits.topk(k + 1, 1)
    idx = top.indices[:, :k]
    gates = torch.softmax(logits.gather(1, idx), 1)
    y, edge = 0.0, float((top.values[:, k - 1] - top.values[:, k]).min().detach())
    border = 1e30
    for s in range(k):
        e = idx[:, s]
        pre = torch.einsum("td,tdh->th", xn, leaf["W1"][e]) + leaf["b1"][e]
        border = min(border, float(pre.abs().min().detach()))
        y = y + gates[:, s:s + 1] * (torch.einsum("th,thd->td", pre.clamp(min=0.0), leaf["W2"][e]) + leaf["b2"][e])
    out = SCALE * leaf["x"] + leaf["gate"][torch.arange(T) // tr.per] * norm(y, leaf["w"])
    nxt = norm(out, leaf["w_next"])
    ((out * tr.io["dOut"].double()).sum() + (nxt * tr.io["dNext"].double()).sum()).backward()
    return out.detach(), nxt.detach(), {q: v.grad for q, v in leaf.items()}, idx, edge, border


def off(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


TRAIN = (96, 64, 48, 6, 2)


def test_gradients_of_the_block():
    """Seven float stages, each within 160 u = 1e-5 of the magnitudes of its terms; what is summed over 96 rows of both signs is up to some twenty times smaller than its terms: 2e-3. A
    term that is missing, or a wrong link, is a hundred times that. The inputs are such that no rounding changes the routing or a unit's side of 0."""
    k = TRAIN[4]
    tr = Trainer(*TRAIN, "f32", 32, seed=4)
    out, nxt, grads, idx, edge, border = in_64_bits(tr, k)
    assert edge > 1e-4 and border > 1e-5
    tr.forward()
    assert torch.equal(B.ctx_views(tr.cfg, tr.ctx)["topk_idx"].cpu().long(), idx)
    tr.backward()
    assert B.moe_check_status(tr.ws) == 0
    assert off(tr.o["out"], out) < 1e-4 and off(tr.o["next"], nxt) < 1e-4
    for q, want in grads.items():
        assert off(tr.o["dX"] if q == "x" else tr.g[q], want) < 2e-3, q

    # against differences, along the gradient itself. A step of 0.02 / |g| moves an element by 3e-4: a few units change sides, whose error is of second order
    for q in ("x", "w_in", "W1", "gate"):
        at, g = (tr.t["x"], tr.o["dX"].clone()) if q == "x" else (tr.w[q], tr.g[q].clone())
        size, start, values = float(g.double().norm()), at.clone(), []
        for sign in (1.0, -1.0):
            at.copy_(start + sign * 0.02 / size * g)
            tr.forward()
            values.append(tr.loss())
        at.copy_(start)
        assert abs((values[0] - values[1]) / 0.04 - size) < 1e-2 * size, q


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_that_train(bits):
    """bf16 weights with float masters. Every step's AdamW against its 64-bit form on the gradients at hand; then the same two steps as replays of one graph, bit for bit."""
    def start():
        tr = Trainer(200, 128, 256, 16, 4, "bf16", 50)
        ts = []
        for q, w in tr.w.items():
            pad = torch.zeros(-(-w.numel() // 128), device="cuda")
            t = dict(w=w.view(-1), g=tr.g[q].view(-1), weight_decay=0.1 if w.dim() > 1 else 0.0, master=w.float().view(-1).clone() if w.dtype == torch.bfloat16 else None)
            if bits == 8:
                codes = lambda: torch.zeros(w.numel(), device="cuda").to(torch.float8_e4m3fn)
                t.update(m=codes(), v=codes(), m_scale=pad.clone(), v_scale=pad.clone())
            else:
                t.update(m=torch.zeros(w.numel(), device="cuda"), v=torch.zeros(w.numel(), device="cuda"))
            ts.append(t)
        return tr, ts, B.moe_adamw_list(ts)

    tr, ts, opt = start()
    for step in (1, 2):
        tr.forward()
        tr.backward()
        before = A.copy(ts)
        B.moe_adamw(opt, A.LR, A.B1, A.B2, A.EPS, step, 70 + step)
        torch.cuda.synchronize()
        assert B.moe_check_status(tr.ws) == 0
        A.check(before, ts, step, 70 + step)
        assert all(float(t["g"].float().abs().max()) > 0 for t in ts)

    again, ts2, opt2 = start()
    rates, side, graph = torch.zeros(5, device="cuda"), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        again.forward()
        again.backward()
        B.moe_adamw(opt2, A.LR, A.B1, A.B2, A.EPS, 0, rates=rates)
        graph.capture_end()
    for step in (1, 2):
        rates[:4] = torch.tensor([A.LR, 1 - A.B1 ** step, 1 - A.B2 ** step, 1.0])
        rates[4:].view(torch.int32).fill_(70 + step)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    for a, b in zip(ts, ts2):
        for q in a:
            if torch.is_tensor(a[q]):
                assert torch.equal(a[q].view(torch.uint8), b[q].view(torch.uint8)), q


def test_tensors_of_another_device_are_refused(monkeypatch):
    s, tr = Server(2, 64, 64, 4, 2, "bf16"), Trainer(8, 64, 48, 4, 2, "f32", 4)
    t = torch.zeros(256, device="cuda")
    opt = B.moe_adamw_list([dict(w=t, g=t.clone(), m=t.clone(), v=t.clone())])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)  # of tensors on device 0
    w, o, c = s.blocks[0], s.o[0], s.cfg
    g, q, tc = tr.g, tr.o, tr.cfg
    for call in (lambda: B.moe_norm_in(c, s.x, w["w_in"], EPS, s.xn, s.r),
                 lambda: B.moe_forward_few(c, s.xn, w["Wg"], w["W1"], w["b1"], w["W2"], w["b2"], o["y"], o["idx"], o["gates"], s.ws),
                 lambda: B.moe_norm_out(c, s.x, o["y"], w["w"], None, 0, SCALE, None, EPS, o["out"], None, o["rstd"], None),
                 lambda: B.moe_norm_out_bwd(tc, tr.t["dOut"], None, None, q["y"], tr.w["w"], None, 0, SCALE, None, q["rstd"], None, q["dX"], q["dY"], g["w"], None, None, tr.ws),
                 lambda: B.moe_norm_in_bwd(tc, q["dxn"], tr.t["x"], tr.w["w_in"], q["r_in"], None, q["dX"], g["w_in"], tr.ws),
                 lambda: B.moe_adamw(opt, 1e-3, 0.9, 0.999, 1e-8, 1)):
        with pytest.raises(ValueError):
            call()
