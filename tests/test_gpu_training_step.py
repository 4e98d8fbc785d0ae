"""A training step of a pre-norm block as a program makes it: layer norm, the layer, the router's losses on its logits, the backward passes with the losses' gradient added, and a Muon step on the
matrices; against automatic differentiation in 64 bits, over several steps, and recorded."""
import pytest
import torch

import training_reference as R
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS, WB, WZ, LR, MU = 1e-5, 0.5, 0.05, 0.02, 0.9
MATRICES = ("Wg", "Wn", "W1", "W2")


class Trainer:
    def __init__(self, T, d, h, n, k, act, sequences, seed=0):
        self.dt = torch.bfloat16 if act == "bf16" else torch.float32
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0, mean=0.0, dt=torch.float32: (torch.randn(*s, generator=g) * std + mean).to(dt).cuda()
        self.k, self.c = k, B.make_config(T, d, h, n, k, act, w_importance=0.0, w_load=0.0)
        self.w = dict(ln=r(d, std=0.1, mean=1.0), lb=r(d, std=0.1), Wg=r(d, n, std=d ** -0.5), Wn=r(d, n, std=0.2 * d ** -0.5), W1=r(n, d, h, std=d ** -0.5, dt=self.dt), b1=r(n, h, std=0.1, dt=self.dt),
                      W2=r(n, h, d, std=h ** -0.5, dt=self.dt), b2=r(n, d, std=0.1, dt=self.dt))
        self.x, self.noise, self.dY, self.dres = r(T, d, dt=self.dt), r(T, n), r(T, d, dt=self.dt), r(T, d, dt=self.dt)
        self.keep = (torch.rand(T, generator=g) < 0.9).to(torch.uint8).cuda()
        self.offsets = torch.linspace(0, T - 3, sequences + 1).int().cuda()
        S = B.moe_query_sizes(self.c)
        e = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)
        self.g = {q: torch.zeros_like(v) for q, v in self.w.items()}
        self.m = {q: torch.zeros_like(self.w[q], dtype=torch.float32) for q in MATRICES}
        self.ctx = B.empty_bytes(S.ctx_bytes)
        self.o = dict(xn=e(T, d, dt=self.dt), mean=e(T), rstd=e(T), y=e(T, d, dt=self.dt), losses=e(2), importance=e(n), load=e(n), counts=e(n, dt=torch.int32), rl=e(2),
                      rcounts=e(sequences, n, dt=torch.int32), sums=e(sequences, n), dlogits=e(T, n), dxn=e(T, d, dt=self.dt), dX=e(T, d, dt=self.dt))
        self.S = sequences
        self.list = B.moe_muon_list([dict(w=self.w[q], g=self.g[q], m=self.m[q], scale=0.2 * max(self.w[q].shape[-2:]) ** 0.5, weight_decay=0.1) for q in MATRICES])
        # in turn by all calls of the stream
        self.ws = B.empty_bytes(max(S.ws_fwd_bytes, S.ws_bwd_bytes, B.moe_layer_norm_workspace_bytes(self.c), B.moe_router_losses_workspace_bytes(self.c, sequences), B.moe_muon_workspace_bytes(self.list)))

    def step(self):
        c, w, g, o, ws = self.c, self.w, self.g, self.o, self.ws
        B.moe_layer_norm(c, self.x, w["ln"], w["lb"], EPS, o["xn"], o["mean"], o["rstd"])
        B.moe_forward(c, o["xn"], w["Wg"], w["Wn"], self.noise, w["W1"], w["b1"], w["W2"], w["b2"], o["y"], o["losses"], o["importance"], o["load"], o["counts"], self.ctx, ws)
        v = B.ctx_views(c, self.ctx)
        B.moe_router_losses(c, v["clean"].view(self.noise.shape), v["topk_idx"], self.keep, self.offsets, self.S, WB, WZ, o["rl"], o["rcounts"], o["sums"], o["dlogits"], ws)
        B.moe_backward_added(c, self.dY, o["xn"], w["Wg"], w["Wn"], self.noise, w["W1"], w["b1"], w["W2"], w["b2"], self.ctx, o["dlogits"], o["dxn"], g["Wg"], g["Wn"], g["W1"], g["b1"], g["W2"],
                             g["b2"], ws)
        B.moe_layer_norm_bwd(c, o["dxn"], self.x, w["ln"], o["mean"], o["rstd"], self.dres, o["dX"], g["ln"], g["lb"], ws)
        B.moe_muon(self.list, LR, MU, 1e-7, 5, True, ws)

    def reference(self, idx):
        """Gradients of sum(y dY) + sum(x dres) + the router's losses, with the kernels' choice of experts."""
        w = {q: R.f64(v).requires_grad_(True) for q, v in self.w.items()}
        x = R.f64(self.x).requires_grad_(True)
        mean = x.mean(1, keepdim=True)
        xn = (x - mean) / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS) * w["ln"] + w["lb"]
        logits = xn @ w["Wg"]
        H = logits + R.f64(self.noise) * torch.nn.functional.softplus(xn @ w["Wn"])
        gates = torch.softmax(H.gather(1, idx), 1)
        y = 0.0
        for s in range(self.k):
            e = idx[:, s]
            hid = torch.relu(torch.einsum("td,tdh->th", xn, w["W1"][e]) + w["b1"][e])
            y = y + gates[:, s:s + 1] * (torch.einsum("th,thd->td", hid, w["W2"][e]) + w["b2"][e])
        losses, counts, _, _ = R.router_losses(logits, idx.int(), self.keep, self.offsets.cpu(), WB, WZ)
        (losses.sum() + (y * R.f64(self.dY)).sum() + (x * R.f64(self.dres)).sum()).backward()
        return losses.detach(), counts, dict(x=x.grad, **{q: v.grad for q, v in w.items()})


@pytest.mark.parametrize("T,d,h,n,k,act,S", [(96, 64, 72, 6, 2, "f32", 1), (200, 68, 64, 20, 3, "f32", 5), (256, 64, 128, 8, 2, "bf16", 3)])
def test_steps(T, d, h, n, k, act, S):
    t = Trainer(T, d, h, n, k, act, S)
    # float: sums of some hundred terms; bf16: xn, hid, ys, dys, dz and the results are rounded by 2^-8 / sqrt(3) each, one behind the other, and ReLUs near zero switch
    tol = 1e-4 if act == "f32" else 3e-2
    for turn in range(3):
        before = {q: v.clone() for q, v in t.w.items()}
        m = {q: v.clone() for q, v in t.m.items()}
        t.step()
        assert B.moe_check_status(t.ws) == 0
        now, t.w = t.w, before
        idx = B.ctx_views(t.c, t.ctx)["topk_idx"].cpu().long()
        losses, counts, g = t.reference(idx)
        t.w = now
        assert torch.equal(t.o["rcounts"].cpu().long(), counts)
        assert float((R.f64(t.o["rl"]) - losses).abs().max() / losses.abs().max()) < tol
        for q, v in [("x", t.o["dX"])] + list(t.g.items()):
            assert float((R.f64(v) - g[q]).norm() / g[q].norm()) < tol, (turn, q)
        for q in MATRICES:  # from the gradients that the step has had
            three = lambda v: v if v.dim() == 3 else v[None]
            scale = 0.2 * max(before[q].shape[-2:]) ** 0.5
            w, _, x = R.muon(three(before[q]), three(t.g[q]), three(m[q]), LR, MU, 1e-7, 5, True, scale, 0.1, 1.0, torch.float32)
            step = torch.finfo(now[q].dtype).eps / 2
            size = LR * scale * x.flatten(1).norm(dim=1)
            # experts that few rows came to have gradients of low rank: as in test_gpu_muon's, 0.15 of the norm that X begins with
            off = (R.f64(three(now[q])) - w).flatten(1).norm(dim=1) / (4e-3 * size + 0.15 * LR * scale + 2 * step * w.flatten(1).norm(dim=1))
            assert float(off.max()) < 1.0, (turn, q)


def test_a_recorded_step():
    a, b = Trainer(200, 64, 128, 16, 2, "bf16", 4), Trainer(200, 64, 128, 16, 2, "bf16", 4)
    b.step()
    torch.cuda.synchronize()
    a.step()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        b.step()
        graph.capture_end()
    for _ in range(3):
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.w[q], b.w[q]) for q in a.w) and all(torch.equal(a.o[q], b.o[q]) for q in a.o) and all(torch.equal(a.m[q], b.m[q]) for q in a.m)
