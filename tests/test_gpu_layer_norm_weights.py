"""Layer norm right behind the launch that writes its weights: every step's norm has that step's weights, in a stream and recorded."""
import pytest
import torch

from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Run:
    """AdamW over a long list whose last tensors are the norm's, then the norm and its backward pass; gradients that change the weights at every step."""

    def __init__(self, T, d, act, seed=0):
        dt = {"f32": torch.float32, "bf16": torch.bfloat16}[act]
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0, mean=0.0, t=torch.float32: (torch.randn(*s, generator=g) * std + mean).to(t).cuda()
        self.c = B.make_config(T, d, d, 1, 1, act)
        self.x, self.dxn, self.w, self.b, self.gw, self.gb = r(T, d, t=dt), r(T, d, t=dt), r(d, std=0.1, mean=1.0), r(d), r(d), r(d)
        other = [r(1 << 20) for _ in range(8)]
        zeros = lambda t: dict(m=torch.zeros_like(t), v=torch.zeros_like(t))
        self.list = B.moe_adamw_list([dict(w=t, g=t.clone(), **zeros(t)) for t in other] + [dict(w=self.w, g=self.gw, **zeros(self.w)), dict(w=self.b, g=self.gb, **zeros(self.b))])
        e = lambda *s, t=torch.float32: torch.zeros(*s, device="cuda", dtype=t)
        self.o = dict(xn=e(T, d, t=dt), mean=e(T), rstd=e(T), dX=e(T, d, t=dt), dw=e(d), db=e(d))
        self.ws = B.empty_bytes(B.moe_layer_norm_workspace_bytes(self.c))

    def adamw(self, step=1):
        B.moe_adamw(self.list, 0.05, 0.9, 0.99, 1e-8, step)

    def forward(self):
        B.moe_layer_norm(self.c, self.x, self.w, self.b, EPS, self.o["xn"], self.o["mean"], self.o["rstd"])

    def backward(self):
        o = self.o
        B.moe_layer_norm_bwd(self.c, self.dxn, self.x, self.w, o["mean"], o["rstd"], None, o["dX"], o["dw"], o["db"], self.ws)


@pytest.mark.parametrize("T,d,act", [(1, 512, "bf16"), (300, 512, "bf16"), (40, 4096, "f32"), (20, 16384, "bf16")])
def test_weights_of_the_launch_before(T, d, act):
    a, b, graph, side = Run(T, d, act), Run(T, d, act), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    recorded = Run(T, d, act)

    def step(r, between):
        r.adamw()
        between()
        r.forward()
        between()
        r.adamw()
        between()
        r.backward()
        between()

    none = lambda: None
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        step(recorded, none)
        graph.capture_end()
    for turn in range(30):
        step(a, torch.cuda.synchronize)
        step(b, none)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.o[q], b.o[q]) and torch.equal(a.o[q], recorded.o[q]) for q in a.o), turn
        assert torch.equal(a.w, b.w) and not torch.equal(a.w, torch.ones_like(a.w))
