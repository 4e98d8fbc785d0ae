"""moe_layer_norm_bwd of rows whose mean is far larger than their spread, with the statistics that it is given: (x - mean) r is off by two roundings of itself, not by roundings of x r.

Tolerances are those of test_gpu_layer_norm, of terms of the differences' size."""
import pytest
import torch

import training_reference as R
from block_reference import within
from paper_1701_06538_b200 import binding as B
from test_gpu_layer_norm import K, U, data, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mean", [10.0, 100.0, 1000.0, -3e4])
@pytest.mark.parametrize("T,d,act", [(40, 512, "f32"), (40, 512, "bf16"), (300, 72, "f32"), (700, 320, "f32"), (12, 4096, "f32"), (6, 16384, "f32"), (5, 16384, "bf16"), (33, 2048, "bf16")])
@pytest.mark.parametrize("res", [False, True])
def test_backward(T, d, act, mean, res):
    t, c = data(T, d, act, mean=mean), B.make_config(T, d, d, 1, 1, act)
    if act == "bf16":  # whose numbers at that size are further apart than the spread
        t["x"] = (t["x"].float() + 0.2 * mean * torch.randn(T, d, generator=torch.Generator().manual_seed(1)).cuda()).bfloat16()
    _, m, r = forward(c, t)
    o = dict(dX=torch.full_like(t["x"], 7.0), dw=torch.full((d,), 7.0, device="cuda"), db=torch.full((d,), 7.0, device="cuda"))
    B.moe_layer_norm_bwd(c, t["dxn"], t["x"], t["w"], m, r, t["dres"] if res else None, o["dX"], o["dw"], o["db"], B.empty_bytes(B.moe_layer_norm_workspace_bytes(c)))
    want = R.layer_norm_bwd(t["dxn"], t["x"], t["w"], m, r, t["dres"] if res else None)
    dxn, x, w, mean64, rstd = map(R.f64, (t["dxn"], t["x"], t["w"], m, r))
    n, u = (x - mean64[:, None]).abs() * rstd[:, None], (dxn * w).abs()
    terms = rstd[:, None] * (u + u.mean(1, keepdim=True) + n * (u * n).mean(1, keepdim=True))
    if res:
        terms = terms + R.f64(t["dres"]).abs()
    slack = K + (T / 100) * U
    within(o["dX"], want["dX"][0], slack * terms, "dX")
    within(o["dw"], want["dw"][0], slack * (dxn.abs() * n).sum(0), "dw")
    within(o["db"], want["db"][0], slack * dxn.abs().sum(0), "db")
