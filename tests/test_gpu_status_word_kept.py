"""Calls without bounded waits leave the status word of their workspace as they find it: a report of an earlier call stays."""
import pytest
import torch

import test_gpu_norms as N
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
TIMEOUT = 5


@pytest.mark.parametrize("d", [64, 4104])
def test_norms(d):
    T, act = 40, "bf16"
    cfg, t = N.config(T, d, act), N.tensors(T, d, act, 31)
    ws, word = B.empty_bytes(B.moe_norm_workspace_bytes(cfg)), lambda: int(ws[:4].view(torch.int32))
    f = N.forward(cfg, t)
    dX, dY, dw, dw_next = (torch.empty_like(t[q]) for q in ("x", "x", "w", "w"))
    for report in (TIMEOUT, 0):
        ws.fill_(0xff)
        ws[:4].view(torch.int32).fill_(report)
        B.moe_norm_out_bwd(cfg, t["dOut"], t["dNext"], f[0], t["y"], t["w"], None, 0, 0.7, t["w_next"], f[2], f[3], dX, dY, dw, None, dw_next, ws)
        assert word() == report and B.moe_check_status(ws) == report
        B.moe_norm_in_bwd(cfg, t["dNext"], f[0], t["w_next"], f[3], None, dX, dw, ws)
        assert word() == report and B.moe_check_status(ws) == report


def test_factored_adam():
    n, d, h = 3, 64, 128
    cfg = B.make_config(8, d, h, n, 1, "f32")
    S = B.moe_query_sizes(cfg)
    w = [torch.randn(*s, device="cuda") for s in ((n, d, h), (n, h), (n, h, d), (n, d))]
    g = [torch.randn_like(x) for x in w]
    ws = B.empty_bytes(S.ws_adam_bytes)
    for report in (TIMEOUT, 0):
        ws.fill_(0xff)
        ws[:4].view(torch.int32).fill_(report)
        B.moe_expert_adam_factored(cfg, *w, *g, torch.zeros(S.adam_state_elems, device="cuda"), 1e-3, 0.99, 1e-8, 1, ws)
        assert B.moe_check_status(ws) == report
