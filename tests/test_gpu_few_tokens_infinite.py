"""Weights of W2 that are not finite, and sums beyond float's range, in moe_forward_few: what moe_forward gives, whose hid is one bf16 number. The second term of hid has either sign, or is 0:
times an infinity it would make a NaN of the infinity that the first term gives."""
import pytest
import torch

import test_gpu_few_tokens as F
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
INF = float("inf")


def given(T, d, h, hid, act="bf16", n=1, k=1):
    """A layer whose hid of token t and unit j is exactly hid[t][j], a sum of two products with 1."""
    t, cfg = F.layer(T, d, h, n, k, act), B.make_config(T, d, h, n, k, act)
    x, w1 = torch.zeros_like(t["x"]), torch.zeros_like(t["W1"])
    # unit 0 alone has what x says, in two columns: the first bf16 number and the rest
    hi = hid.to(torch.bfloat16)
    x[:, 0], x[:, 1] = hi, (hid - hi.float()).to(x.dtype)
    w1[:, 0, 0] = w1[:, 1, 0] = 1.0
    t["x"], t["W1"] = x, w1
    t["b1"].zero_()
    return t, cfg


@pytest.mark.parametrize("T,d,h", [(1, 64, 64), (16, 72, 40), (64, 64, 200)])
@pytest.mark.parametrize("size", [INF, -INF])
def test_an_infinite_weight_gives_its_infinity(T, d, h, size):
    """Remainders of hid above 0, below 0, and 0 (every third token)."""
    j = torch.arange(T, device="cuda")
    hid = 1.0 + torch.tensor([0.0, 1.0, -1.0], device="cuda")[j % 3] * 2.0 ** -11 + (j // 3) * 2.0 ** -6
    t, cfg = given(T, d, h, hid)
    t["W2"][0, 0, 7], t["W2"][0, 0, d - 1] = size, -size
    y = F.run(cfg, t)[0].float()
    assert (y[:, 7] == size).all() and (y[:, d - 1] == -size).all()
    others = [c for c in range(d) if c not in (7, d - 1)]
    t["W2"][0, 0, 7] = t["W2"][0, 0, d - 1] = 0.0
    assert torch.equal(y[:, others], F.run(cfg, t)[0].float()[:, others])  # their own columns alone


def test_random_layers_with_infinite_weights():
    """As moe_forward: infinities where it has infinities, NaN where it has NaN (hid 0, or infinities of both signs)."""
    for seed, (T, d, h, n, k) in enumerate([(64, 64, 64, 1, 1), (64, 128, 256, 8, 3), (24, 264, 136, 9, 2), (5, 512, 1024, 4, 2)]):
        t, cfg = F.layer(T, d, h, n, k, "bf16", seed=seed), B.make_config(T, d, h, n, k, "bf16", flags=B.MOE_FLAG_GATE_SCREEN_OFF)
        for e in range(n):
            for c, v in ((1, INF), (3, -INF), (40, INF)):
                t["b1"][e, (7 * e + c) % h] = 20.0  # the units that meet one are on
                t["W2"][e, (7 * e + c) % h, c + e] = v
        t["W2"][0, 3, 20] = t["W2"][0, 4, 20] = INF
        y = F.run(cfg, t)[0]
        S = B.moe_query_sizes(cfg)
        e = lambda *s, dt=torch.float32: torch.empty(*s, device="cuda", dtype=dt)
        full, ctx = torch.empty_like(y), B.empty_bytes(S.ctx_bytes)
        B.moe_forward(cfg, t["x"], t["Wg"].reshape(-1), torch.zeros_like(t["Wg"]), torch.zeros(T * n, device="cuda"), t["W1"], t["b1"], t["W2"], t["b2"], full, e(2), e(n), e(n),
                      e(n, dt=torch.int32), ctx, B.empty_bytes(S.ws_fwd_bytes))
        assert torch.isinf(full).any() and torch.equal(torch.isnan(y), torch.isnan(full)), (T, d, h, n, k)
        inf = torch.isinf(full)
        assert torch.equal(torch.isinf(y), inf) and torch.equal(y[inf], full[inf])


def test_sums_beyond_the_range_are_infinities():
    """hid times a finite weight is beyond float's range: an infinity of the product's sign, whatever the remainder's."""
    T, d, h = 6, 64, 64
    hid = torch.tensor([1.0, 1.0 + 2.0 ** -11, 1.0 - 2.0 ** -11] * 2, device="cuda") * 2.0 ** 100
    t, cfg = given(T, d, h, hid)
    t["W2"][0, 0, 5], t["W2"][0, 0, 6] = 2.0 ** 120, -(2.0 ** 120)
    y = F.run(cfg, t)[0].float()
    assert (y[:, 5] == INF).all() and (y[:, 6] == -INF).all()


def test_nan_weights_stay_nan():
    T, d, h = 4, 64, 64
    t, cfg = F.layer(T, d, h, 1, 1, "bf16"), B.make_config(T, d, h, 1, 1, "bf16")
    clean = F.run(cfg, t)[0]
    t["W2"][0, 9, 11] = float("nan")
    y = F.run(cfg, t)[0]
    assert torch.isnan(y[:, 11]).all()
    keep = [c for c in range(d) if c != 11]
    assert torch.equal(y[:, keep], clean[:, keep])


@pytest.mark.parametrize("size", [INF, -INF])
def test_float_layers(size):
    t, cfg = given(5, 64, 68, torch.tensor([1.0, 1.5, 0.75, 1.0, 3.0], device="cuda"), act="f32")
    t["W2"][0, 0, 7] = size
    assert (F.run(cfg, t)[0][:, 7] == size).all()
