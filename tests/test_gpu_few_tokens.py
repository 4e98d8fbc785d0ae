"""moe_forward_few against the layer in 64 bits, and its routing against moe_gate bit for bit. The tolerances are worked out in block_reference.few."""
import pytest
import torch

import block_reference as R
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def layer(T, d, h, n, k, act, seed=0, gate_std=None):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * T + d + h + n)
    f = lambda *s, std=1.0, dt=DT[act]: (torch.randn(*s, device="cuda", generator=g) * std).to(dt)
    return dict(x=f(T, d), Wg=f(d, n, std=d ** -0.5 if gate_std is None else gate_std, dt=torch.float32), W1=f(n, d, h, std=d ** -0.5), b1=f(n, h, std=0.3),
                W2=f(n, h, d, std=h ** -0.5), b2=f(n, d, std=0.3))


def run(cfg, t, ws=None):
    y = torch.full_like(t["x"], 7.0)
    idx, gates = torch.full((cfg.T, cfg.k), -7, dtype=torch.int32, device="cuda"), torch.full((cfg.T, cfg.k), 7.0, device="cuda")
    if ws is None:
        ws = B.empty_bytes(B.moe_few_workspace_bytes(cfg))
        ws.fill_(0xff)
    B.moe_forward_few(cfg, t["x"], t["Wg"], t["W1"], t["b1"], t["W2"], t["b2"], y, idx, gates, ws)
    assert B.moe_check_status(ws) == 0
    return y, idx, gates


def routed_by_moe_gate(cfg, t):
    T, n, k = cfg.T, cfg.n, cfg.k
    c = B.make_config(T, cfg.d, cfg.h, n, k, cfg.act, flags=B.MOE_FLAG_GATE_SCREEN_OFF)
    e = lambda *s, dt=torch.float32: torch.empty(*s, device="cuda", dtype=dt)
    idx, gates = e(T, k, dt=torch.int32), e(T, k)
    B.moe_gate(c, t["x"], t["Wg"], torch.zeros_like(t["Wg"]), torch.zeros(T, n, device="cuda"), idx, gates, e(T, n), e(T, n), e(T, 2), e(T, 2, dt=torch.int32),
               B.empty_bytes(B.moe_query_sizes(c).ws_bytes))
    return idx, gates


def check(cfg, t):
    y, idx, gates = run(cfg, t)
    want_idx, want_gates = routed_by_moe_gate(cfg, t)
    assert torch.equal(idx, want_idx) and torch.equal(gates, want_gates)
    want, slack, g, gate_slack = R.few(t["x"], t["Wg"], t["W1"], t["b1"], t["W2"], t["b2"], cfg.k, idx)
    R.within(gates, g, gate_slack, "gates")
    R.within(y, want, slack, "y")
    again = run(cfg, t)[0]
    assert torch.equal(y, again)


# one token; every number of rows an expert can have (1, 8, 9, 17, 33, 64 of 64); widths of one vector, odd ones, several tiles and pieces of h; more experts than a warp has
# lanes, one expert, as many as there are
@pytest.mark.parametrize("T,d,h,n,k,act", [(1, 64, 64, 4, 2, "bf16"), (1, 8, 8, 1, 1, "bf16"), (1, 4, 4, 3, 3, "f32"), (1, 512, 1024, 32, 4, "bf16"), (2, 72, 40, 5, 2, "bf16"),
                                           (9, 72, 136, 3, 2, "bf16"), (24, 512, 1024, 32, 4, "bf16"), (33, 264, 328, 7, 3, "bf16"), (64, 128, 192, 1, 1, "bf16"), (64, 64, 128, 2, 2, "bf16"),
                                           (64, 200, 72, 4, 2, "bf16"), (17, 64, 64, 300, 8, "bf16"), (40, 128, 64, 33, 6, "bf16"), (5, 72, 520, 20, 3, "f32"), (64, 36, 52, 2, 2, "f32"),
                                           (33, 256, 512, 16, 2, "f32"), (8, 1028, 68, 9, 1, "f32"), (3, 1024, 2056, 8, 2, "bf16"), (4, 64, 64, 8192, 8, "bf16")])
def test_against_64_bits(T, d, h, n, k, act):
    check(B.make_config(T, d, h, n, k, act), layer(T, d, h, n, k, act))


@pytest.mark.parametrize("T,d,h,n,k,act", [(64, 2048, 2056, 9, 8, "bf16"), (64, 1024, 4104, 8, 8, "f32"), (64, 8192, 200, 8, 8, "bf16")])
def test_parts_of_y_of_several_slices(T, d, h, n, k, act):
    """Parts of y for every 64 hidden units would be more than 64 MiB: a task has several of them."""
    check(B.make_config(T, d, h, n, k, act), layer(T, d, h, n, k, act))


# one to four tiles of either product, for every number of warps in a team; a single slice and many
@pytest.mark.parametrize("T,d,h,n,k,act", [(1, 64, 40, 2, 1, "bf16"), (60, 64, 2048, 200, 4, "bf16"), (64, 128, 1024, 256, 8, "bf16"), (64, 72, 512, 512, 8, "bf16"), (20, 520, 64, 100, 2, "bf16"),
                                           (64, 32, 1024, 128, 8, "f32"), (50, 100, 260, 300, 4, "f32"), (16, 36, 4096, 20, 2, "f32")])
def test_teams_of_all_sizes(T, d, h, n, k, act):
    check(B.make_config(T, d, h, n, k, act), layer(T, d, h, n, k, act))


def test_every_number_of_rows():
    """T tokens that all pick the same expert, T = 1 .. 64: expert 1 has T rows, the other none."""
    d, h = 64, 72
    for T in range(1, 65):
        t = layer(T, d, h, 2, 1, "bf16", seed=T, gate_std=0.0)
        t["x"][:, 0] = 1.0
        t["Wg"][0, 1] = 1.0
        cfg = B.make_config(T, d, h, 2, 1, "bf16")
        y, idx, _ = run(cfg, t)
        assert (idx == 1).all()
        want, slack, _, _ = R.few(t["x"], t["Wg"], t["W1"], t["b1"], t["W2"], t["b2"], 1, idx)
        R.within(y, want, slack, f"y of {T}")


def test_equal_logits_and_not_finite_ones():
    """All logits equal: the first k experts, equal gates. A NaN ranks below every number; an infinite weight of an expert that no token picks is not read."""
    T, d, h, n, k = 3, 64, 64, 40, 4
    t, cfg = layer(T, d, h, n, k, "bf16", gate_std=0.0), B.make_config(T, d, h, n, k, "bf16")
    t["W1"][k:], t["W2"][k:], t["b2"][k:] = float("nan"), float("inf"), float("nan")
    y, idx, gates = run(cfg, t)
    assert torch.equal(idx.cpu(), torch.arange(k, dtype=torch.int32).expand(T, k)) and torch.equal(gates, torch.full_like(gates, 0.25)) and torch.isfinite(y).all()
    t["Wg"][:, 0] = float("nan")
    t["W1"][0], t["W1"][k] = float("nan"), 0.0
    t["W2"][k], t["b2"][k] = 0.0, 0.0
    y, idx, _ = run(cfg, t)
    assert torch.equal(idx.cpu(), torch.arange(1, k + 1, dtype=torch.int32).expand(T, k)) and torch.isfinite(y).all()
    assert torch.equal(routed_by_moe_gate(cfg, t)[0], idx)


def test_not_finite_inputs_stay_with_their_tokens():
    T, d, h, n, k = 6, 128, 136, 4, 2
    t, cfg = layer(T, d, h, n, k, "bf16"), B.make_config(T, d, h, n, k, "bf16")
    clean = run(cfg, t)[0]
    t["x"][2, 5] = float("inf")
    y = run(cfg, t)[0]
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(y[keep], clean[keep]) and not torch.isfinite(y[2]).all()


def test_a_weight_that_is_not_finite_reaches_the_output():
    """relu(NaN) is a NaN, and an infinity times a positive activation an infinity."""
    T, d, h, n, k = 2, 64, 64, 1, 1
    t, cfg = layer(T, d, h, n, k, "bf16"), B.make_config(T, d, h, n, k, "bf16")
    t["W1"][0, 3, 9] = float("nan")
    assert torch.isnan(run(cfg, t)[0]).all()
    t = layer(T, d, h, n, k, "bf16")
    t["b1"][0, 5], t["W2"][0, 5, 7] = 100.0, float("inf")
    assert torch.isinf(run(cfg, t)[0][:, 7]).all()


def test_rows_behind_the_last_are_left_and_outputs_may_be_missing():
    T, d, h, n, k = 5, 72, 64, 6, 2
    t, cfg = layer(T, d, h, n, k, "bf16"), B.make_config(T, d, h, n, k, "bf16")
    want = run(cfg, t)[0]
    big, ws = torch.full((T + 2, d), 5.0, device="cuda", dtype=torch.bfloat16), B.empty_bytes(B.moe_few_workspace_bytes(cfg))
    B.moe_forward_few(cfg, t["x"], t["Wg"], t["W1"], t["b1"], t["W2"], t["b2"], big[:T], None, None, ws)
    assert torch.equal(big[:T], want) and (big[T:] == 5.0).all()


def test_the_layer_of_moe_forward():
    """What moe_forward without noise gives, which rounds ys to bf16 as well: half a step of each of the k rows more."""
    T, d, h, n, k = 24, 256, 512, 16, 4
    t, cfg = layer(T, d, h, n, k, "bf16"), B.make_config(T, d, h, n, k, "bf16", flags=B.MOE_FLAG_GATE_SCREEN_OFF)
    y, idx, gates = run(cfg, t)
    S = B.moe_query_sizes(cfg)
    e = lambda *s, dt=torch.float32: torch.empty(*s, device="cuda", dtype=dt)
    full, ctx = torch.empty_like(y), B.empty_bytes(S.ctx_bytes)
    B.moe_forward(cfg, t["x"], t["Wg"].reshape(-1), torch.zeros_like(t["Wg"]), torch.zeros(T * n, device="cuda"), t["W1"], t["b1"], t["W2"], t["b2"], full, e(2), e(n), e(n),
                  e(n, dt=torch.int32), ctx, B.empty_bytes(S.ws_fwd_bytes))
    V = B.ctx_views(cfg, ctx)
    assert torch.equal(V["topk_idx"], idx)
    want, slack, g, _ = R.few(t["x"], t["Wg"], t["W1"], t["b1"], t["W2"], t["b2"], k, idx)
    rows = V["ys"].double().cpu()[V["inv_perm"].cpu().long()].view(T, k, d).abs()
    R.within(full, want, slack + 1.01 * R.half_step(torch.bfloat16) * (g[:, :, None] * rows).sum(1), "moe_forward")
    R.within(y, want, slack, "moe_forward_few")


def test_one_workspace_in_turn_by_layers_of_other_sizes():
    """The counters are set anew by every call, whatever the one before has left in the workspace."""
    sizes = [(1, 64, 64, 4, 2), (24, 128, 256, 8, 3), (64, 64, 72, 3, 1), (2, 256, 64, 16, 4)]
    cfgs = [B.make_config(*s, "bf16") for s in sizes]
    ts = [layer(*s, "bf16") for s in sizes]
    want = [run(c, t)[0] for c, t in zip(cfgs, ts)]
    ws = B.empty_bytes(max(B.moe_few_workspace_bytes(c) for c in cfgs))
    ws.random_(0, 256)
    for _ in range(3):
        for c, t, w in zip(cfgs, ts, want):
            assert torch.equal(run(c, t, ws)[0], w)


def test_two_streams_at_once_and_recorded_graphs():
    """Blocks of two calls share the GPU in any proportion; replays of two graphs, a workspace each."""
    sizes = [(24, 256, 1024, 16, 4), (64, 512, 512, 12, 2)]
    cfgs = [B.make_config(*s, "bf16") for s in sizes]
    ts = [layer(*s, "bf16") for s in sizes]
    want = [run(c, t)[0] for c, t in zip(cfgs, ts)]
    ys = [torch.zeros_like(w) for w in want]
    ws = [B.empty_bytes(B.moe_few_workspace_bytes(c)) for c in cfgs]
    streams, graphs = [torch.cuda.Stream() for _ in sizes], []
    torch.cuda.synchronize()

    def call(i):
        t = ts[i]
        B.moe_forward_few(cfgs[i], t["x"], t["Wg"], t["W1"], t["b1"], t["W2"], t["b2"], ys[i], None, None, ws[i])

    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                call(i)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(ys[i], want[i]) and B.moe_check_status(ws[i]) == 0
        ys[i].zero_()
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(s):
            graphs[i].capture_begin()
            call(i)
            call(i)
            graphs[i].capture_end()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(ys[i], want[i]) and B.moe_check_status(ws[i]) == 0
    for i in range(2):  # new inputs in the same place
        ts[i]["x"].mul_(-0.5)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(ys[i], run(cfgs[i], ts[i])[0])
