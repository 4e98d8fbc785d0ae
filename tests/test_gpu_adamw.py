"""moe_adamw against the step in 64 bits. Float: three roundings in each moment and a dozen in the update. Eight bits: a code is the one that the 64-bit value
and the same random bits give, unless float arithmetic (a handful of roundings of the value and the scale, 24 u of the quotient, times the up to 16 units of a code) decides a
value next to the border between two codes the other way."""
import numpy as np
import pytest
import torch

import block_reference as R
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS = 1e-2, 0.9, 0.999, 1e-8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def tensor(count, w="f32", g="f32", master=False, bits=32, decay=0.1, seed=0, first=None, fresh=False):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + count)
    f = lambda std: torch.randn(count, device="cuda", generator=gen) * std
    big = f(0.5)
    t = dict(w=big.to(DT[w]), g=(f(1e-2) * torch.exp(f(2.0))).to(DT[g]), weight_decay=decay, master=big if master else None)
    m, v = f(5e-3), f(1e-2).square()
    if bits == 32:
        t.update(m=torch.zeros_like(m) if fresh else m, v=torch.zeros_like(v) if fresh else v)
    else:
        n = -(-count // 128)
        for q, x in (("m", m), ("v", v.sqrt())):
            pad = torch.zeros(n * 128, device="cuda")
            pad[:count] = 0 if fresh else x
            scale = pad.view(n, 128).abs().amax(1) / 448.0
            t[q] = (pad / scale.clamp(min=1e-30).repeat_interleave(128))[:count].to(torch.float8_e4m3fn)
            t[q + "_scale"] = scale
    if first is not None:
        t["first"] = first
    return t


def copy(ts):
    return [{q: v.clone() if torch.is_tensor(v) else v for q, v in t.items()} for t in ts]


def reference(t, step, grad_scale=1.0):
    """m, its terms, v, the new weight and its terms, in 64 bits."""
    f = lambda x: x.double().cpu().numpy()
    eight = t["m"].element_size() == 1
    m0 = R.held(t["m"], t["m_scale"]) if eight else f(t["m"])
    v0 = R.held(t["v"], t["v_scale"]) ** 2 if eight else f(t["v"])
    g = f(t["g"]) * grad_scale
    w = f(t["master"] if t.get("master") is not None else t["w"])
    m, v = B1 * m0 + (1 - B1) * g, B2 * v0 + (1 - B2) * g * g
    part = LR * (m / (1 - B1 ** step)) / (np.sqrt(v / (1 - B2 ** step)) + EPS)
    part_terms = LR * ((B1 * np.abs(m0) + (1 - B1) * np.abs(g)) / (1 - B1 ** step)) / (np.sqrt(v / (1 - B2 ** step)) + EPS)
    new = w - part - LR * t["weight_decay"] * w
    return m, B1 * np.abs(m0) + (1 - B1) * np.abs(g), v, new, np.abs(w) * (1 + LR * t["weight_decay"]) + part_terms


def check(before, after, step, seed=0, grad_scale=1.0, at=0):
    for b, a in zip(before, after):
        first = b.get("first", at)
        count = b["w"].numel()
        at = max(at, first + -(-count // 128) * 128)
        m, m_terms, v, new, w_terms = reference(b, step, grad_scale)
        if b.get("master") is not None:
            R.within(a["master"], new, 24 * R.U * w_terms, "master")
            assert torch.equal(a["w"], a["master"].to(a["w"].dtype))
        else:
            R.within(a["w"], new, 24 * R.U * w_terms, "w")
        if a["m"].element_size() == 4:
            R.within(a["m"], m, 4 * R.U * m_terms, "m")
            R.within(a["v"], v, 8 * R.U * v, "v")
            continue
        bits = R.dither(first, count, seed)
        for q, value, terms, root, use in (("m", m, m_terms, False, bits[0]), ("v", np.sqrt(v), np.sqrt(v), True, bits[1])):
            want, scale, off, unit = R.eight_bits(value, use, root)
            big = np.abs(R.blocks(terms)).max(1)
            R.within(a[q + "_scale"], scale, 16 * R.U * big / 448, q + "_scale")
            got = a[q].view(torch.float8_e4m3fn).double().cpu().numpy()
            # how far the quotient may be off, in units of its code
            s = np.repeat(np.where(scale > 0, scale, 1.0), 128)[:count]
            slack = (24 * R.U * terms + 24 * R.U * np.abs(value) * np.repeat(np.where(scale > 0, big / (448 * np.where(scale > 0, scale, 1.0)), 1.0), 128)[:count]) / s / unit
            same = got == want
            assert (same | ((off <= slack + 1e-12) & (np.abs(got - want) <= 2 * unit))).all(), q
            assert same.mean() > 0.999 or count < 4000


def run(ts, step=7, seed=0, **kw):
    before = copy(ts)
    B.moe_adamw(B.moe_adamw_list(ts), LR, B1, B2, EPS, step, seed, **kw)
    torch.cuda.synchronize()
    return before


KINDS = [("f32", "f32", False), ("bf16", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", False), ("bf16", "f32", True), ("bf16", "bf16", True)]


@pytest.mark.parametrize("w,g,master", KINDS)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 7, 8, 127, 128, 129, 2048, 2055, 8192, 8193, 70001])
def test_one_tensor(w, g, master, bits, count):
    ts = [tensor(count, w, g, master, bits)]
    check(run(ts, seed=123), ts, 7, 123)


@pytest.mark.parametrize("bits", [32, 8])
def test_from_nothing_and_several_steps(bits):
    ts = [tensor(5000, "bf16", "bf16", True, bits, fresh=True), tensor(300, bits=bits, decay=0.0, fresh=True)]
    for step in (1, 2, 3):
        check(run(ts, step, seed=step), ts, step, step)


def test_many_tensors_of_all_kinds():
    """More than one launch's worth, empty ones among them; the numbers of the elements run on from tensor to tensor."""
    ts = []
    for i in range(230):
        w, g, master = KINDS[i % 6]
        ts.append(tensor([0, 1, 130, 999, 4096][i % 5], w, g, master, (32, 8)[i % 2], decay=0.1 * (i % 3), seed=i))
    before = run(ts, 3, seed=9)
    check([b for b in before if b["w"].numel()], [t for t in ts if t["w"].numel()], 3, 9)


def test_numbers_of_elements_past_32_bits():
    ts = [tensor(1000, bits=8, first=2 ** 32 - 512), tensor(500, bits=8, first=2 ** 40)]
    check(run(ts, seed=5), ts, 7, 5)


def test_rounding_is_unbiased_and_follows_the_seed():
    """A moment between two codes goes up for a share of the elements that is its distance to the lower: 65024 draws, whose mean is off by 0.4 % of a code's unit (standard deviation)."""
    n = 2 ** 16
    t = dict(w=torch.zeros(n, device="cuda"), g=torch.zeros(n, device="cuda"), weight_decay=0.0, m=torch.full((n,), 32.0, device="cuda").to(torch.float8_e4m3fn),
             v=torch.zeros(n, device="cuda", dtype=torch.float8_e4m3fn), m_scale=torch.ones(n // 128, device="cuda"), v_scale=torch.zeros(n // 128, device="cuda"))
    t["g"][::128] = 4174.0  # the block's largest: m = 28.8 + 417.4, which sets the scale
    codes = []
    for seed in (1, 2, 1):
        u = copy([t])
        B.moe_adamw(B.moe_adamw_list(u), LR, B1, B2, EPS, 1, seed)
        codes.append(u[0]["m"].float())
    assert torch.equal(codes[0], codes[2]) and not torch.equal(codes[0], codes[1])
    rest = codes[0].view(-1, 128)[:, 1:]
    value = 28.8 / float(u[0]["m_scale"][0])
    assert abs(float(rest.mean()) - value) <= 0.01 * value
    assert len(rest.unique()) == 2


def test_a_second_moment_stays_above_zero_and_not_finite_gradients_stay_alone():
    n = 384
    t = tensor(n, bits=8, fresh=True)
    t["g"] = torch.full((n,), 1e-9, device="cuda")
    t["g"][0] = 1.0
    t["g"][200], t["g"][300] = float("inf"), float("nan")
    run([t], 1)
    v, m = t["v"].float(), t["m"].float()
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    fine[[200, 300]] = False
    assert (v[fine] > 0).all() and torch.isfinite(t["w"][fine]).all() and torch.isfinite(m[fine]).all()
    assert torch.isnan(v[~fine]).all() and torch.isnan(m[~fine]).all()
    assert torch.isfinite(t["v_scale"]).all() and torch.isfinite(t["m_scale"]).all()
    # no gradient, no moment: the weights stay
    z = tensor(n, bits=8, fresh=True, decay=0.0)
    z["g"].zero_()
    w = z["w"].clone()
    run([z], 1)
    assert torch.equal(z["w"], w) and not z["v"].float().any() and not z["m_scale"].any()


@pytest.mark.parametrize("size", [1e-42, 1e-38, 1e-30, 1e17])
def test_moments_of_extreme_size(size):
    """Scales that underflow are held at float's smallest normal number; large gradients whose squares are finite."""
    ts = [tensor(256, bits=8, fresh=True)]
    ts[0]["g"] = (torch.randn(256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * size)
    run(ts, 1)
    for q in ("w", "m", "v", "m_scale", "v_scale"):
        assert torch.isfinite(ts[0][q].float()).all(), q


def test_rates_in_device_memory_and_a_recorded_step():
    ts = [tensor(5000, "bf16", "bf16", True, 8), tensor(700)]
    ref = copy(ts)
    rates = torch.zeros(5, device="cuda")
    l, side, graph = B.moe_adamw_list(ts), torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def fill(step, seed, scale):
        rates[:4] = torch.tensor([LR, 1 - B1 ** step, 1 - B2 ** step, scale])
        rates[4:].view(torch.int32).fill_(seed)

    B.moe_adamw(B.moe_adamw_list(copy(ts)), LR, B1, B2, EPS, 1)  # an eager call first
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        B.moe_adamw(l, LR, B1, B2, EPS, 0, rates=rates)
        graph.capture_end()
    for step, scale in ((4, 1.0), (5, 0.25)):
        fill(step, 40 + step, scale)
        graph.replay()
        B.moe_adamw(B.moe_adamw_list(ref), LR, B1, B2, EPS, step, 40 + step, grad_scale=scale)
    torch.cuda.synchronize()
    for a, b in zip(ts, ref):
        for q in a:
            if torch.is_tensor(a[q]):
                assert torch.equal(a[q].view(torch.uint8), b[q].view(torch.uint8)), q


def test_what_stands_behind_a_tensor_is_left():
    big = torch.full((1000,), 3.0, device="cuda")
    t = tensor(77, seed=3)
    big[:77] = t["w"]
    t["w"] = big[:77]
    run([t])
    assert (big[77:] == 3.0).all()


def in_float(t, step, seed):
    """The step with 8-bit moments in float, every operation rounded by itself."""
    count = t["w"].numel()
    f = lambda x: torch.tensor(x, device="cuda", dtype=torch.float32)
    pad = lambda x: torch.cat([x, x.new_zeros(-count % 128)]).view(-1, 128)
    g = pad(t["g"].float())
    m, root = (pad(t[q].float()) * t[q + "_scale"][:, None] for q in ("m", "v"))
    m = f(B1) * m + f(1 - B1) * g
    root = (f(B2) * (root * root) + f(1 - B2) * (g * g)).sqrt()
    bits = R.dither(0, count, seed)
    for q, value, use in (("m", m, bits[0]), ("v", root, bits[1])):
        scale = value.abs().amax(1) * f(1.0 / 448.0)
        x = value / scale[:, None]
        dither = pad(torch.from_numpy((use * np.uint64(16) + np.uint64(8)).astype(np.int32)).cuda())
        small = x.abs() < 2.0 ** -6
        z = ((torch.where(small, x.abs() + 2.0 ** -6, x.abs()).view(torch.int32) + dither) & ~0xfffff).view(torch.float32)
        z = torch.where(small, z - 2.0 ** -6, z).clamp(max=448.0)
        if q == "v":
            z = torch.where((x > 0) & (z == 0), torch.full_like(z, 2.0 ** -9), z)
        t[q].copy_(torch.copysign(z, x).view(-1)[:count].to(torch.float8_e4m3fn))
        t[q + "_scale"].copy_(scale)


@pytest.mark.parametrize("g", ["f32", "bf16"])
def test_codes_stay_those_of_the_formulas_in_float(g):
    # 12 million codes: with a root or a quotient that is a unit of the last place off, some ten of them would turn over
    ts = [tensor(1000003, "f32", g, bits=8, seed=5)]
    want = copy(ts)[0]
    for step in range(1, 7):
        run(ts, step, 40 + step)
        in_float(want, step, 40 + step)
    for q in ("m_scale", "v_scale"):
        assert torch.equal(ts[0][q], want[q])
    for q in ("m", "v"):
        assert (ts[0][q].float() == want[q].float()).all()


@pytest.mark.parametrize("count", [8000003, 30000100])
def test_codes_of_blocks_of_several_steps(count):
    ts = [tensor(count, "bf16", "bf16", bits=8, seed=6)]
    want = copy(ts)[0]
    run(ts, 3, 9)
    in_float(want, 3, 9)
    for q in ("m_scale", "v_scale"):
        assert torch.equal(ts[0][q], want[q])
    for q in ("m", "v"):
        assert (ts[0][q].float() == want[q].float()).all()
