"""Every refusal of moe_norm_*, moe_forward_few and moe_adamw by itself: arguments that are good, each with an address of its own, and one of them broken. The good ones are not refused (without a
GPU they come to the launch, which fails with another status), so that a refusal is that of the one argument."""
import ctypes

import pytest
import torch

from paper_1701_06538_b200 import binding as B
from paper_1701_06538_b200 import build as moe_build

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")
OK, INVALID, UNSUPPORTED = 0, 1, 2
T, D, H, N, K = 16, 64, 64, 8, 2
INF, NAN = float("inf"), float("nan")

# name: ((argument, its kind), ...). Kinds: p a pointer, o one that may be NULL, i an int, f a float; g, d, n pointers that are needed with a gate (g the gate, d its gradient) or a next norm
# (n; N is w_next itself)
CALLS = {
    "moe_norm_in": "x p, w p, eps f, xn p, rstd o",
    "moe_norm_in_bwd": "dxn p, x p, w p, rstd p, dres o, dX p, dw p, ws p",
    "moe_norm_out": "x p, y p, w p, gate g, rows_per_gate i, residual_scale f, w_next N, eps f, out p, next n, rstd p, rstd_next n",
    "moe_norm_out_bwd": "dOut p, dNext n, out n, y p, w p, gate g, rows_per_gate i, residual_scale f, w_next N, rstd p, rstd_next n, dX p, dY p, dw p, dgate d, dw_next n, ws p",
    "moe_forward_few": "x p, Wg p, W1 p, b1 p, W2 p, b2 p, y p, topk_idx o, gates o, ws p",
}
CALLS = {name: [tuple(a.split()) for a in spec.split(", ")] for name, spec in CALLS.items()}
NUMBERS = dict(eps=1e-6, rows_per_gate=4, residual_scale=0.7)
CASES = [(name, gate, nxt) for name in CALLS for gate in ((False, True) if name.startswith("moe_norm_out") else (False,)) for nxt in ((False, True) if name.startswith("moe_norm_out") else (False,))]


@pytest.fixture(scope="module", autouse=True)
def lib():
    moe_build.build()
    return B.lib()


def call(name, with_gate=True, with_next=True, cfg=None, **broken):
    """With every argument good but those of `broken`."""
    args = []
    for i, (arg, kind) in enumerate(CALLS[name]):
        if kind in "fi":
            v = broken.get(arg, NUMBERS[arg])
            args.append(ctypes.c_float(v) if kind == "f" else ctypes.c_int32(v))
            continue
        there = kind in "po" or (with_gate if kind in "gd" else with_next)
        v = broken.get(arg, (i + 1) << 30 if there else 0)
        args.append(ctypes.c_void_p(v))
    cfg = cfg or B.make_config(T, D, H, N, K, "f32")
    return getattr(B.lib(), name)(ctypes.byref(cfg), *args, ctypes.c_void_p(0))


@pytest.mark.parametrize("name,gate,nxt", CASES)
def test_good_arguments_are_not_refused(name, gate, nxt):
    for act in ("f32", "bf16"):
        assert call(name, gate, nxt, B.make_config(T, D, H, N, K, act)) not in (INVALID, UNSUPPORTED)


@pytest.mark.parametrize("name,gate,nxt", CASES)
def test_every_pointer(name, gate, nxt):
    for i, (arg, kind) in enumerate(CALLS[name]):
        if kind in "fi":
            continue
        needed = kind == "p" or (kind == "d" and gate) or (kind == "n" and nxt)
        if needed:
            assert call(name, gate, nxt, **{arg: 0}) == INVALID, f"{arg} missing"
        else:
            assert call(name, gate, nxt, **{arg: 0}) not in (INVALID, UNSUPPORTED), f"{arg} may be missing"
        used = needed or kind == "o" or (kind == "g" and gate) or (kind == "N" and nxt)
        for off in (4, 16):
            status = call(name, gate, nxt, **{arg: ((i + 1) << 30) + off})
            if used:
                assert status == INVALID, f"{arg} off its boundary"
            elif kind in "dn":
                assert status not in (INVALID, UNSUPPORTED), f"{arg} is ignored"


@pytest.mark.parametrize("name", ["moe_norm_in", "moe_norm_out"])
def test_eps(name):
    for eps in (0.0, -1.0, NAN, INF, -INF):
        assert call(name, eps=eps) == INVALID
    assert call(name, eps=1e-30) != INVALID


@pytest.mark.parametrize("name", ["moe_norm_out", "moe_norm_out_bwd"])
def test_gates_and_scales(name):
    for rows in (0, -1, -2 ** 31):
        assert call(name, rows_per_gate=rows) == INVALID
        assert call(name, with_gate=False, rows_per_gate=rows) != INVALID  # ignored without a gate
    for rows in (1, T, T + 1, 2 ** 31 - 1):
        assert call(name, rows_per_gate=rows) != INVALID
    for scale in (NAN, INF, -INF):
        assert call(name, residual_scale=scale) == INVALID
    for scale in (0.0, -1.0):
        assert call(name, residual_scale=scale) != INVALID


def test_widths():
    for name in CALLS:
        wide = B.make_config(T, 16388, H, N, K, "f32")
        assert (call(name, cfg=wide) == UNSUPPORTED) == name.startswith("moe_norm")
        assert call(name, cfg=B.make_config(T, 16384, H, N, K, "f32")) not in (INVALID, UNSUPPORTED)
        for bad in (B.make_config(T, 3, H, N, K, "f32"), B.make_config(T, 4, H, N, K, "bf16"), B.make_config(-1, D, H, N, K, "f32"), B.make_config(T, D, H, N, K, 2)):
            assert call(name, cfg=bad) == INVALID, name


def test_outputs_in_one_place():
    at = lambda name, arg: ([a for a, _ in CALLS[name]].index(arg) + 1) << 30
    for name, arg, other in (("moe_norm_out", "next", "out"), ("moe_norm_out_bwd", "dX", "dY"), ("moe_forward_few", "y", "x")):
        assert call(name, **{arg: at(name, other)}) == INVALID
    # what may
    for name, pairs in (("moe_norm_in", [("xn", "x")]), ("moe_norm_in_bwd", [("dX", "dxn"), ("dX", "dres"), ("dX", "x")]),
                        ("moe_norm_out", [("out", "x"), ("out", "y"), ("next", "x"), ("next", "y")]),
                        ("moe_norm_out_bwd", [(a, b) for a in ("dX", "dY") for b in ("dOut", "dNext", "out", "y")])):
        for arg, other in pairs:
            assert call(name, **{arg: at(name, other)}) not in (INVALID, UNSUPPORTED), (name, arg, other)
    assert call("moe_norm_out", with_next=False, next=at("moe_norm_out", "out")) != INVALID  # next is ignored then


def test_few_tokens_sizes():
    few = lambda **kw: call("moe_forward_few", cfg=B.make_config(**{**dict(T=T, d=D, h=H, n=N, k=K, act="bf16"), **kw}))
    for kw in (dict(T=64), dict(T=1), dict(n=8192, k=8), dict(n=1, k=1)):
        assert few(**kw) not in (INVALID, UNSUPPORTED)
    for kw in (dict(T=65), dict(a=2, b=4, k1=1, k2=2)):
        assert few(**kw) == UNSUPPORTED
    for kw in (dict(k=9, n=16), dict(k=3, n=2), dict(n=8193), dict(h=4), dict(d=12)):
        assert few(**kw) == INVALID, kw


# ------------------------------------------------------------------------------------------ AdamW
GOOD = dict(w=1 << 30, g=2 << 30, m=3 << 30, v=4 << 30, master=0, m_scale=0, v_scale=0, count=100, first=0, w_type=0, g_type=0, moment_bits=32, weight_decay=0.1)
FORMS = [dict(), dict(w_type=1), dict(w_type=1, master=5 << 30), dict(g_type=1), dict(moment_bits=8, m_scale=6 << 30, v_scale=7 << 30)]


def adamw(rates=0, tensor=None, **kw):
    t, p = B.moe_adamw_tensor(), B.moe_adamw_params(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 0)
    for q, v in {**GOOD, **(tensor or {})}.items():
        setattr(t, q, v)
    for q, v in kw.items():
        setattr(p, q, v)
    return B.lib().moe_adamw(ctypes.byref(t), ctypes.c_int32(1), ctypes.byref(p), ctypes.c_void_p(rates), ctypes.c_void_p(0))


@pytest.mark.parametrize("form", FORMS)
def test_adamw(form):
    assert adamw(tensor=form) not in (INVALID, UNSUPPORTED)
    whole = {**GOOD, **form}
    for q in ("w", "g", "m", "v"):
        for bad in (0, whole[q] + 4, whole[q] + 16):
            assert adamw(tensor={**form, q: bad}) == INVALID, q
    if whole["master"]:
        assert adamw(tensor={**form, "master": whole["master"] + 16}) == INVALID
    if whole["moment_bits"] == 8:
        for q in ("m_scale", "v_scale"):
            assert adamw(tensor={**form, q: 0}) == INVALID and adamw(tensor={**form, q: whole[q] + 2}) == INVALID
            assert adamw(tensor={**form, q: whole[q] + 4}) != INVALID
    for kw in (dict(count=-1), dict(count=2 ** 41), dict(w_type=2), dict(g_type=-1), dict(moment_bits=16), dict(weight_decay=-0.1), dict(weight_decay=NAN), dict(weight_decay=INF), dict(first=64),
               dict(first=-128)):
        assert adamw(tensor={**form, **kw}) == INVALID, kw
    for kw in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=0.0), dict(eps=1e-46), dict(eps=INF), dict(step=0), dict(lr=NAN), dict(grad_scale=INF)):
        assert adamw(tensor=form, **kw) == INVALID, kw
    for kw in (dict(beta1=0.0), dict(beta2=0.0), dict(lr=0.0), dict(step=2 ** 31 - 1), dict(eps=1.2e-38)):
        assert adamw(tensor=form, **kw) != INVALID, kw


def test_adamw_masters_are_for_bf16_weights():
    assert adamw(tensor=dict(master=5 << 30)) == INVALID


def test_adamw_rates():
    assert adamw(rates=1 << 20) != INVALID and adamw(rates=(1 << 20) + 2) == INVALID
    for kw in (dict(step=0), dict(lr=NAN), dict(grad_scale=INF)):  # in the place of which the rates are read
        assert adamw(rates=1 << 20, **kw) != INVALID
