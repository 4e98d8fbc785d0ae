"""What moe_norm_*, moe_forward_few and moe_adamw refuse, before anything is launched (no GPU), and their sizes."""
import ctypes

import pytest
import torch

from paper_1701_06538_b200 import binding as B
from paper_1701_06538_b200 import build as moe_build

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
NULL, SOME, ODD = ctypes.c_void_p(0), ctypes.c_void_p(4096), ctypes.c_void_p(4100)
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    return B.lib()


def cfg(T=16, d=64, h=64, n=8, k=2, act="f32", **kw):
    return B.make_config(T, d, h, n, k, act, **kw)


def test_struct_layouts_match_header():
    assert ctypes.sizeof(B.moe_adamw_tensor) == 7 * 8 + 2 * 8 + 4 * 4
    assert ctypes.sizeof(B.moe_adamw_params) == 5 * 8 + 2 * 4


def test_norms(lib):
    c = ctypes.byref(cfg())
    good = [SOME, SOME, F(1e-6), SOME, SOME, NULL]
    for i in (0, 1, 3):
        for bad in (NULL, ODD):
            assert lib.moe_norm_in(c, *good[:i], bad, *good[i + 1:]) == INVALID
    assert lib.moe_norm_in(c, SOME, SOME, F(1e-6), SOME, ODD, NULL) == INVALID
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert lib.moe_norm_in(c, SOME, SOME, F(eps), SOME, SOME, NULL) == INVALID
    out = lambda c=c, x=SOME, gate=NULL, per=0, scale=1.0, nxt=NULL, eps=1e-6, next_out=NULL: lib.moe_norm_out(
        c, x, SOME, SOME, gate, per, F(scale), nxt, F(eps), SOME, next_out, SOME, next_out, NULL)
    assert out(x=NULL) == INVALID and out(gate=ODD, per=1) == INVALID and out(gate=SOME, per=0) == INVALID and out(gate=SOME, per=-3) == INVALID
    assert out(scale=float("inf")) == INVALID and out(eps=0.0) == INVALID and out(nxt=SOME) == INVALID
    wide = ctypes.byref(cfg(d=16388))
    assert out(c=wide) == UNSUPPORTED and lib.moe_norm_in(wide, *good) == UNSUPPORTED
    assert out(c=ctypes.byref(cfg(d=3))) == INVALID
    for i in (0, 1, 2, 3, 5, 6, 7):
        args = [SOME, SOME, SOME, SOME, NULL, SOME, SOME, SOME, NULL]
        args[i] = NULL
        assert lib.moe_norm_in_bwd(c, *args) == INVALID
    bwd = lambda gate=NULL, per=0, dgate=NULL, nxt=NULL, dnext=SOME, ws=SOME: lib.moe_norm_out_bwd(
        c, SOME, dnext, SOME, SOME, SOME, gate, per, F(1.0), nxt, SOME, SOME, SOME, SOME, SOME, dgate, SOME, ws, NULL)
    assert bwd(gate=SOME, per=1) == INVALID and bwd(gate=SOME, per=0, dgate=SOME) == INVALID and bwd(nxt=SOME, dnext=NULL) == INVALID and bwd(ws=NULL) == INVALID
    assert lib.moe_norm_workspace_bytes(c, None) == INVALID


def test_few_tokens(lib):
    c = cfg()
    for i in (0, 1, 2, 3, 4, 5, 6, 9):
        args = [SOME] * 7 + [NULL, NULL, SOME, NULL]
        args[i] = ODD
        assert lib.moe_forward_few(ctypes.byref(c), *args) == INVALID
        args[i] = NULL
        assert lib.moe_forward_few(ctypes.byref(c), *args) == INVALID
    assert lib.moe_forward_few(ctypes.byref(c), *([SOME] * 7), ODD, NULL, SOME, NULL) == INVALID
    for other in (cfg(T=65), cfg(T=16, n=8, k=2, a=2, b=4, k1=1, k2=2)):
        assert lib.moe_forward_few(ctypes.byref(other), *([SOME] * 10), NULL) == UNSUPPORTED
        with pytest.raises(B.MoeError):
            B.moe_few_workspace_bytes(other)
    assert lib.moe_forward_few(None, *([SOME] * 10), NULL) == INVALID


def test_workspace_sizes(lib):
    for c in (cfg(T=1), cfg(T=64, d=512, h=1024, n=256, k=4, act="bf16"), cfg(T=0)):
        for which, need in ((5, B.moe_norm_workspace_bytes(c)), (6, B.moe_few_workspace_bytes(c))):
            assert need > 0
            assert B.moe_check_buffer_sizes(c, which, need) == 0 and B.moe_check_buffer_sizes(c, which, need - 1) == WORKSPACE
    assert B.moe_check_buffer_sizes(cfg(T=65), 6, 1 << 40) == UNSUPPORTED
    # a few percent of the rows themselves once there are many
    assert B.moe_norm_workspace_bytes(cfg(T=131072, d=1024, act="bf16")) < 0.2 * 131072 * 1024 * 2


def test_adamw(lib):
    def one(**kw):
        t = B.moe_adamw_tensor(4096, 4096, None, 4096, 4096, None, None, 100, 0, 0, 0, 32, 0.0)
        for q, v in kw.items():
            setattr(t, q, v)
        return t

    def call(t, count=1, **kw):
        p = B.moe_adamw_params(1e-3, 0.9, 0.999, 1e-8, 1.0, 1, 0)
        for q, v in kw.items():
            setattr(p, q, v)
        return lib.moe_adamw(ctypes.byref(t) if t is not None else None, ctypes.c_int32(count), ctypes.byref(p), None, NULL)

    for kw in (dict(w=0), dict(g=0), dict(m=0), dict(v=4100), dict(w=4112), dict(count=-1), dict(count=2 ** 41), dict(w_type=2), dict(g_type=-1), dict(moment_bits=16),
               dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(first=64), dict(first=-128), dict(master=4096), dict(w_type=1, master=4100), dict(moment_bits=8),
               dict(moment_bits=8, m_scale=4096), dict(moment_bits=8, m_scale=4096, v_scale=4097)):
        assert call(one(**kw)) == INVALID, kw
    for kw in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=1e-46), dict(eps=float("inf")), dict(step=0), dict(lr=float("nan")),
               dict(grad_scale=float("inf"))):
        assert call(one(), **kw) == INVALID, kw
    assert call(one(), count=-1) == INVALID and call(None) == INVALID
    assert lib.moe_adamw(None, ctypes.c_int32(0), None, None, NULL) == INVALID
    assert call(None, count=0) == 0 and call(one(count=0, w=0, g=0, m=0, v=0)) == 0  # nothing to do


def test_adamw_list_checks_its_tensors():
    t = dict(w=torch.zeros(8), g=torch.zeros(8), m=torch.zeros(8), v=torch.zeros(8))
    for kw in (dict(g=None), dict(m=torch.zeros(7)), dict(v=torch.zeros(8, dtype=torch.float64)), dict(w=torch.zeros(8, dtype=torch.float16)),
               dict(m=torch.zeros(8, dtype=torch.uint8), v=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises((ValueError, AssertionError)):
            B.moe_adamw_list([dict(t, **kw)])


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")
def test_outputs_in_one_place(lib):
    """Distinct addresses but for two that may not be one."""
    at = lambda i: ctypes.c_void_p(4096 * (i + 1))
    c = ctypes.byref(cfg())
    p = [at(i) for i in range(20)]
    assert lib.moe_forward_few(c, p[0], *p[1:6], p[0], NULL, NULL, p[7], NULL) == INVALID                                      # y in the place of x
    assert lib.moe_norm_out(c, p[0], p[1], p[2], NULL, 0, F(1.0), p[3], F(1e-6), p[4], p[4], p[5], p[6], NULL) == INVALID      # next in the place of out
    assert lib.moe_norm_out_bwd(c, p[0], NULL, NULL, p[1], p[2], NULL, 0, F(1.0), NULL, p[3], NULL, p[4], p[4], p[5], NULL, NULL, p[6], NULL) == INVALID  # dX and dY
