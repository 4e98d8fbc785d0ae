"""What moe_layer_norm*, moe_router_losses, the *_added calls and moe_muon refuse, before anything is launched (no GPU), and their sizes."""
import ctypes

import pytest
import torch

from paper_1701_06538_b200 import binding as B
from paper_1701_06538_b200 import build as moe_build

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
NULL, SOME, ODD = ctypes.c_void_p(0), ctypes.c_void_p(4096), ctypes.c_void_p(4100)
F, I = ctypes.c_float, ctypes.c_int32


@pytest.fixture(scope="module")
def lib():
    moe_build.build()
    return B.lib()


def cfg(T=16, d=64, h=64, n=8, k=2, act="f32", **kw):
    return B.make_config(T, d, h, n, k, act, **kw)


def at(i):
    return ctypes.c_void_p(1 << 20 | i << 16)


def test_layer_norm(lib):
    c = ctypes.byref(cfg())
    good = [SOME, SOME, NULL, F(1e-5), SOME, NULL, NULL, NULL]
    for i in (0, 1, 4):
        for bad in (NULL, ODD):
            assert lib.moe_layer_norm(c, *good[:i], bad, *good[i + 1:]) == INVALID, i
    for i in (2, 5, 6):
        assert lib.moe_layer_norm(c, *good[:i], ODD, *good[i + 1:]) == INVALID, i
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert lib.moe_layer_norm(c, SOME, SOME, NULL, F(eps), SOME, NULL, NULL, NULL) == INVALID
    wide = ctypes.byref(cfg(d=16388))
    assert lib.moe_layer_norm(wide, *good) == UNSUPPORTED and lib.moe_layer_norm(ctypes.byref(cfg(d=3)), *good) == INVALID and lib.moe_layer_norm(None, *good) == INVALID
    full = [SOME] * 10 + [NULL]
    for i in (0, 1, 2, 3, 4, 6, 7, 9):
        for bad in (NULL, ODD):
            assert lib.moe_layer_norm_bwd(c, *full[:i], bad, *full[i + 1:]) == INVALID, i
    for i in (5, 8):
        assert lib.moe_layer_norm_bwd(c, *full[:i], ODD, *full[i + 1:]) == INVALID, i
    assert lib.moe_layer_norm_bwd(wide, *full) == UNSUPPORTED
    assert lib.moe_layer_norm_workspace_bytes(c, None) == INVALID
    for x in (cfg(T=0), cfg(T=1), cfg(T=100000, d=1024, act="bf16")):
        need = B.moe_layer_norm_workspace_bytes(x)
        assert need > 0 and B.moe_check_buffer_sizes(x, 7, need) == 0 and B.moe_check_buffer_sizes(x, 7, need - 1) == WORKSPACE
    assert B.moe_check_buffer_sizes(cfg(d=16388), 7, 1 << 40) == UNSUPPORTED


def router(lib, c=None, logits=at(0), idx=at(1), keep=NULL, off=NULL, S=1, wb=0.1, wz=0.1, losses=at(2), counts=at(3), sums=NULL, dlogits=NULL, ws=at(8)):
    return lib.moe_router_losses(ctypes.byref(c or cfg()), logits, idx, keep, off, I(S), F(wb), F(wz), losses, counts, sums, dlogits, ws, NULL)


def test_router_losses(lib):
    for q in ("logits", "idx", "losses", "counts", "ws"):
        for bad in (NULL, ODD):
            assert router(lib, **{q: bad}) == INVALID, q
    for q in ("keep", "off", "sums", "dlogits"):
        assert router(lib, **{q: ODD}) == INVALID, q
    for S in (0, -1, 4097):
        assert router(lib, S=S, off=at(4)) == INVALID
        out = ctypes.c_size_t(0)
        assert lib.moe_router_losses_workspace_bytes(ctypes.byref(cfg()), I(S), ctypes.byref(out)) == INVALID
    assert router(lib, S=2) == INVALID  # sequences without their offsets
    for bad in (float("nan"), float("inf")):
        assert router(lib, wb=bad) == INVALID and router(lib, wz=bad) == INVALID
    assert router(lib, c=cfg(n=8, k=2, a=2, b=4, k1=1, k2=2)) == UNSUPPORTED
    assert lib.moe_router_losses(None, *([SOME] * 4), I(1), F(1), F(1), *([SOME] * 5), NULL) == INVALID
    assert lib.moe_router_losses_workspace_bytes(ctypes.byref(cfg()), I(1), None) == INVALID
    # outputs that share memory with an input or another output: 16 x 8 logits are 512 bytes
    inside = ctypes.c_void_p(at(0).value + 480)
    for q in ("losses", "counts", "sums", "dlogits"):
        assert router(lib, **{q: at(0)}) == INVALID and router(lib, **{q: inside}) == INVALID and router(lib, **{q: at(1)}) == INVALID, q
    assert router(lib, losses=at(3)) == INVALID and router(lib, dlogits=at(3)) == INVALID and router(lib, sums=at(3)) == INVALID
    assert router(lib, keep=at(4), dlogits=at(4)) == INVALID and router(lib, off=at(4), sums=at(4), S=3) == INVALID
    assert B.moe_router_losses_workspace_bytes(cfg(T=100000, n=128), 1) < 100000 * 128 * 4 / 100


def test_added(lib):
    hier = cfg(n=8, k=2, a=2, b=4, k1=1, k2=2)
    gate = lambda c, more: lib.moe_gate_bwd_added(ctypes.byref(c), *([SOME] * 12), more, *([SOME] * 4), NULL)
    back = lambda c, more: lib.moe_backward_added(ctypes.byref(c), *([SOME] * 10), more, *([SOME] * 8), NULL)
    layer = lambda c, more, keep=SOME: lib.moe_layer_backward_added(ctypes.byref(c), *([SOME] * 9), keep, F(0.1), SOME, more, *([SOME] * 8), NULL)
    for call in (gate, back, layer):
        assert call(cfg(), ODD) == INVALID and call(hier, SOME) == UNSUPPORTED and call(cfg(k=9), SOME) == INVALID
    assert layer(cfg(), SOME, NULL) == INVALID
    for i in range(12):
        args = [SOME] * 17 + [NULL]
        args[i] = NULL
        assert lib.moe_gate_bwd_added(ctypes.byref(cfg()), *args) == INVALID, i


def test_muon(lib):
    def one(**kw):
        t = B.moe_muon_tensor(4096, 8192, None, 12288, 2, 8, 16, 0, 0, 0, 0.0, 1.0)
        for q, v in kw.items():
            setattr(t, q, v)
        return t

    def call(t, count=1, ws=SOME, rates=None, **kw):
        p = B.moe_muon_params(1e-3, 0.95, 1e-7, 1.0, 5, 1)
        for q, v in kw.items():
            setattr(p, q, v)
        return lib.moe_muon(ctypes.byref(t) if t is not None else None, I(count), ctypes.byref(p), rates, ws, NULL)

    nan, inf = float("nan"), float("inf")
    for kw in (dict(w=0), dict(g=0), dict(m=0), dict(w=4100), dict(g=4100), dict(m=4104), dict(count=-1), dict(count=2 ** 24 + 1), dict(rows=0), dict(cols=-1), dict(rows=32769), dict(cols=32769), dict(w_type=2),
               dict(g_type=-1), dict(m_type=7), dict(weight_decay=-0.1), dict(weight_decay=nan), dict(weight_decay=inf), dict(scale=nan), dict(scale=inf), dict(master=16384),
               dict(w_type=1, master=16388)):
        assert call(one(**kw)) == INVALID, kw
        out = ctypes.c_size_t(0)
        assert lib.moe_muon_workspace_bytes(ctypes.byref(one(**kw)), I(1), ctypes.byref(out)) == INVALID, kw
    for kw in (dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-46), dict(eps=inf), dict(eps=nan), dict(steps=0), dict(steps=17), dict(nesterov=2),
               dict(lr=nan), dict(lr=inf), dict(grad_scale=nan), dict(ws=NULL), dict(ws=ctypes.c_void_p(4096 + 32)), dict(rates=ctypes.c_void_p(4098))):
        assert call(one(), **kw) == INVALID, kw
    assert call(None) == INVALID and call(one(), count=-1) == INVALID
    assert lib.moe_muon(None, I(0), None, None, SOME, NULL) == INVALID
    assert call(None, count=0) == 0 and call(one(count=0, w=0, g=0, m=0)) == 0  # nothing to do
    assert lib.moe_muon_workspace_bytes(None, I(0), None) == INVALID


def test_muon_sizes(lib):
    assert ctypes.sizeof(B.moe_muon_tensor) == 4 * 8 + 8 + 5 * 4 + 2 * 4 + 4 and ctypes.sizeof(B.moe_muon_params) == 4 * 8 + 2 * 4

    def need(*shapes):
        a = (B.moe_muon_tensor * len(shapes))(*[B.moe_muon_tensor(4096, 8192, None, 12288, *s, 0, 0, 0, 0.0, 1.0) for s in shapes])
        out = ctypes.c_size_t(0)
        assert lib.moe_muon_workspace_bytes(a, I(len(shapes)), ctypes.byref(out)) == 0
        return out.value

    one = need((256, 512, 1024))
    assert one < 3 * 256 * 512 * 1024 * 2
    assert need((256, 512, 1024), (256, 1024, 512), (1, 512, 256)) < 2.1 * one
    assert need((100000, 512, 1024)) < 2 ** 30 + 2 ** 29                        # 1 GiB of X at a time
    assert need((128, 512, 1024), (128, 512, 1024)) == one                      # taken together
    assert need((1, 32768, 32768)) > 2 * 2 * 2 ** 30
    assert need((1000, 64, 128), (3, 8, 768)) == 256                            # one block's work from beginning to end


def test_muon_list_checks_its_tensors():
    t = dict(w=torch.zeros(4, 8), g=torch.zeros(4, 8), m=torch.zeros(4, 8))
    for kw in (dict(g=None), dict(m=None), dict(m=torch.zeros(8, 4)), dict(g=torch.zeros(4, 8, dtype=torch.float64)), dict(w=torch.zeros(4, 8, dtype=torch.float16)), dict(w=torch.zeros(32)),
               dict(master=torch.zeros(4, 8, dtype=torch.bfloat16)), dict(g=torch.zeros(1, 4, 8))):
        with pytest.raises((ValueError, AssertionError)):
            B.moe_muon_list([dict(t, **kw)])
