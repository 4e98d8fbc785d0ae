"""ctypes binding of the C ABI declared in include/moe.h.

Argument marshalling only: every function here has the name and the argument order of its
C counterpart, takes torch CUDA tensors (device memory) where the C function takes device
pointers, enqueues on torch's current stream and raises `MoeError` on a non-zero status.
There is no fallback: if the shared library has not been built, importing it fails loudly.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmoe_b200.so")

MOE_F32, MOE_BF16 = 0, 1
MOE_FLAG_GATE_SCREEN_OFF, MOE_FLAG_GATE_SCREEN_ON, MOE_FLAG_TC_ONE_CTA, MOE_FLAG_RECOMPUTE_HID = 1, 2, 4, 8
STATUS_NAMES = {0: "MOE_OK", 1: "MOE_ERR_INVALID_ARG", 2: "MOE_ERR_UNSUPPORTED", 3: "MOE_ERR_WORKSPACE",
                4: "MOE_ERR_CUDA", 5: "MOE_ERR_TIMEOUT"}

EXPORTS = ["moe_debug_launch_count", "moe_validate", "moe_query_sizes", "moe_workspace_bytes", "moe_query_ctx_layout", "moe_status_string", "moe_check_status",
           "moe_gate", "moe_dispatch", "moe_dispatch_noalloc", "moe_expert_ffn", "moe_combine", "moe_losses", "moe_combine_bwd",
           "moe_expert_ffn_bwd", "moe_dispatch_bwd", "moe_losses_bwd", "moe_gate_bwd", "moe_forward",
           "moe_backward", "moe_combine_layer", "moe_combine_layer_bwd", "moe_layer_forward", "moe_layer_backward",
           "moe_expert_adam_factored", "moe_check_buffer_sizes", "moe_debug_wait_timeout", "moe_debug_bounds_violations",
           "moe_expert_ffn_bits", "moe_expert_ffn_bwd_bits", "moe_query_balanced_sizes", "moe_gate_balanced", "moe_dispatch_balanced", "moe_combine_balanced",
           "moe_combine_balanced_bwd", "moe_gate_balanced_bwd", "moe_dispatch_balanced_bwd",
           "moe_norm_in", "moe_norm_in_bwd", "moe_norm_out", "moe_norm_out_bwd", "moe_norm_workspace_bytes", "moe_few_workspace_bytes",
           "moe_forward_few", "moe_adamw", "moe_muon_workspace_bytes", "moe_muon", "moe_router_losses_workspace_bytes", "moe_router_losses", "moe_gate_bwd_added",
           "moe_backward_added", "moe_layer_backward_added", "moe_layer_norm", "moe_layer_norm_bwd", "moe_layer_norm_workspace_bytes"]


class MoeError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__(f"{fn} returned {STATUS_NAMES.get(status, status)}")
        self.status = status


class moe_config(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("T", "d", "h", "n", "k", "a", "k1", "b", "k2", "act")] + \
               [("w_importance", ctypes.c_float), ("w_load", ctypes.c_float), ("flags", ctypes.c_int32)]


class moe_sizes(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in
                ("R", "gate_cols", "logits_elems", "gates_elems", "kth_elems", "wg_elems", "load_elems",
                 "dload_elems", "ws_bytes", "ws_fwd_bytes", "ws_bwd_bytes", "ctx_bytes", "adam_state_elems",
                 "ws_adam_bytes")]


class moe_ctx_layout(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in
                ("topk_idx", "gates", "clean", "raw_noise", "kth_vals", "kth_idx", "xs", "perm", "inv_perm",
                 "counts", "offsets", "hid", "ys", "importance", "load", "losses", "relu_bits")]


class moe_balanced_sizes(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in ("m", "R", "mask_words", "ws_bytes")]


class moe_adamw_tensor(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("w", "g", "master", "m", "v", "m_scale", "v_scale")] + \
               [(name, ctypes.c_int64) for name in ("count", "first")] + \
               [(name, ctypes.c_int32) for name in ("w_type", "g_type", "moment_bits")] + [("weight_decay", ctypes.c_float)]


class moe_adamw_params(ctypes.Structure):
    _fields_ = [(name, ctypes.c_double) for name in ("lr", "beta1", "beta2", "eps", "grad_scale")] + [("step", ctypes.c_int32), ("seed", ctypes.c_uint32)]


class moe_muon_tensor(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("w", "g", "master", "m")] + [("count", ctypes.c_int64)] + \
               [(name, ctypes.c_int32) for name in ("rows", "cols", "w_type", "g_type", "m_type")] + [(name, ctypes.c_float) for name in ("weight_decay", "scale")]


class moe_muon_params(ctypes.Structure):
    _fields_ = [(name, ctypes.c_double) for name in ("lr", "momentum", "eps", "grad_scale")] + [("steps", ctypes.c_int32), ("nesterov", ctypes.c_int32)]


_lib = None


def lib():
    """The loaded shared library. Raises if it was not built (python -m paper_1701_06538_b200.build)."""
    global _lib
    if _lib is None:
        path = os.environ.get("MOE_B200_LIB", LIB_PATH)  # e.g. the checking build (libmoe_b200_check.so), for the test that runs it
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with `python -m paper_1701_06538_b200.build`; "
                              "there is no fallback path")
        L = ctypes.CDLL(path)
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int32
        L.moe_status_string.restype = ctypes.c_char_p
        L.moe_debug_launch_count.restype = ctypes.c_int64
        L.moe_debug_bounds_violations.restype = ctypes.c_int64
        _lib = L
    return _lib


def make_config(T, d, h, n, k, act, w_importance=0.1, w_load=0.1, a=0, k1=0, b=0, k2=0, flags=0) -> moe_config:
    act_id = {"f32": MOE_F32, "bf16": MOE_BF16}.get(act, act)
    return moe_config(T, d, h, n, k, a, k1, b, k2, act_id, w_importance, w_load, flags)


def act_dtype(cfg: moe_config):
    return torch.bfloat16 if cfg.act == MOE_BF16 else torch.float32


def _p(t):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


# The current stream's handle without an object for the stream, 0.3 us instead of 4 to 5 (half of what a call's marshalling took)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


_prototypes = {}  # (name, kinds of the arguments) -> function with these argument types, so that pointers are passed as plain integers
_KINDS = {float: ctypes.c_float, int: ctypes.c_int32}


def _function(name, kinds):
    fn = getattr(lib(), name)
    types = [ctypes.POINTER(moe_config)] + [_KINDS.get(k, ctypes.c_void_p) for k in kinds]
    return ctypes.CFUNCTYPE(ctypes.c_int32, *types)(ctypes.cast(fn, ctypes.c_void_p).value)


def _call(name, cfg, *tensors, stream=True):
    # device tensors become pointers; a Python float is a `float` argument passed by value
    kinds, args = [], [cfg]
    for t in tensors:
        kind = None if isinstance(t, torch.Tensor) else float if isinstance(t, float) else int if isinstance(t, int) else None
        kinds.append(kind)
        args.append(t if kind else _p(t))
    if stream:
        kinds.append(None)
        args.append(_stream())
    key = (name, *kinds)
    fn = _prototypes.get(key)
    if fn is None:
        fn = _prototypes[key] = _function(name, kinds)
    status = fn(*args)
    if status != 0:
        raise MoeError(name, status)


def moe_debug_launch_count() -> int:
    return int(lib().moe_debug_launch_count())


def moe_validate(cfg) -> int:
    return lib().moe_validate(ctypes.byref(cfg))


def moe_workspace_bytes(cfg):
    """(forward, backward) workspace bytes."""
    f, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    status = lib().moe_workspace_bytes(ctypes.byref(cfg), ctypes.byref(f), ctypes.byref(b))
    if status:
        raise MoeError("moe_workspace_bytes", status)
    return f.value, b.value


def moe_query_sizes(cfg) -> moe_sizes:
    out = moe_sizes()
    status = lib().moe_query_sizes(ctypes.byref(cfg), ctypes.byref(out))
    if status != 0:
        raise MoeError("moe_query_sizes", status)
    return out


def moe_query_ctx_layout(cfg) -> moe_ctx_layout:
    out = moe_ctx_layout()
    status = lib().moe_query_ctx_layout(ctypes.byref(cfg), ctypes.byref(out))
    if status != 0:
        raise MoeError("moe_query_ctx_layout", status)
    return out


def moe_check_buffer_sizes(cfg, which, nbytes) -> int:
    return lib().moe_check_buffer_sizes(ctypes.byref(cfg), ctypes.c_int32(which), ctypes.c_size_t(nbytes))


def moe_debug_wait_timeout(ws, limit_ns):
    status = lib().moe_debug_wait_timeout(ctypes.c_void_p(_p(ws)), ctypes.c_int64(limit_ns), ctypes.c_void_p(_stream()))
    if status:
        raise MoeError("moe_debug_wait_timeout", status)


def moe_debug_bounds_violations() -> int:
    return int(lib().moe_debug_bounds_violations())


def moe_check_status(ws) -> int:
    return lib().moe_check_status(ctypes.c_void_p(_p(ws)), ctypes.c_void_p(_stream()))


def moe_gate(cfg, x, Wg, Wnoise, noise, topk_idx, gates, clean, raw_noise, kth_vals, kth_idx, ws):
    _call("moe_gate", cfg, x, Wg, Wnoise, noise, topk_idx, gates, clean, raw_noise, kth_vals, kth_idx, ws)


def moe_dispatch(cfg, x, topk_idx, xs, perm, inv_perm, counts, offsets, ws):
    _call("moe_dispatch", cfg, x, topk_idx, xs, perm, inv_perm, counts, offsets, ws)


def moe_dispatch_noalloc(cfg, x, topk_idx, xs, perm, inv_perm, counts, offsets):
    """moe_dispatch for callers that cannot provide a workspace: the scratch is a fixed array inside
    the library (see include/moe.h for the size limit and the sharing rules)."""
    _call("moe_dispatch_noalloc", cfg, x, topk_idx, xs, perm, inv_perm, counts, offsets)


def moe_expert_ffn(cfg, xs, offsets, W1, b1, W2, b2, hid, ys, ws):
    _call("moe_expert_ffn", cfg, xs, offsets, W1, b1, W2, b2, hid, ys, ws)


def moe_expert_ffn_bits(cfg, xs, offsets, W1, b1, W2, b2, hid, ys, relu_bits, ws):
    _call("moe_expert_ffn_bits", cfg, xs, offsets, W1, b1, W2, b2, hid, ys, relu_bits, ws)


def moe_expert_ffn_bwd_bits(cfg, xs, hid, relu_bits, dys, offsets, W1, W2, dxs, dW1, db1, dW2, db2, ws):
    _call("moe_expert_ffn_bwd_bits", cfg, xs, hid, relu_bits, dys, offsets, W1, W2, dxs, dW1, db1, dW2, db2, ws)


def moe_combine(cfg, ys, gates, inv_perm, y):
    _call("moe_combine", cfg, ys, gates, inv_perm, y)


def moe_losses(cfg, topk_idx, gates, clean, raw_noise, kth_vals, importance, load, losses, ws):
    _call("moe_losses", cfg, topk_idx, gates, clean, raw_noise, kth_vals, importance, load, losses, ws)


def moe_combine_bwd(cfg, dY, ys, gates, inv_perm, dgates, dys):
    _call("moe_combine_bwd", cfg, dY, ys, gates, inv_perm, dgates, dys)


def moe_expert_ffn_bwd(cfg, xs, hid, dys, offsets, W1, W2, dxs, dW1, db1, dW2, db2, ws):
    _call("moe_expert_ffn_bwd", cfg, xs, hid, dys, offsets, W1, W2, dxs, dW1, db1, dW2, db2, ws)


def moe_dispatch_bwd(cfg, dxs, inv_perm, dX_expert):
    _call("moe_dispatch_bwd", cfg, dxs, inv_perm, dX_expert)


def moe_losses_bwd(cfg, importance, load, topk_idx, dgates, dload, ws):
    _call("moe_losses_bwd", cfg, importance, load, topk_idx, dgates, dload, ws)


def moe_gate_bwd(cfg, x, Wg, Wnoise, noise, clean, raw_noise, topk_idx, gates, kth_vals, kth_idx, dgates, dload,
                 dWg, dWnoise, dX_gate, ws):
    _call("moe_gate_bwd", cfg, x, Wg, Wnoise, noise, clean, raw_noise, topk_idx, gates, kth_vals, kth_idx, dgates,
          dload, dWg, dWnoise, dX_gate, ws)


def moe_forward(cfg, x, Wg, Wnoise, noise, W1, b1, W2, b2, y, losses, importance, load, counts, ctx, ws):
    _call("moe_forward", cfg, x, Wg, Wnoise, noise, W1, b1, W2, b2, y, losses, importance, load, counts, ctx, ws)


def moe_backward(cfg, dY, x, Wg, Wnoise, noise, W1, b1, W2, b2, ctx, dX, dWg, dWnoise, dW1, db1, dW2, db2, ws):
    _call("moe_backward", cfg, dY, x, Wg, Wnoise, noise, W1, b1, W2, b2, ctx, dX, dWg, dWnoise, dW1, db1, dW2, db2,
          ws)


def moe_query_balanced_sizes(cfg) -> moe_balanced_sizes:
    out = moe_balanced_sizes()
    status = lib().moe_query_balanced_sizes(ctypes.byref(cfg), ctypes.byref(out))
    if status != 0:
        raise MoeError("moe_query_balanced_sizes", status)
    return out


def moe_gate_balanced(cfg, x, Wg, thresholds, logits, probs, mask_bits, tok_of_row, offsets, den, tok_ptr, tok_rows,
                      loss_batchwise, thr_counts, ws):
    _call("moe_gate_balanced", cfg, x, Wg, thresholds, logits, probs, mask_bits, tok_of_row, offsets, den, tok_ptr,
          tok_rows, loss_batchwise, thr_counts, ws)


def moe_dispatch_balanced(cfg, x, tok_of_row, xs):
    _call("moe_dispatch_balanced", cfg, x, tok_of_row, xs)


def moe_combine_balanced(cfg, ys, probs, den, tok_ptr, tok_rows, y):
    _call("moe_combine_balanced", cfg, ys, probs, den, tok_ptr, tok_rows, y)


def moe_combine_balanced_bwd(cfg, dY, ys, probs, den, tok_of_row, dG_row, dys):
    _call("moe_combine_balanced_bwd", cfg, dY, ys, probs, den, tok_of_row, dG_row, dys)


def moe_gate_balanced_bwd(cfg, x, Wg, probs, mask_bits, den, thresholds, tok_ptr, tok_rows, dG_row, thr_counts, w_batchwise,
                          dWg, dX_gate, dthresholds, ws):
    _call("moe_gate_balanced_bwd", cfg, x, Wg, probs, mask_bits, den, thresholds, tok_ptr, tok_rows, dG_row, thr_counts,
          float(w_batchwise), dWg, dX_gate, dthresholds, ws)


def moe_dispatch_balanced_bwd(cfg, dxs, tok_ptr, tok_rows, dX_gate, dX):
    _call("moe_dispatch_balanced_bwd", cfg, dxs, tok_ptr, tok_rows, dX_gate, dX)


def moe_expert_adam_factored(cfg, W1, b1, W2, b2, dW1, db1, dW2, db2, state, lr, beta2, eps, step, ws):
    _call("moe_expert_adam_factored", cfg, W1, b1, W2, b2, dW1, db1, dW2, db2, state, float(lr), float(beta2), float(eps),
          int(step), ws)


def moe_combine_layer(cfg, ys, gates, inv_perm, x, keep_bits, drop_prob, out):
    _call("moe_combine_layer", cfg, ys, gates, inv_perm, x, keep_bits, float(drop_prob), out)


def moe_combine_layer_bwd(cfg, dOut, ys, gates, inv_perm, keep_bits, drop_prob, dgates, dys):
    _call("moe_combine_layer_bwd", cfg, dOut, ys, gates, inv_perm, keep_bits, float(drop_prob), dgates, dys)


def moe_layer_forward(cfg, x, Wg, Wnoise, noise, W1, b1, W2, b2, keep_bits, drop_prob, out, losses, importance, load,
                      counts, ctx, ws):
    _call("moe_layer_forward", cfg, x, Wg, Wnoise, noise, W1, b1, W2, b2, keep_bits, float(drop_prob), out, losses,
          importance, load, counts, ctx, ws)


def moe_layer_backward(cfg, dOut, x, Wg, Wnoise, noise, W1, b1, W2, b2, keep_bits, drop_prob, ctx, dX, dWg, dWnoise,
                       dW1, db1, dW2, db2, ws):
    _call("moe_layer_backward", cfg, dOut, x, Wg, Wnoise, noise, W1, b1, W2, b2, keep_bits, float(drop_prob), ctx, dX,
          dWg, dWnoise, dW1, db1, dW2, db2, ws)


def _one_size(name, cfg):
    out = ctypes.c_size_t(0)
    status = getattr(lib(), name)(ctypes.byref(cfg), ctypes.byref(out))
    if status:
        raise MoeError(name, status)
    return out.value


def moe_norm_workspace_bytes(cfg) -> int:
    return _one_size("moe_norm_workspace_bytes", cfg)


_bound_functions = {}


def _bound(name, kinds):
    """The function of the library with its argument types: c a configuration, p a pointer, i an int, f a float; the stream comes last. Calls of a few microseconds
    go this way: sorting out a call's fifteen arguments by their types took as long as the launch."""
    fn = _bound_functions.get(name)
    if fn is None:
        types = dict(c=ctypes.POINTER(moe_config), p=ctypes.c_void_p, i=ctypes.c_int32, f=ctypes.c_float)
        raw = ctypes.cast(getattr(lib(), name), ctypes.c_void_p).value
        fn = _bound_functions[name] = ctypes.CFUNCTYPE(ctypes.c_int32, *[types[k] for k in kinds], ctypes.c_void_p)(raw)
    return fn


def _checked(name, status):
    if status != 0:
        raise MoeError(name, status)


def _here():
    """_p for a call whose tensors have to be where it runs: on the current device."""
    device = torch.cuda.current_device()

    def p(t):
        if t is None:
            return None
        if t.get_device() != device:
            raise ValueError("a tensor is not on the current device")
        assert t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
        return t.data_ptr()
    return p


def moe_norm_in(cfg, x, w, eps, xn, rstd):
    p = _here()
    _checked("moe_norm_in", _bound("moe_norm_in", "cppfpp")(cfg, p(x), p(w), eps, p(xn), p(rstd), _stream()))


def moe_norm_in_bwd(cfg, dxn, x, w, rstd, dres, dX, dw, ws):
    p = _here()
    _checked("moe_norm_in_bwd", _bound("moe_norm_in_bwd", "cpppppppp")(cfg, p(dxn), p(x), p(w), p(rstd), p(dres), p(dX), p(dw), p(ws), _stream()))


def moe_norm_out(cfg, x, y, w, gate, rows_per_gate, residual_scale, w_next, eps, out, next, rstd, rstd_next):
    p = _here()
    _checked("moe_norm_out", _bound("moe_norm_out", "cppppifpfpppp")(cfg, p(x), p(y), p(w), p(gate), rows_per_gate, residual_scale, p(w_next), eps, p(out),
                                                                     p(next), p(rstd), p(rstd_next), _stream()))


def moe_norm_out_bwd(cfg, dOut, dNext, out, y, w, gate, rows_per_gate, residual_scale, w_next, rstd, rstd_next, dX, dY, dw, dgate, dw_next,
                     ws):
    p = _here()
    _checked("moe_norm_out_bwd", _bound("moe_norm_out_bwd", "cppppppifppppppppp")(cfg, p(dOut), p(dNext), p(out), p(y), p(w), p(gate), rows_per_gate, residual_scale,
                                                                                  p(w_next), p(rstd), p(rstd_next), p(dX), p(dY), p(dw), p(dgate), p(dw_next), p(ws),
                                                                                  _stream()))


def moe_few_workspace_bytes(cfg) -> int:
    return _one_size("moe_few_workspace_bytes", cfg)


def moe_forward_few(cfg, x, Wg, W1, b1, W2, b2, y, topk_idx, gates, ws):
    p = _here()
    _checked("moe_forward_few", _bound("moe_forward_few", "cpppppppppp")(cfg, p(x), p(Wg), p(W1), p(b1), p(W2), p(b2), p(y), p(topk_idx), p(gates), p(ws),
                                                                         _stream()))


class moe_adamw_list:
    """The tensors of an optimiser step, made once for a model. `tensors`: dicts with w, g, m, v and, where they apply, master, m_scale,
    v_scale (8-bit moments: m and v are torch.float8_e4m3fn or uint8), weight_decay (0), first (a running number from 0, tensor behind tensor).
    Keeps references to the tensors: their addresses are what the call gets."""

    def __init__(self, tensors):
        self.tensors = [dict(t) for t in tensors]
        self.array = (moe_adamw_tensor * max(len(self.tensors), 1))()
        types, at, self.device = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}, 0, None
        for t, r in zip(self.tensors, self.array):
            count = t["w"].numel()
            eight = t["m"].element_size() == 1
            moment = (torch.float8_e4m3fn, torch.uint8) if eight else (torch.float32,)
            blocks = -(-count // 128)
            want = dict(w=(tuple(types), count), g=(tuple(types), count), master=((torch.float32,), count), m=(moment, count), v=(moment, count),
                        m_scale=((torch.float32,), blocks), v_scale=((torch.float32,), blocks))
            for q, (dtypes, n) in want.items():
                x = t.get(q)
                if x is None:
                    if q in ("w", "g", "m", "v") or (eight and q != "master"):
                        raise ValueError(f"moe_adamw_list: {q} is missing")
                    continue
                if x.dtype not in dtypes or x.numel() != n:
                    raise ValueError(f"moe_adamw_list: {q} has {x.numel()} elements of {x.dtype}, wanted {n} of {dtypes}")
                if self.device is None:
                    self.device = x.get_device()
                if x.get_device() != self.device:
                    raise ValueError("moe_adamw_list: the tensors are on different devices")
                setattr(r, q, _p(x))
            r.count, r.first = count, t.get("first", at)
            r.w_type, r.g_type, r.moment_bits, r.weight_decay = types[t["w"].dtype], types[t["g"].dtype], 8 if eight else 32, t.get("weight_decay", 0.0)
            at = max(at, r.first + 128 * blocks)


def moe_adamw(tensors, lr, beta1, beta2, eps, step, seed=0, grad_scale=1.0, rates=None):
    """`tensors`: a moe_adamw_list. `rates`: five 4-byte words of device memory (lr, 1 - beta1^step, 1 - beta2^step, grad_scale as floats, seed) that
    are read when the kernels run."""
    if tensors.device is not None and tensors.device != torch.cuda.current_device():
        raise ValueError("moe_adamw: the tensors are not on the current device")
    if rates is not None:
        if rates.dtype not in (torch.float32, torch.int32, torch.uint32) or rates.numel() < 5 or not rates.is_contiguous():
            raise ValueError(f"moe_adamw: rates are {rates.numel()} elements of {rates.dtype}, wanted 5 contiguous 4-byte words")
        if rates.get_device() != torch.cuda.current_device():
            raise ValueError("moe_adamw: rates are not on the current device")
    p = moe_adamw_params(lr, beta1, beta2, eps, grad_scale, step, seed & 0xffffffff)
    status = lib().moe_adamw(tensors.array, ctypes.c_int32(len(tensors.tensors)), ctypes.byref(p), ctypes.c_void_p(_p(rates)), ctypes.c_void_p(_stream()))
    if status:
        raise MoeError("moe_adamw", status)


class moe_muon_list:
    """The matrices of a Muon step, made once for a model. `tensors`: dicts with w, g, m of [rows, cols] or [count, rows, cols] and, where they apply, master, weight_decay (0),
    scale (1). Keeps references to the tensors: their addresses are what the call gets."""

    def __init__(self, tensors):
        self.tensors = [dict(t) for t in tensors]
        self.array = (moe_muon_tensor * max(len(self.tensors), 1))()
        types, self.device = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}, None
        for t, r in zip(self.tensors, self.array):
            shape = tuple(t["w"].shape)
            if len(shape) not in (2, 3):
                raise ValueError(f"moe_muon_list: w is {shape}, wanted [rows, cols] or [count, rows, cols]")
            for q, dtypes in (("w", tuple(types)), ("g", tuple(types)), ("m", tuple(types)), ("master", (torch.float32,))):
                x = t.get(q)
                if x is None:
                    if q != "master":
                        raise ValueError(f"moe_muon_list: {q} is missing")
                    continue
                if x.dtype not in dtypes or tuple(x.shape) != shape:
                    raise ValueError(f"moe_muon_list: {q} is {tuple(x.shape)} of {x.dtype}, wanted {shape} of {dtypes}")
                if self.device is None:
                    self.device = x.get_device()
                if x.get_device() != self.device:
                    raise ValueError("moe_muon_list: the tensors are on different devices")
                setattr(r, q, _p(x))
            r.count, (r.rows, r.cols) = shape[0] if len(shape) == 3 else 1, shape[-2:]
            r.w_type, r.g_type, r.m_type = types[t["w"].dtype], types[t["g"].dtype], types[t["m"].dtype]
            r.weight_decay, r.scale = t.get("weight_decay", 0.0), t.get("scale", 1.0)


def moe_muon_workspace_bytes(tensors) -> int:
    out = ctypes.c_size_t(0)
    _checked("moe_muon_workspace_bytes", lib().moe_muon_workspace_bytes(tensors.array, ctypes.c_int32(len(tensors.tensors)), ctypes.byref(out)))
    return out.value


def moe_muon(tensors, lr, momentum, eps, steps, nesterov, ws, grad_scale=1.0, rates=None):
    """`tensors`: a moe_muon_list. `rates`: two floats of device memory (lr, grad_scale) that are read when the kernels run."""
    here = torch.cuda.current_device()
    if tensors.device is not None and tensors.device != here:
        raise ValueError("moe_muon: the tensors are not on the current device")
    if ws.get_device() != here:
        raise ValueError("moe_muon: the workspace is not on the current device")
    if rates is not None:
        if rates.dtype != torch.float32 or rates.numel() < 2 or not rates.is_contiguous():
            raise ValueError(f"moe_muon: rates are {rates.numel()} elements of {rates.dtype}, wanted 2 contiguous floats")
        if rates.get_device() != here:
            raise ValueError("moe_muon: rates are not on the current device")
    if ws.numel() * ws.element_size() < moe_muon_workspace_bytes(tensors):
        raise ValueError("moe_muon: the workspace is too small")
    p = moe_muon_params(lr, momentum, eps, grad_scale, steps, int(nesterov))
    _checked("moe_muon", lib().moe_muon(tensors.array, ctypes.c_int32(len(tensors.tensors)), ctypes.byref(p), ctypes.c_void_p(_p(rates)), ctypes.c_void_p(_p(ws)),
                                        ctypes.c_void_p(_stream())))


def moe_router_losses_workspace_bytes(cfg, sequences=1) -> int:
    out = ctypes.c_size_t(0)
    _checked("moe_router_losses_workspace_bytes", lib().moe_router_losses_workspace_bytes(ctypes.byref(cfg), ctypes.c_int32(sequences), ctypes.byref(out)))
    return out.value


def moe_router_losses(cfg, logits, topk_idx, keep, seq_offsets, sequences, w_balance, w_z, losses, counts, prob_sums, dlogits, ws):
    p = _here()
    _checked("moe_router_losses", _bound("moe_router_losses", "cppppiffppppp")(cfg, p(logits), p(topk_idx), p(keep), p(seq_offsets), sequences, w_balance, w_z, p(losses), p(counts),
                                                                               p(prob_sums), p(dlogits), p(ws), _stream()))


def moe_gate_bwd_added(cfg, x, Wg, Wnoise, noise, clean, raw_noise, topk_idx, gates, kth_vals, kth_idx, dgates, dload, dlogits, dWg, dWnoise, dX_gate, ws):
    _call("moe_gate_bwd_added", cfg, x, Wg, Wnoise, noise, clean, raw_noise, topk_idx, gates, kth_vals, kth_idx, dgates, dload, dlogits, dWg, dWnoise, dX_gate, ws)


def moe_backward_added(cfg, dY, x, Wg, Wnoise, noise, W1, b1, W2, b2, ctx, dlogits, dX, dWg, dWnoise, dW1, db1, dW2, db2, ws):
    _call("moe_backward_added", cfg, dY, x, Wg, Wnoise, noise, W1, b1, W2, b2, ctx, dlogits, dX, dWg, dWnoise, dW1, db1, dW2, db2, ws)


def moe_layer_backward_added(cfg, dOut, x, Wg, Wnoise, noise, W1, b1, W2, b2, keep_bits, drop_prob, ctx, dlogits, dX, dWg, dWnoise, dW1, db1, dW2, db2, ws):
    _call("moe_layer_backward_added", cfg, dOut, x, Wg, Wnoise, noise, W1, b1, W2, b2, keep_bits, float(drop_prob), ctx, dlogits, dX, dWg, dWnoise, dW1, db1, dW2, db2, ws)


def moe_layer_norm_workspace_bytes(cfg) -> int:
    return _one_size("moe_layer_norm_workspace_bytes", cfg)


def moe_layer_norm(cfg, x, w, b, eps, xn, mean, rstd):
    p = _here()
    _checked("moe_layer_norm", _bound("moe_layer_norm", "cpppfppp")(cfg, p(x), p(w), p(b), eps, p(xn), p(mean), p(rstd), _stream()))


def moe_layer_norm_bwd(cfg, dxn, x, w, mean, rstd, dres, dX, dw, db, ws):
    p = _here()
    _checked("moe_layer_norm_bwd", _bound("moe_layer_norm_bwd", "cpppppppppp")(cfg, p(dxn), p(x), p(w), p(mean), p(rstd), p(dres), p(dX), p(dw), p(db), p(ws), _stream()))


# ----------------------------------------------------------------------------------------------
# Buffer helpers (allocation only; torch is the allocator, nothing is computed here)
# ----------------------------------------------------------------------------------------------
def empty_bytes(nbytes, device="cuda"):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def ctx_views(cfg, ctx):
    """Typed views of the tensors moe_forward saved in `ctx` (no copies)."""
    L, S = moe_query_ctx_layout(cfg), moe_query_sizes(cfg)
    T, d, h, n, k, R = cfg.T, cfg.d, cfg.h, cfg.n, cfg.k, S.R
    adt = act_dtype(cfg)
    esz = 2 if cfg.act == MOE_BF16 else 4

    def view(off, count, dtype, shape):
        size = torch.empty((), dtype=dtype).element_size()
        return ctx[off:off + count * size].view(dtype).view(*shape)

    views = dict(topk_idx=view(L.topk_idx, R, torch.int32, (T, k)),
                gates=view(L.gates, S.gates_elems, torch.float32, (-1,)),
                clean=view(L.clean, S.logits_elems, torch.float32, (-1,)),
                raw_noise=view(L.raw_noise, S.logits_elems, torch.float32, (-1,)),
                kth_vals=view(L.kth_vals, S.kth_elems, torch.float32, (-1, 2)),
                kth_idx=view(L.kth_idx, S.kth_elems, torch.int32, (-1, 2)),
                xs=view(L.xs, R * d, adt, (R, d)), perm=view(L.perm, R, torch.int32, (R,)),
                inv_perm=view(L.inv_perm, R, torch.int32, (R,)), counts=view(L.counts, n, torch.int32, (n,)),
                offsets=view(L.offsets, n + 1, torch.int32, (n + 1,)),
                ys=view(L.ys, R * d, adt, (R, d)), importance=view(L.importance, n, torch.float32, (n,)),
                load=view(L.load, S.load_elems, torch.float32, (-1,)), losses=view(L.losses, 2, torch.float32, (2,)))
    if not cfg.flags & MOE_FLAG_RECOMPUTE_HID:  # with the flag the context keeps no hidden activations
        views["hid"] = view(L.hid, R * h, adt, (R, h))
        if L.relu_bits + R * (h // 32) * 4 <= S.ctx_bytes and h % 32 == 0 and L.relu_bits > L.losses:
            views["relu_bits"] = view(L.relu_bits, R * (h // 32), torch.int32, (R, h // 32))
    return views
