"""Plain 64-bit statements of the block's norms, of the layer without gating noise and of AdamW, with what their tolerances are made of.

u is half a step of float, 2^-24. `terms` of a result is the sum of the magnitudes that it is a sum of: float arithmetic is off by a number of
roundings times u times that, whatever the order."""
import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def within(got, want, slack, what):
    """|got - want| <= half a step of got's type (of what is wanted) + slack, element by element."""
    g = got.detach().double().cpu()
    want, slack = torch.as_tensor(want, dtype=torch.float64), torch.as_tensor(slack, dtype=torch.float64)
    assert g.shape == want.shape, (what, g.shape, want.shape)
    bound = half_step(got.dtype) * (want.abs() + slack) + slack + 1e-300
    bad = ~((g - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} elements off, worst {float(((g - want).abs() / bound).max()):.3g} times the bound"


def norm_in(x, w, eps):
    x = x.double().cpu()
    w = w.double().cpu()
    r = (x.square().mean(1) + eps).rsqrt()
    return x * r[:, None] * w, r


def rows_of_gate(gate, T, rows_per_gate):
    return gate.double().cpu()[torch.arange(T) // rows_per_gate]


def norm_out(x, y, w, gate, rows_per_gate, scale, w_next, eps):
    """out, next, rstd, rstd_next and the magnitudes of out's terms."""
    T = x.shape[0]
    x, y, w = x.double().cpu(), y.double().cpu(), w.double().cpu()
    r = (y.square().mean(1) + eps).rsqrt()
    u = y * r[:, None] * w
    if gate is not None:
        u = u * rows_of_gate(gate, T, rows_per_gate)
    out, terms = scale * x + u, (scale * x).abs() + u.abs()
    r2 = (out.square().mean(1) + eps).rsqrt()
    nxt = out * r2[:, None] * w_next.double().cpu() if w_next is not None else None
    return out, nxt, r, r2, terms


def norm_out_bwd(dOut, dNext, out, y, w, gate, rows_per_gate, scale, w_next, rstd, rstd_next):
    """{name: (value, magnitudes of its terms)}, written with the derivatives of a quotient, not with the kernel's order."""
    T, d = dOut.shape
    f = lambda t: None if t is None else t.double().cpu()
    dOut, dNext, out, y, w, w_next, rstd, rstd_next = map(f, (dOut, dNext, out, y, w, w_next, rstd, rstd_next))
    res = {}
    dt, m = dOut, dOut.abs()
    if w_next is not None:
        r2 = rstd_next[:, None]
        n2, dn2 = out * r2, dNext * w_next
        dt = dt + r2 * (dn2 - n2 * (dn2 * n2).mean(1, keepdim=True))
        m = m + r2 * (dn2.abs() + n2.abs() * (dn2 * n2).abs().mean(1, keepdim=True))
        res["dw_next"] = ((dNext * n2).sum(0), (dNext * n2).abs().sum(0))
    if y is None:
        res["dX"] = (dt, m)
        return res
    r = rstd[:, None]
    n = y * r
    g = torch.ones(1, 1, dtype=torch.float64) if gate is None else rows_of_gate(gate, T, rows_per_gate)
    b = g * w * n
    c1_terms = (m * b.abs()).mean(1, keepdim=True)
    if w_next is not None:  # the kernel's mean of dt b goes through mean(dn2 n2) mean(n2 b)
        c1_terms = c1_terms + rstd_next[:, None] * (dn2 * n2).abs().mean(1, keepdim=True) * (n2 * b).abs().mean(1, keepdim=True)
    dn = dt * g * w
    res["dY"] = (r * (dn - n * (dn * n).mean(1, keepdim=True)), r * (m * (g * w).abs() + n.abs() * c1_terms))
    res["dX"] = (scale * dt, abs(scale) * m)
    res["dw"] = ((dt * g * n).sum(0), (m * (g * n).abs()).sum(0))
    if gate is not None:
        which = torch.arange(T) // rows_per_gate
        zero = torch.zeros(gate.shape, dtype=torch.float64)
        res["dgate"] = (zero.clone().index_add_(0, which, dt * n * w), zero.clone().index_add_(0, which, (m * n * w).abs()))
    return res


def few(x, Wg, W1, b1, W2, b2, k, idx):
    """The layer for the given routing idx [T, k]: y, gates, and the bounds on how far float arithmetic with hid in two terms of the weights' type may be off."""
    dt = W1.dtype
    f = lambda t: t.detach().double().cpu()
    xd, Wgd, idx = f(x), f(Wg), idx.cpu().long()
    used = sorted(set(idx.reshape(-1).tolist()))
    W1d, b1d, W2d, b2d = ({e: f(w[e]) for e in used} for w in (W1, b1, W2, b2))
    T, d = xd.shape
    h = W1.shape[2]
    logits, logit_terms = xd @ Wgd, xd.abs() @ Wgd.abs()
    top = logits.gather(1, idx)
    gates = torch.softmax(top, 1)
    off = (d + 8) * U * logit_terms.gather(1, idx).amax(1, keepdim=True)  # of a logit: a chain of d multiply-adds
    gate_slack = gates * (4 * off + 32 * U)
    # sums of products: the matrix instruction adds with truncation, a whole step of float instead of half of one
    steps = 2 if dt == torch.bfloat16 else 1
    y, slack = torch.zeros(T, d, dtype=torch.float64), torch.zeros(T, d, dtype=torch.float64)
    for t in range(T):
        for s in range(k):
            e = int(idx[t, s])
            pre = xd[t] @ W1d[e] + b1d[e]
            hid = pre.clamp(min=0.0)
            hid_slack = steps * (d + 16) * U * (xd[t].abs() @ W1d[e].abs() + b1d[e].abs())
            if dt == torch.bfloat16:
                hid_slack = hid_slack + 2.0 ** -17 * (hid + hid_slack)  # two bf16 terms: the first is off by 2^-9 of hid at most, the second by 2^-9 of that
            ys, terms = hid @ W2d[e] + b2d[e], hid @ W2d[e].abs() + b2d[e].abs()
            ys_slack = hid_slack @ W2d[e].abs() + steps * (h + 32) * U * (terms + hid_slack @ W2d[e].abs())
            y[t] += gates[t, s] * ys
            slack[t] += gates[t, s] * (ys_slack + (k + 4) * U * terms) + gate_slack[t, s] * (terms + ys_slack)
    return y, slack, gates, gate_slack


def mix(x):
    x = np.asarray(x, np.uint64)
    for shift, factor in ((16, 0x7feb352d), (15, 0x846ca68b)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xffffffff)
    return x ^ (x >> np.uint64(16))


def dither(first, count, seed):
    """The 16 random bits of m and of sqrt(v) for elements first .. first + count."""
    number = np.arange(count, dtype=np.uint64) + np.uint64(first)
    key = mix((np.uint64(seed) + (number >> np.uint64(32)) * np.uint64(0x9e3779b9)) & np.uint64(0xffffffff))
    bits = mix((number & np.uint64(0xffffffff)) ^ key)
    return bits & np.uint64(0xffff), bits >> np.uint64(16)


def blocks(t, fill=0.0):
    t = np.asarray(t, np.float64)
    pad = -len(t) % 128
    return np.concatenate([t, np.full(pad, fill)]).reshape(-1, 128)


def held(codes, scale):
    """Values of e4m3 codes under their blocks' scales."""
    c = codes.view(torch.float8_e4m3fn).float().cpu().numpy()
    return (blocks(c) * scale.double().cpu().numpy()[:, None]).reshape(-1)[:len(c)]


def eight_bits(value, bits, root):
    """(codes' values, scales, how far from the border between two codes each decision was, in units of the code, and the units)."""
    value = np.asarray(value, np.float64)
    scale = np.abs(np.where(np.isfinite(blocks(value)), blocks(value), 0.0)).max(1) / 448.0
    scale = np.where(scale > 0, np.maximum(scale, 1.17549435e-38), 0.0)
    q = (blocks(value) / np.where(scale > 0, scale, 1.0)[:, None]).reshape(-1)[:len(value)]
    size = np.abs(q)
    power = np.maximum(np.floor(np.log2(np.where(size > 0, size, 1e-30))), -6.0)
    unit = 2.0 ** (power - 3.0)
    at = size / unit + (bits.astype(np.float64) + 0.5) / 65536.0
    code = np.minimum(np.floor(at) * unit, 448.0)
    if root:
        code = np.where((q > 0) & (code == 0), 2.0 ** -9, code)
    return np.copysign(code, q), scale, np.abs(at - np.round(at)), unit
