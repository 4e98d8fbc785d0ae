"""The operators around a mixture-of-experts layer, as cases that can be timed and compared.

kind     "norm_in"       the norm before the block
         "norm_in_bwd"   its backward pass, with the gradient that comes through the residual connection added
         "norm_out"      the norm behind the block with its gate and residual scale, and the next block's norm with it
         "norm_out_bwd"  the backward pass of that
         "few"           a whole layer for a few tokens (serving): routing, experts, combine
         "adamw"         an AdamW step over all tensors of a model's layers, moments in 32 or 8 bits

With `own` the calls are those of `paper_1701_06538_b200.binding`; without it every operator is written in elementary torch
operations. Sizes are those of the workloads in `synth.CONFIGS`, of `perf/cases.py` and of the tests; x, y and upstream gradients are
standard normal, weights are scaled by their fan-in, norm weights and gates lie around 1.
"""
import math

import torch

own = False

EPS = 1e-6                                        # of the norms
BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.1
BLOCK = 128                                       # elements of an 8-bit moment that share a scale


def _norm(name, kind, T, d, act="bf16", rows_per_gate=0, next=True, scale=1.0):
    c = dict(kind=kind, T=T, d=d, act=act, rows_per_gate=rows_per_gate, next=next, scale=scale)
    return dict(c, name=name) if name else c


def _few(name, T, d, h, n, k, act="bf16"):
    c = dict(kind="few", T=T, d=d, h=h, n=n, k=k, act=act)
    return dict(c, name=name) if name else c


def _adamw(name, layers, d, h, n, act="bf16", grad="bf16", master=False, bits=32):
    c = dict(kind="adamw", layers=layers, d=d, h=h, n=n, act=act, grad=grad, master=master, bits=bits)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving one token: the norms between two blocks are latency and nothing else
        _norm("norm-out-one-token", "norm_out", 1, 512),
        # training the 256-expert layer: a gate and residual scale per channel, the next block's norm along with it
        _norm("norm-out-32768", "norm_out", 32768, 512, rows_per_gate=32768, scale=0.7),
        # the backward pass of that at the size of the wide layer: six tensors of 268 MB, three weight gradients
        _norm("norm-out-bwd-wide", "norm_out_bwd", 131072, 1024, rows_per_gate=131072),
        # float, odd sizes, a gate row for every 100 tokens (a sequence each), no norm behind it
        _norm("norm-out-bwd-odd-f32", "norm_out_bwd", 3001, 320, act="f32", rows_per_gate=100, next=False),
        # the first norm of a model, backward, at an ordinary batch
        _norm("norm-in-bwd-8192", "norm_in_bwd", 8192, 512),
        # decoding one sequence with the wide layer: two experts of 16 MB each
        _few("few-one-token-wide", 1, 1024, 4096, 128, 2),
        # serving two dozen sequences with 32 experts: nearly every expert is read for two or three rows
        _few("few-24-tokens", 24, 512, 1024, 32, 4),
        # the largest batch of this form over 256 experts
        _few("few-64-tokens-256", 64, 512, 1024, 256, 4),
        # a float layer of odd widths
        _few("few-odd-f32", 5, 72, 520, 20, 3, act="f32"),
        # the optimiser of a unit-test sized float model: latency
        _adamw("adamw-tiny-f32", 1, 64, 128, 8, act="f32", grad="f32"),
        # a 32-expert language-model layer: bf16 weights with float masters, float moments
        _adamw("adamw-32-experts", 1, 512, 1024, 32, master=True),
        # the 256-expert layer with moments in 8 bits
        _adamw("adamw-256-experts-8bit", 1, 512, 1024, 256, bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_in", "norm_in_bwd", "norm_out", "norm_out_bwd", "norm_out_bwd", "few", "few", "few", "few", "adamw", "adamw", "adamw"])
    act = "f32" if rng.random() < 0.25 else "bf16"
    unit = 8 if rng.random() < 0.4 else 64
    if kind.startswith("norm"):
        d = unit * max(1, _log_int(rng, 64, 8192) // unit)
        T = max(1, min(_log_int(rng, 1, 131072), 2 ** 26 // d))
        per = rng.choice([0, 1, T, _log_int(rng, 1, T)]) if kind.startswith("norm_out") else 0
        return _norm(None, kind, T, d, act, per, kind.startswith("norm_in") or rng.random() < 0.6, rng.choice([1.0, 1.0, 0.5, 0.7]))
    if kind == "few":
        d = unit * max(1, _log_int(rng, 64, 2048) // unit)
        h = unit * max(1, _log_int(rng, 64, 4096) // unit)
        T, n = _log_int(rng, 1, 64), _log_int(rng, 2, 512)
        k = min(n, rng.choice([1, 2, 2, 4, 4, 8]))
        while T * k * d * h > 2 ** 27 and T > 1:  # what the plain form gathers: a matrix for every row
            T //= 2
        while n * d * h > 2 ** 28:
            n = max(k, n // 2)
            if n == k:
                break
        return _few(None, T, d, h, n, k, act)
    d, h = unit * max(1, _log_int(rng, 64, 1024) // unit), unit * max(1, _log_int(rng, 64, 2048) // unit)
    layers, n = _log_int(rng, 1, 24), _log_int(rng, 1, 256)
    while layers * n * d * h > 2 ** 26 and layers * n > 1:
        layers, n = max(1, layers // 2), max(1, n // 2)
    return _adamw(None, layers, d, h, n, act, rng.choice(["f32", "bf16"]) if act == "bf16" else "f32", act == "bf16" and rng.random() < 0.5, rng.choice([8, 32]))


# ------------------------------------------------------------------------------------------------ inputs
def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.randn(*shape, generator=g, device="cuda", dtype=dtype)
        return t.mul_(std).add_(mean) if std != 1.0 or mean else t

    kind, s = case["kind"], dict(case=case)
    if kind == "adamw":
        return _prepare_adamw(case, s, g)
    adt = _type(case["act"])
    if kind == "few":
        T, d, h, n = (case[q] for q in ("T", "d", "h", "n"))
        s.update(x=normal(T, d).to(adt), Wg=normal(d, n, std=d ** -0.5), W1=normal(n, d, h, std=d ** -0.5, dtype=adt),
                 b1=normal(n, h, std=0.1, dtype=adt), W2=normal(n, h, d, std=h ** -0.5, dtype=adt), b2=normal(n, d, std=0.1, dtype=adt))
        return s
    T, d, per = case["T"], case["d"], case["rows_per_gate"]
    s["w"] = normal(d, std=0.1, mean=1.0)
    if kind in ("norm_in", "norm_in_bwd"):
        s["x"] = normal(T, d).to(adt)
        if kind == "norm_in_bwd":
            s["rstd"] = (s["x"].double().square().mean(1) + EPS).rsqrt().float()
            s.update(dxn=normal(T, d).to(adt), dres=normal(T, d).to(adt))
        return s
    s["y"] = normal(T, d, std=0.5).to(adt)
    s["gate"] = normal(-(-T // per), d, std=0.2, mean=1.0).to(adt) if per else None
    s["w_next"] = normal(d, std=0.1, mean=1.0) if case["next"] else None
    if kind == "norm_out":
        s["x"] = normal(T, d).to(adt)
        return s
    s["rstd"] = (s["y"].double().square().mean(1) + EPS).rsqrt().float()
    s["dOut"] = normal(T, d).to(adt)
    if case["next"]:  # what the forward pass has left
        s["out"] = normal(T, d, std=1.4).to(adt)
        s["rstd_next"] = (s["out"].double().square().mean(1) + EPS).rsqrt().float()
        s["dNext"] = normal(T, d).to(adt)
    else:
        s["out"] = s["rstd_next"] = s["dNext"] = None
    return s


def _tensors(case):
    """(elements, weight decay) of every parameter tensor: experts and gates decay, biases and norms do not."""
    d, h, n = case["d"], case["h"], case["n"]
    layer = [(n * d * h, DECAY), (n * h, 0.0), (n * h * d, DECAY), (n * d, 0.0), (d * n, DECAY), (d * n, DECAY), (d, 0.0), (d, 0.0)]
    return layer * case["layers"]


def _prepare_adamw(case, s, g):
    # all tensors stand one behind the other in flat buffers, each from a multiple of BLOCK elements on
    spans, at = [], 0
    for count, decay in _tensors(case):
        spans.append((at, count, decay))
        at += -(-count // BLOCK) * BLOCK
    live = torch.zeros(at, device="cuda", dtype=torch.bool)
    decay = torch.zeros(at, device="cuda")
    for first, count, wd in spans:
        live[first:first + count] = True
        decay[first:first + count] = wd

    def normal(std):
        return torch.randn(at, generator=g, device="cuda").mul_(std).mul_(live)

    s.update(spans=spans, total=at, decay=decay, step=100)
    master = normal(0.03)
    s["w"] = master.to(_type(case["act"])) if case["act"] == "bf16" else master
    s["master"] = master if case["master"] else None
    # gradients whose size differs from tensor to tensor and from element to element
    s["g"] = (normal(1e-3) * torch.exp(normal(1.0))).to(_type(case["grad"]))
    m, root = normal(4e-4), normal(1e-3).abs_()
    if case["bits"] == 32:
        s.update(m=m, v=root.square_(), m_scale=None, v_scale=None)
        return s
    for q, t in (("m", m), ("v", root)):
        t = t.view(-1, BLOCK)
        scale = t.abs().amax(1) / 448.0
        s[q] = (t / scale.clamp(min=1e-30).unsqueeze(1)).to(torch.float8_e4m3fn).view(-1)
        s[q + "_scale"] = scale
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _plain_norm(s):
    c = s["case"]
    kind, adt, T = c["kind"], _type(c["act"]), c["T"]
    w = s["w"]
    if kind == "norm_in":
        x = s["x"].float()
        r = (x.square().mean(1) + EPS).rsqrt()
        return dict(xn=(x * r[:, None] * w).to(adt), rstd=r)
    if kind == "norm_in_bwd":
        xh, dn = s["x"].float() * s["rstd"][:, None], s["dxn"].float() * w
        dX = s["dres"].float() + s["rstd"][:, None] * (dn - xh * (dn * xh).mean(1, keepdim=True))
        return dict(dX=dX.to(adt), dw=(s["dxn"].float() * xh).sum(0, dtype=torch.float64).float())
    per = c["rows_per_gate"]
    gate = None
    if per:
        gate = s["gate"].float()
        gate = gate if gate.shape[0] == 1 else gate[torch.arange(T, device="cuda") // per]
    y = s["y"].float()
    if kind == "norm_out":
        r = (y.square().mean(1) + EPS).rsqrt()
        u = y * r[:, None] * w
        out = c["scale"] * s["x"].float() + (u if gate is None else gate * u)
        res = dict(out=out.to(adt), rstd=r)
        if c["next"]:
            r2 = (out.square().mean(1) + EPS).rsqrt()
            res.update(next=(out * r2[:, None] * s["w_next"]).to(adt), rstd_next=r2)
        return res
    dt = s["dOut"].float()
    res = {}
    if c["next"]:
        n2, dnext = s["out"].float() * s["rstd_next"][:, None], s["dNext"].float()
        dn2 = dnext * s["w_next"]
        res["dw_next"] = (dnext * n2).sum(0, dtype=torch.float64).float()
        dt = dt + s["rstd_next"][:, None] * (dn2 - n2 * (dn2 * n2).mean(1, keepdim=True))
    n1 = y * s["rstd"][:, None]
    a = dt * n1
    if per:
        groups = -(-T // per)
        rows = torch.zeros(groups * per, a.shape[1], device="cuda")
        rows[:T] = a
        dgate = rows.view(groups, per, -1).sum(1, dtype=torch.float64) * w
        res["dgate"] = dgate.float().to(adt)
        a, dn = a * gate, dt * gate * w
    else:
        dn = dt * w
    res["dw"] = a.sum(0, dtype=torch.float64).float()
    res["dY"] = (s["rstd"][:, None] * (dn - n1 * (dn * n1).mean(1, keepdim=True))).to(adt)
    res["dX"] = (c["scale"] * dt).to(adt)
    return res


def _plain_few(s):
    c = s["case"]
    T, k = c["T"], c["k"]
    logits = s["x"].double() @ s["Wg"].double()  # in 64 bits: a routing decision is a comparison
    top, idx = logits.topk(k, dim=1)
    e = torch.exp(top - top[:, :1])
    gates = (e / e.sum(1, keepdim=True)).float()
    rows, x = idx.reshape(-1), s["x"].float().repeat_interleave(k, 0).unsqueeze(1)
    hid = torch.clamp(torch.bmm(x, s["W1"][rows].float()).squeeze(1) + s["b1"][rows].float(), min=0.0)
    ys = torch.bmm(hid.unsqueeze(1), s["W2"][rows].float()).squeeze(1) + s["b2"][rows].float()
    y = (gates.unsqueeze(2) * ys.view(T, k, -1)).sum(1)
    return dict(y=y.to(_type(c["act"])), gates=gates)


def _mix(x):
    """A hash of 32 bits, in 64-bit integers."""
    x = (x ^ (x >> 16)) * 0x7feb352d & 0xffffffff
    x = (x ^ (x >> 15)) * 0x846ca68b & 0xffffffff
    return x ^ (x >> 16)


def _to_eight_bits(t, dither, keep_positive):
    """e4m3 codes and scales of blocks of BLOCK: rounded up or down by the dither, 20 bits below the code's last."""
    t = t.view(-1, BLOCK)
    largest = t.abs().amax(1)
    scale = torch.where(largest > 0, (largest * torch.tensor(1.0 / 448.0, device="cuda")).clamp(min=1.17549435e-38), torch.zeros_like(largest))
    q = (t / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(1)).view(-1)
    size = q.abs()
    small = size < 2.0 ** -6
    up = torch.where(small, size + 2.0 ** -6, size)
    z = ((up.view(torch.int32) + dither) & ~0xfffff).view(torch.float32)
    z = torch.where(small, z - 2.0 ** -6, z).clamp(max=448.0)
    if keep_positive:
        z = torch.where((size > 0) & (z == 0), torch.full_like(z, 2.0 ** -9), z)
    return torch.copysign(z, q).to(torch.float8_e4m3fn), scale


def _plain_adamw(s):
    c = s["case"]
    s["step"] += 1
    g = s["g"].float()
    eight = c["bits"] == 8
    old = [s["m"], s["v"]]
    if eight:
        old = [(s[q].float().view(-1, BLOCK) * s[q + "_scale"].unsqueeze(1)).view(-1) for q in ("m", "v")]
    m = BETA1 * old[0] + (1.0 - BETA1) * g
    v = BETA2 * (old[1].square() if eight else old[1]) + (1.0 - BETA2) * g.square()
    root = v.sqrt()
    w = (s["master"] if c["master"] else s["w"]).float()
    step_m, step_v = 1.0 - BETA1 ** s["step"], 1.0 - BETA2 ** s["step"]
    w = w - LR * ((m / step_m) / (root / math.sqrt(step_v) + ADAM_EPS) + s["decay"] * w)
    s["w"].copy_(w)
    if c["master"]:
        s["master"].copy_(w)
    if eight:
        key = _mix(torch.tensor(s["step"], device="cuda", dtype=torch.int64))
        bits = _mix(torch.arange(s["total"], device="cuda", dtype=torch.int64) ^ key)
        for q, t, part in (("m", m, bits & 0xffff), ("v", root, bits >> 16)):
            code, scale = _to_eight_bits(t, (part * 16 + 8).to(torch.int32), q == "v")
            s[q].copy_(code)
            s[q + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {q: s[q] for q in ("w", "master", "m", "v", "m_scale", "v_scale") if s[q] is not None}


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handle(s):
    """What a program makes once for a size: configuration, output buffers, workspace; for the optimiser the list of its tensors."""
    from paper_1701_06538_b200 import binding as B

    c = s["case"]
    kind, adt = c["kind"], _type(c["act"])
    o = s["handle"] = dict(B=B)
    if kind == "adamw":
        t = []
        for first, count, decay in s["spans"]:
            a, b = first, first + count
            blocks = slice(a // BLOCK, -(-b // BLOCK))
            t.append(dict(w=s["w"][a:b], g=s["g"][a:b], master=None if s["master"] is None else s["master"][a:b], m=s["m"][a:b], v=s["v"][a:b],
                          m_scale=None if s["m_scale"] is None else s["m_scale"][blocks], v_scale=None if s["v_scale"] is None else s["v_scale"][blocks],
                          weight_decay=decay, first=first))
        o["list"] = B.moe_adamw_list(t)
        return o
    T, d = c["T"], c["d"]

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    if kind == "few":
        o["cfg"] = B.make_config(T, d, c["h"], c["n"], c["k"], c["act"])
        o.update(y=empty(T, d, dtype=adt), gates=empty(T, c["k"]), ws=B.empty_bytes(B.moe_few_workspace_bytes(o["cfg"])))
        return o
    o["cfg"] = B.make_config(T, d, d, 1, 1, c["act"])
    if kind == "norm_in":
        o.update(xn=empty(T, d, dtype=adt), rstd=empty(T))
    elif kind == "norm_out":
        o.update(out=empty(T, d, dtype=adt), rstd=empty(T), next=empty(T, d, dtype=adt) if c["next"] else None, rstd_next=empty(T) if c["next"] else None)
    else:
        o.update(dX=empty(T, d, dtype=adt), dw=empty(d), ws=B.empty_bytes(B.moe_norm_workspace_bytes(o["cfg"])))
        if kind == "norm_out_bwd":
            o.update(dY=empty(T, d, dtype=adt), dgate=None if s["gate"] is None else torch.empty_like(s["gate"]), dw_next=empty(d) if c["next"] else None)
    return o


def _own(s):
    c = s["case"]
    o = s.get("handle") or _handle(s)
    B, kind = o["B"], c["kind"]
    if kind == "adamw":
        s["step"] += 1
        B.moe_adamw(o["list"], LR, BETA1, BETA2, ADAM_EPS, s["step"], s["step"])
        return _adamw_outputs(s)
    if kind == "few":
        B.moe_forward_few(o["cfg"], s["x"], s["Wg"], s["W1"], s["b1"], s["W2"], s["b2"], o["y"], None, o["gates"], o["ws"])
        return dict(y=o["y"], gates=o["gates"])
    if kind == "norm_in":
        B.moe_norm_in(o["cfg"], s["x"], s["w"], EPS, o["xn"], o["rstd"])
        return dict(xn=o["xn"], rstd=o["rstd"])
    if kind == "norm_in_bwd":
        B.moe_norm_in_bwd(o["cfg"], s["dxn"], s["x"], s["w"], s["rstd"], s["dres"], o["dX"], o["dw"], o["ws"])
        return dict(dX=o["dX"], dw=o["dw"])
    if kind == "norm_out":
        B.moe_norm_out(o["cfg"], s["x"], s["y"], s["w"], s["gate"], c["rows_per_gate"], c["scale"], s["w_next"], EPS, o["out"], o["next"], o["rstd"],
                       o["rstd_next"])
        return {q: o[q] for q in ("out", "rstd", "next", "rstd_next") if o[q] is not None}
    B.moe_norm_out_bwd(o["cfg"], s["dOut"], s["dNext"], s["out"], s["y"], s["w"], s["gate"], c["rows_per_gate"], c["scale"], s["w_next"], s["rstd"],
                       s["rstd_next"], o["dX"], o["dY"], o["dw"], o["dgate"], o["dw_next"], o["ws"])
    return {q: o[q] for q in ("dX", "dY", "dw", "dgate", "dw_next") if o[q] is not None}


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    return _plain_adamw(s) if kind == "adamw" else _plain_few(s) if kind == "few" else _plain_norm(s)


# ------------------------------------------------------------------------------------------------ work and exact values
def work(case):
    kind, a = case["kind"], 2 if case["act"] == "bf16" else 4
    if kind == "adamw":
        count = sum(t[0] for t in _tensors(case))
        moments = 16 if case["bits"] == 32 else 4 + 16.0 / BLOCK
        weights = 8 + a if case["master"] else 2 * a
        return {"bytes": count * (weights + (2 if case["grad"] == "bf16" else 4) + moments), "flops": 15.0 * count}
    T, d = case["T"], case["d"]
    if kind == "few":
        h, n, k = case["h"], case["n"], case["k"]
        used = n * (1.0 - (1.0 - k / n) ** T)  # experts that some token picks, expected
        return {"bytes": 2.0 * T * d * a + 4.0 * d * n + used * (2 * d * h + d + h) * a, "flops": 4.0 * T * k * d * h + 2.0 * T * d * n}
    nxt = bool(case["next"])
    per = case["rows_per_gate"]
    gates = -(-T // per) * d * a if per else 0
    tensors = {"norm_in": 2, "norm_in_bwd": 4, "norm_out": 3 + nxt, "norm_out_bwd": 4 + 2 * nxt}[kind]
    byts = tensors * T * d * a + T * 4 * (2 if kind.startswith("norm_out") and nxt else 1) + gates * (2 if kind == "norm_out_bwd" else 1)
    byts += d * 4 * (2 if kind.endswith("bwd") else 1) * (2 if kind.startswith("norm_out") and nxt else 1)
    return {"bytes": float(byts), "flops": {"norm_in": 5.0, "norm_in_bwd": 10.0, "norm_out": 12.0, "norm_out_bwd": 25.0}[kind] * T * d}


def _exact_norm(case, s):
    f64 = torch.float64
    T, d, per, kind = case["T"], case["d"], case["rows_per_gate"], case["kind"]
    w = s["w"].to(f64)

    def normed(t):
        return t / torch.sqrt((t * t).sum(1, keepdim=True) / d + EPS)

    def through(grad, t, r):
        """The gradient that reaches t from grad at t * r, r being the function of t that the norm is."""
        r = r.to(f64).view(T, 1)
        return r * grad - r ** 3 * t * ((grad * t).sum(1, keepdim=True) / d)

    if kind == "norm_in":
        x = s["x"].to(f64)
        return dict(xn=normed(x) * w, rstd=((x * x).sum(1) / d + EPS) ** -0.5)
    if kind == "norm_in_bwd":
        x, dxn, r = s["x"].to(f64), s["dxn"].to(f64), s["rstd"].to(f64).view(T, 1)
        return dict(dX=s["dres"].to(f64) + through(dxn * w, x, s["rstd"]), dw=(dxn * x * r).sum(0))
    y = s["y"].to(f64)
    which = torch.div(torch.arange(T, device="cuda"), per, rounding_mode="floor") if per else None
    gate = s["gate"].to(f64).index_select(0, which) if per else torch.ones(1, 1, device="cuda", dtype=f64)
    if kind == "norm_out":
        out = s["x"].to(f64) * case["scale"] + normed(y) * w * gate
        res = dict(out=out, rstd=((y * y).sum(1) / d + EPS) ** -0.5)
        if case["next"]:
            res.update(next=normed(out) * s["w_next"].to(f64), rstd_next=((out * out).sum(1) / d + EPS) ** -0.5)
        return res
    grad, res = s["dOut"].to(f64), {}
    if case["next"]:
        out, dnext = s["out"].to(f64), s["dNext"].to(f64)
        res["dw_next"] = (dnext * out * s["rstd_next"].to(f64).view(T, 1)).sum(0)
        grad = grad + through(dnext * s["w_next"].to(f64), out, s["rstd_next"])
    hat = y * s["rstd"].to(f64).view(T, 1)
    if per:
        res["dgate"] = torch.zeros(s["gate"].shape, device="cuda", dtype=f64).index_add_(0, which, grad * hat * w)
    res.update(dw=(grad * hat * gate).sum(0), dY=through(grad * gate * w, y, s["rstd"]), dX=grad * case["scale"])
    return res


def _exact_few(case, s):
    f64 = torch.float64
    T, k = case["T"], case["k"]
    x = s["x"].to(f64)
    logits = torch.mm(x, s["Wg"].to(f64))
    order = logits.argsort(dim=1, descending=True, stable=True)[:, :k]
    p = torch.softmax(logits.gather(1, order), dim=1)
    y = torch.zeros(T, case["d"], device="cuda", dtype=f64)
    for e in torch.unique(order).tolist():
        t, slot = (order == e).nonzero(as_tuple=True)
        hid = torch.relu(torch.addmm(s["b1"][e].to(f64), x[t], s["W1"][e].to(f64)))
        y.index_add_(0, t, p[t, slot].view(-1, 1) * torch.addmm(s["b2"][e].to(f64), hid, s["W2"][e].to(f64)))
    return dict(y=y, gates=p)


def _exact_adamw(case, s):
    f64 = torch.float64
    if s["total"] > 3e8:
        return None
    eight, t = case["bits"] == 8, s["step"] + 1
    g = s["g"].to(f64)

    def held(q):
        if not eight:
            return s[q].to(f64)
        return (s[q].to(f64).view(-1, BLOCK) * s[q + "_scale"].to(f64).view(-1, 1)).view(-1)

    m = held("m") * BETA1 + g * (1.0 - BETA1)
    v = (held("v") ** 2 if eight else held("v")) * BETA2 + g * g * (1.0 - BETA2)
    del g
    w = (s["master"] if case["master"] else s["w"]).to(f64)
    w = w * (1.0 - LR * s["decay"].to(f64)) - LR * (m / (1.0 - BETA1 ** t)) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + ADAM_EPS)
    res = dict(w=w)
    if case["master"]:
        res["master"] = w
    if not eight:
        return dict(res, m=m, v=v)

    def word(a, shift, factor):
        return torch.bitwise_and(torch.bitwise_xor(a, torch.bitwise_right_shift(a, shift)) * factor, 2 ** 32 - 1)

    def scrambled(a):
        a = word(word(a, 16, 0x7feb352d), 15, 0x846ca68b)
        return torch.bitwise_xor(a, torch.bitwise_right_shift(a, 16))

    number = torch.bitwise_xor(torch.arange(s["total"], device="cuda"), scrambled(torch.tensor([t], device="cuda")))
    number = scrambled(number)
    for q, value, u in (("m", m, number % 65536), ("v", v.sqrt(), number // 65536)):
        value = value.view(-1, BLOCK)
        scale = value.abs().max(dim=1).values / 448.0
        ratio = (value / torch.where(scale > 0, scale, torch.ones_like(scale)).view(-1, 1)).view(-1)
        power = torch.frexp(ratio.abs())[1].to(f64) - 1.0  # of two, at most the ratio
        step = torch.exp2(power.clamp(min=-6.0) - 3.0)
        code = torch.floor(ratio.abs() / step + (u.to(f64) + 0.5) / 65536.0) * step
        code = code.clamp(max=448.0)
        if q == "v":
            code = torch.where((ratio > 0) & (code == 0), torch.full_like(code, 2.0 ** -9), code)
        res[q], res[q + "_scale"] = code * torch.sign(ratio), scale
    return res


def exact(case, seed):
    """The results of `run` on these inputs from the definitions in 64 bits. Experts are taken one after the other."""
    s = prepare(case, seed)
    kind = case["kind"]
    return _exact_adamw(case, s) if kind == "adamw" else _exact_few(case, s) if kind == "few" else _exact_norm(case, s)
