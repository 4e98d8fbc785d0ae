"""Operators of training a mixture-of-experts model, as cases that can be timed and compared.

kind     "muon"            an optimiser step over the matrices of a model's layers: momentum, the update orthogonalised by Newton-Schulz products
         "router"          the router's losses: counts of every expert, balance loss and z loss, with the gradient of the logits
         "layer_norm"      layer norm before the block
         "layer_norm_bwd"  its backward pass, with the gradient that comes through the residual connection added

With `own` the calls are those of `paper_1701_06538_b200.binding`; without it every operator is written in elementary torch
operations. Sizes are those of the workloads in `synth.CONFIGS`, of `perf/operators.py` and of the tests; weights are scaled by their fan-in,
gradients of weights are products of rows and their gradients, as many rows as an expert gets.
"""
import math

import torch

own = False

NORM_EPS = 1e-5
LR, MOMENTUM, DECAY, MUON_EPS, STEPS = 1e-3, 0.95, 0.1, 1e-7, 5
NS_A, NS_B, NS_C = 3.4445, -4.775, 2.0315         # of X <- a X + b (X X') X + c (X X')^2 X
W_BALANCE, W_Z = 0.01, 0.001


def _muon(name, layers, d, h, n, rows, act="bf16", grad="bf16", master=False, moment="f32"):
    c = dict(kind="muon", layers=layers, d=d, h=h, n=n, rows=rows, act=act, grad=grad, master=master, moment=moment)
    return dict(c, name=name) if name else c


def _router(name, T, n, k, sequences=0, keep=False, grad=True):
    c = dict(kind="router", T=T, n=n, k=k, sequences=sequences, keep=keep, grad=grad)
    return dict(c, name=name) if name else c


def _norm(name, kind, T, d, act="bf16", bias=True, res=True):
    c = dict(kind=kind, T=T, d=d, act=act, bias=bias, res=res)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a unit-test sized float model: eight experts of 64 x 128 and their gate, latency
        _muon("muon-tiny-f32", 1, 64, 128, 8, 64, act="f32", grad="f32"),
        # odd widths, a float layer of twenty experts with few rows each
        _muon("muon-odd-f32", 2, 72, 520, 20, 24, act="f32", grad="f32"),
        # a 32-expert language-model layer with its gate: bf16 weights with float masters
        _muon("muon-32-experts", 1, 512, 1024, 32, 1024, master=True),
        # the 256-expert layer: 512 matrices with momentum in bf16
        _muon("muon-256-experts", 1, 512, 1024, 256, 512, moment="bf16"),
        # a quarter of the wide layer's experts
        _muon("muon-wide", 1, 1024, 4096, 32, 512),
        # two dozen tokens on 32 experts: latency
        _router("router-24-tokens", 24, 32, 4),
        # a batch of ragged sequences, padded: losses of every sequence over 256 experts
        _router("router-sequences", 32768, 256, 4, sequences=61, keep=True),
        # the wide layer's batch
        _router("router-131072", 131072, 128, 2),
        # serving one token: latency
        _norm("layer-norm-one-token", "layer_norm", 1, 512),
        # the wide layer's batch, forward
        _norm("layer-norm-131072", "layer_norm", 131072, 1024),
        # training the 256-expert layer
        _norm("layer-norm-bwd-32768", "layer_norm_bwd", 32768, 512),
        # float, odd sizes, nothing beside the norm
        _norm("layer-norm-bwd-odd-f32", "layer_norm_bwd", 3001, 320, act="f32", res=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["muon", "muon", "muon", "muon", "router", "router", "router", "layer_norm", "layer_norm_bwd", "layer_norm_bwd"])
    act = "f32" if rng.random() < 0.25 else "bf16"
    unit = 8 if rng.random() < 0.4 else 64
    if kind == "router":
        n = _log_int(rng, 2, 2048)
        k = min(n, rng.choice([1, 2, 2, 4, 4, 8]))
        T = max(1, min(_log_int(rng, 1, 131072), 2 ** 24 // n))
        sequences = rng.choice([0, 0, 1, _log_int(rng, 1, min(T, 512))])
        return _router(None, T, n, k, sequences, rng.random() < 0.4, rng.random() < 0.8)
    if kind != "muon":
        d = unit * max(1, _log_int(rng, 64, 8192) // unit)
        T = max(1, min(_log_int(rng, 1, 131072), 2 ** 26 // d))
        return _norm(None, kind, T, d, act, rng.random() < 0.7, rng.random() < 0.6)
    d, h = unit * max(1, _log_int(rng, 64, 1024) // unit), unit * max(1, _log_int(rng, 64, 4096) // unit)
    layers, n = _log_int(rng, 1, 12), _log_int(rng, 2, 256)
    c = _muon(None, layers, d, h, n, _log_int(rng, 16, 1024), act, rng.choice(["f32", "bf16"]) if act == "bf16" else "f32", act == "bf16" and rng.random() < 0.5,
              rng.choice(["f32", "bf16"]))
    while c["n"] > 2 and (c["layers"] * c["n"] * d * h > 2 ** 26 or work(c)["flops"] > 2e12):
        c["layers"], c["n"] = max(1, c["layers"] // 2), max(2, c["n"] // 2)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _matrices(case):
    """(name, matrices of a layer, rows, columns, whether they are of the gate, which is float)."""
    d, h, n = case["d"], case["h"], case["n"]
    return [("W1", n, d, h, False), ("W2", n, h, d, False), ("Wg", 1, d, n, True)]


def _scale(rows, cols):
    """Of an orthogonalised update, so that its elements are as large as those of an Adam step."""
    return 0.2 * math.sqrt(max(rows, cols))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.randn(*shape, generator=g, device="cuda", dtype=dtype)
        return t.mul_(std).add_(mean) if std != 1.0 or mean else t

    kind, s = case["kind"], dict(case=case)
    if kind == "muon":
        for name, per_layer, rows, cols, gate in _matrices(case):
            count = per_layer * case["layers"]
            act = torch.float32 if gate else _type(case["act"])
            master = normal(count, rows, cols, std=rows ** -0.5)
            r = case["rows"]  # of the batch that an expert gets: the gradient's rank
            grad = torch.bmm(normal(count, rows, r, std=r ** -0.5, dtype=torch.bfloat16), normal(count, r, cols, std=1e-3, dtype=torch.bfloat16))
            s[name] = dict(w=master.to(act), master=master if case["master"] and not gate else None, g=grad.to(torch.float32 if gate else _type(case["grad"])),
                           m=normal(count, rows, cols, std=3e-3).to(_type(case["moment"])))
        return s
    T = case["T"]
    if kind == "router":
        n, k = case["n"], case["k"]
        # experts that are liked more and less, as they are while a router learns
        s["logits"] = normal(T, n) + normal(n, std=0.5)
        s["topk_idx"] = (s["logits"] + 0.3 * normal(T, n)).topk(k, dim=1).indices.to(torch.int32)
        s["keep"] = (torch.rand(T, generator=g, device="cuda") < 0.9).to(torch.uint8) if case["keep"] else None
        s["offsets"] = None
        if case["sequences"]:  # of any lengths, some tokens behind the last one
            ends = (torch.rand(case["sequences"], generator=g, device="cuda") * T).to(torch.int32).sort().values
            s["offsets"] = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int32), ends]).contiguous()
            s["offsets"][-1] = max(1, T - T // 50)
        return s
    d, adt = case["d"], _type(case["act"])
    s["x"] = normal(T, d, mean=0.3).to(adt)
    s["w"] = normal(d, std=0.1, mean=1.0)
    s["b"] = normal(d, std=0.1) if case["bias"] else None
    if kind == "layer_norm_bwd":
        x = s["x"].double()
        s["mean"] = x.mean(1).float()
        s["rstd"] = ((x - x.mean(1, keepdim=True)).square().mean(1) + NORM_EPS).rsqrt().float()
        s["dxn"] = normal(T, d).to(adt)
        s["dres"] = normal(T, d).to(adt) if case["res"] else None
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _plain_muon(s):
    c, out = s["case"], {}
    for name, _, rows, cols, _ in _matrices(c):
        t = s[name]
        g = t["g"].float()
        t["m"].copy_(MOMENTUM * t["m"].float() + g)
        u = g + MOMENTUM * t["m"].float()
        norm = u.square().sum((1, 2), dtype=torch.float64).sqrt().float()
        x = u / (norm + MUON_EPS).view(-1, 1, 1)
        x = x.transpose(1, 2) if rows > cols else x
        for _ in range(STEPS):
            a = torch.bmm(x, x.transpose(1, 2))
            x = NS_A * x + torch.bmm(NS_B * a + NS_C * torch.bmm(a, a), x)
        x = x.transpose(1, 2) if rows > cols else x
        w = t["w"].float() if t["master"] is None else t["master"]
        w = w - LR * (_scale(rows, cols) * x + DECAY * w)
        t["w"].copy_(w)
        if t["master"] is not None:
            t["master"].copy_(w)
        out.update(_muon_outputs(name, t))
    return out


def _muon_outputs(name, t):
    return {name + "." + q: t[q] for q in ("w", "master", "m") if t[q] is not None}


def _plain_router(s):
    c = s["case"]
    T, n, k = c["T"], c["n"], c["k"]
    x, f64 = s["logits"], torch.float64
    token = torch.arange(T, device="cuda", dtype=torch.int32)
    live = torch.ones(T, device="cuda", dtype=torch.bool) if s["keep"] is None else s["keep"] != 0
    if s["offsets"] is None:
        S, seq = 1, torch.zeros(T, device="cuda", dtype=torch.int64)
    else:
        S = c["sequences"]
        seq = (torch.searchsorted(s["offsets"], token, right=True) - 1).clamp(0, S - 1)
        live = live & (token >= s["offsets"][0]) & (token < s["offsets"][-1])
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    p = e / total * live[:, None]
    tokens = torch.zeros(S, device="cuda", dtype=f64).index_add_(0, seq, live.to(f64))
    places = (seq[:, None] * n + s["topk_idx"]).reshape(-1)
    counts = torch.zeros(S * n, device="cuda", dtype=f64).index_add_(0, places, live.to(f64).repeat_interleave(k)).view(S, n)
    prob_sums = torch.zeros(S, n, device="cuda", dtype=f64).index_add_(0, seq, p.to(f64))
    by = W_BALANCE * n / (k * tokens.sum() * tokens.clamp(min=1.0))
    losses = torch.stack([((counts * prob_sums).sum(1) * by).sum(), W_Z * (lse.to(f64) * live).square().sum() / tokens.sum()])
    res = dict(losses=losses.float(), counts=counts.to(torch.int32), prob_sums=prob_sums.float())
    if c["grad"]:
        pull = (counts * by[:, None]).float()[seq]
        z = (2.0 * W_Z / tokens.sum()).float() * lse * live
        res["dlogits"] = p * (pull - (pull * p).sum(1, keepdim=True) + z[:, None])
    return res


def _plain_norm(s):
    c = s["case"]
    adt, x = _type(c["act"]), s["x"].float()
    if c["kind"] == "layer_norm":
        mean = x.mean(1)
        off = x - mean[:, None]
        rstd = (off.square().mean(1) + NORM_EPS).rsqrt()
        y = off * rstd[:, None] * s["w"]
        return dict(xn=(y if s["b"] is None else y + s["b"]).to(adt), mean=mean, rstd=rstd)
    hat, dxn = (x - s["mean"][:, None]) * s["rstd"][:, None], s["dxn"].float()
    dn = dxn * s["w"]
    dX = s["rstd"][:, None] * (dn - dn.mean(1, keepdim=True) - hat * (dn * hat).mean(1, keepdim=True))
    res = dict(dX=(dX if s["dres"] is None else dX + s["dres"].float()).to(adt), dw=(dxn * hat).sum(0, dtype=torch.float64).float())
    if s["b"] is not None:
        res["db"] = dxn.sum(0, dtype=torch.float64).float()
    return res


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handle(s):
    """What a program makes once for a size: configuration, output buffers, workspace; for the optimiser the list of its tensors."""
    from paper_1701_06538_b200 import binding as B

    c = s["case"]
    kind = c["kind"]
    o = s["handle"] = dict(B=B)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    if kind == "muon":
        tensors = []
        for layer in range(c["layers"]):
            for name, per_layer, rows, cols, _ in _matrices(c):
                part, t = slice(layer * per_layer, (layer + 1) * per_layer), s[name]
                tensors.append(dict(w=t["w"][part], g=t["g"][part], m=t["m"][part], master=None if t["master"] is None else t["master"][part], weight_decay=DECAY,
                                    scale=_scale(rows, cols)))
        o["list"] = B.moe_muon_list(tensors)
        o["ws"] = B.empty_bytes(B.moe_muon_workspace_bytes(o["list"]))
        o["outputs"] = {q: t for name, *_ in _matrices(c) for q, t in _muon_outputs(name, s[name]).items()}
        return o
    T = c["T"]
    if kind == "router":
        S = max(1, c["sequences"])
        o["cfg"] = B.make_config(T, 64, 64, c["n"], c["k"], "bf16")
        o.update(losses=empty(2), counts=empty(S, c["n"], dtype=torch.int32), prob_sums=empty(S, c["n"]), dlogits=empty(T, c["n"]) if c["grad"] else None,
                 ws=B.empty_bytes(B.moe_router_losses_workspace_bytes(o["cfg"], S)))
        return o
    d, adt = c["d"], _type(c["act"])
    o["cfg"] = B.make_config(T, d, d, 1, 1, c["act"])
    if kind == "layer_norm":
        o.update(xn=empty(T, d, dtype=adt), mean=empty(T), rstd=empty(T))
    else:
        o.update(dX=empty(T, d, dtype=adt), dw=empty(d), db=empty(d) if c["bias"] else None, ws=B.empty_bytes(B.moe_layer_norm_workspace_bytes(o["cfg"])))
    return o


def _own(s):
    c = s["case"]
    o = s.get("handle") or _handle(s)
    B, kind = o["B"], c["kind"]
    if kind == "muon":
        B.moe_muon(o["list"], LR, MOMENTUM, MUON_EPS, STEPS, True, o["ws"])
        return o["outputs"]
    if kind == "router":
        B.moe_router_losses(o["cfg"], s["logits"], s["topk_idx"], s["keep"], s["offsets"], max(1, c["sequences"]), W_BALANCE, W_Z, o["losses"], o["counts"], o["prob_sums"],
                            o["dlogits"], o["ws"])
        return {q: o[q] for q in ("losses", "counts", "prob_sums", "dlogits") if o[q] is not None}
    if kind == "layer_norm":
        B.moe_layer_norm(o["cfg"], s["x"], s["w"], s["b"], NORM_EPS, o["xn"], o["mean"], o["rstd"])
        return dict(xn=o["xn"], mean=o["mean"], rstd=o["rstd"])
    B.moe_layer_norm_bwd(o["cfg"], s["dxn"], s["x"], s["w"], s["mean"], s["rstd"], s["dres"], o["dX"], o["dw"], o["db"], o["ws"])
    return {q: o[q] for q in ("dX", "dw", "db") if o[q] is not None}


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    return _plain_muon(s) if kind == "muon" else _plain_router(s) if kind == "router" else _plain_norm(s)


# ------------------------------------------------------------------------------------------------ work and exact values
def work(case):
    kind = case["kind"]
    if kind == "muon":
        size = {"f32": 4, "bf16": 2}
        byts = flops = 0.0
        for _, per_layer, rows, cols, gate in _matrices(case):
            count, lo, hi = per_layer * case["layers"], min(rows, cols), max(rows, cols)
            weight = 8 if gate else (8 + size[case["act"]] if case["master"] else 2 * size[case["act"]])
            byts += count * rows * cols * (weight + (4 if gate else size[case["grad"]]) + 2 * size[case["moment"]])
            # of the two symmetric products one half
            flops += count * (STEPS * (lo * (lo + 1.0) * hi + lo * lo * (lo + 1.0) + 2.0 * lo * lo * hi) + 12.0 * rows * cols)
        return {"bytes": byts, "flops": flops}
    T = case["T"]
    if kind == "router":
        n, S = case["n"], max(1, case["sequences"])
        byts = 4.0 * T * n * (2 if case["grad"] else 1) + 4.0 * T * case["k"] + 8.0 * S * n + (T if case["keep"] else 0) + 4.0 * S
        return {"bytes": byts, "flops": T * n * (10.0 if case["grad"] else 6.0)}
    d, a = case["d"], 2 if case["act"] == "bf16" else 4
    forward = kind == "layer_norm"
    tensors = 2 if forward else 3 + case["res"]
    return {"bytes": float(tensors * T * d * a + 8 * T + 4 * d * (1 + case["bias"] + (0 if forward else 1))), "flops": (7.0 if forward else 13.0) * T * d}


def _exact_muon(case, s):
    f64, res = torch.float64, {}
    for name, per_layer, rows, cols, _ in _matrices(case):
        t = s[name]
        if t["w"].numel() > 1.5e8:
            return None
        g = t["g"].to(f64)
        m = torch.add(g, t["m"].to(f64), alpha=MOMENTUM)
        u = torch.add(g, m.to(t["m"].dtype).to(f64), alpha=MOMENTUM)  # of the momentum as it is held
        u /= (u.flatten(1).norm(dim=1) + MUON_EPS).view(-1, 1, 1)
        wide = rows <= cols
        # the polynomials of the smaller Gram matrix alone, all of them in one product with the update
        gram = torch.bmm(u, u.mT) if wide else torch.bmm(u.mT, u)
        eye = torch.eye(gram.shape[1], device="cuda", dtype=f64)
        all_of = eye.expand_as(gram)
        for _ in range(STEPS):
            q = torch.bmm(gram, gram).mul_(NS_C).add_(gram, alpha=NS_B).add_(eye, alpha=NS_A)
            all_of = torch.bmm(q, all_of)
            gram = torch.bmm(torch.bmm(q, gram), q)
        o = torch.bmm(all_of, u) if wide else torch.bmm(u, all_of)
        w = (t["w"] if t["master"] is None else t["master"]).to(f64)
        w = w * (1.0 - LR * DECAY) - (LR * _scale(rows, cols)) * o
        res[name + ".w"], res[name + ".m"] = w, m
        if t["master"] is not None:
            res[name + ".master"] = w
    return res


def _exact_router(case, s):
    f64 = torch.float64
    T, n, k = case["T"], case["n"], case["k"]
    S = max(1, case["sequences"])
    ends = [0, T] if s["offsets"] is None else s["offsets"].tolist()
    keep = torch.ones(T, device="cuda", dtype=f64) if s["keep"] is None else (s["keep"] != 0).to(f64)
    live = torch.zeros(T, device="cuda", dtype=f64)
    live[ends[0]:ends[-1]] = keep[ends[0]:ends[-1]]
    L = float(live.sum())
    logp = torch.log_softmax(s["logits"].to(f64), dim=1)
    lse = s["logits"][:, 0].to(f64) - logp[:, 0]
    p = logp.exp()
    chosen = torch.nn.functional.one_hot(s["topk_idx"].long(), n).sum(1).to(f64) if T * n * k < 2 ** 27 else None
    if chosen is None:
        chosen = torch.zeros(T, n, device="cuda", dtype=f64).scatter_add_(1, s["topk_idx"].long(), torch.ones(T, k, device="cuda", dtype=f64))
    counts, sums = torch.zeros(S, n, device="cuda", dtype=f64), torch.zeros(S, n, device="cuda", dtype=f64)
    grad = torch.zeros(T, n, device="cuda", dtype=f64)
    balance = torch.zeros((), device="cuda", dtype=f64)
    for i in range(S):
        a, b = ends[i], ends[i + 1]
        if b <= a:
            continue
        here = live[a:b, None]
        number = here.sum().clamp(min=1.0)
        counts[i], sums[i] = (chosen[a:b] * here).sum(0), (p[a:b] * here).sum(0)
        share, mean = counts[i] / (k * number), sums[i] / number  # of the choices, of the probabilities
        balance += (number / L) * n * torch.dot(share, mean)
        pull = (n / L) * share
        grad[a:b] = W_BALANCE * p[a:b] * here * (pull - (p[a:b] @ pull)[:, None])
    res = dict(losses=torch.stack([W_BALANCE * balance, W_Z * (live * lse ** 2).sum() / L]), counts=None, prob_sums=sums)
    res["counts"] = counts.to(torch.int32)
    if case["grad"]:
        res["dlogits"] = grad + (W_Z * 2.0 / L) * (live * lse)[:, None] * p
    return res


def _exact_norm(case, s):
    f64 = torch.float64
    x, w = s["x"].to(f64), s["w"].to(f64)
    if case["kind"] == "layer_norm":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        r = (var + NORM_EPS) ** -0.5
        return dict(xn=torch.addcmul(torch.zeros_like(w) if s["b"] is None else s["b"].to(f64), x * r[:, None] - (mean * r)[:, None], w), mean=mean, rstd=r)
    mean, r, dxn = s["mean"].to(f64).unsqueeze(1), s["rstd"].to(f64).unsqueeze(1), s["dxn"].to(f64)
    hat, d = (x - mean) * r, case["d"]
    up = dxn * w
    dX = r * up - (r / d) * up.sum(1, keepdim=True) - hat * ((r / d) * (up * hat).sum(1, keepdim=True))
    res = dict(dX=dX if s["dres"] is None else dX + s["dres"].to(f64), dw=torch.einsum("td,td->d", dxn, hat))
    if s["b"] is not None:
        res["db"] = dxn.sum(0)
    return res


def exact(case, seed):
    """The results of `run` on these inputs from the definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    return _exact_muon(case, s) if kind == "muon" else _exact_router(case, s) if kind == "router" else _exact_norm(case, s)
