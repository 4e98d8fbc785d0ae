"""Plain 64-bit statements of layer norm, the router's losses and the Muon step, for their tests. `within` and U are those of block_reference."""
import torch

NS = (3.4445, -4.7750, 2.0315)


def f64(t):
    return None if t is None else t.detach().double().cpu()


def layer_norm(x, w, b, eps):
    """xn, mean, rstd."""
    x, w, b = f64(x), f64(w), f64(b)
    mean = x.mean(1)
    off = x - mean[:, None]
    r = (off.square().mean(1) + eps) ** -0.5
    xn = off * r[:, None] * w
    return (xn if b is None else xn + b), mean, r


def layer_norm_bwd(dxn, x, w, mean, rstd, dres):
    """{name: (value, magnitudes of its terms)}."""
    dxn, x, w, mean, rstd, dres = map(f64, (dxn, x, w, mean, rstd, dres))
    r = rstd[:, None]
    n, n_terms = (x - mean[:, None]) * r, (x.abs() + mean.abs()[:, None]) * r
    u = dxn * w
    dX = r * (u - u.mean(1, keepdim=True) - n * (u * n).mean(1, keepdim=True))
    terms = r * (u.abs() + u.abs().mean(1, keepdim=True) + n_terms * (u.abs() * n_terms).mean(1, keepdim=True))
    if dres is not None:
        dX, terms = dX + dres, terms + dres.abs()
    return dict(dX=(dX, terms), dw=((dxn * n).sum(0), (dxn.abs() * n_terms).sum(0)), db=(dxn.sum(0), dxn.abs().sum(0)))


def router_losses(logits, idx, keep, offsets, w_balance, w_z, grad=True):
    """losses (a tensor that may be differentiated), counts, prob_sums, live rows. A row of -inf alone has p = 0 and lse = 0."""
    T, n = logits.shape
    k = idx.shape[1]
    ends = [0, T] if offsets is None else [min(int(e), int(offsets[-1])) for e in offsets]
    S = len(ends) - 1
    live = torch.zeros(T, dtype=torch.bool)
    live[ends[0]:ends[-1]] = True
    if keep is not None:
        live &= keep.cpu() != 0
    L = int(live.sum())
    counts, sums = torch.zeros(S, n, dtype=torch.int64), []
    balance, z = torch.zeros((), dtype=torch.float64), torch.zeros((), dtype=torch.float64)
    for s in range(S):
        rows = [t for t in range(ends[s], ends[s + 1]) if live[t]]
        open_rows = [t for t in rows if bool((logits[t] > -float("inf")).any() | logits[t].isnan().any())]
        for e in idx[rows].reshape(-1).tolist() if rows else []:
            if 0 <= e < n:
                counts[s, e] += 1
        x = logits[open_rows]
        p = torch.softmax(x, 1)
        total = p.sum(0)
        sums.append(total.detach())
        if rows:
            balance = balance + (counts[s].double() * total).sum() / len(rows)
            z = z + torch.logsumexp(x, 1).square().sum()
    scale = max(L, 1)
    return torch.stack([w_balance * n / (k * scale) * balance, w_z / scale * z]), counts, torch.stack(sums), live


def muon(w, g, m, lr, momentum, eps, steps, nesterov, scale, decay, grad_scale, m_type):
    """w, m and the orthogonalised update of one tensor [count, rows, cols] in 64 bits; m is rounded to its type where u is made of it."""
    w, g, m = f64(w), f64(g) * grad_scale, f64(m)
    m = momentum * m + g
    held = m.to(m_type).double()
    u = g + momentum * held if nesterov else held
    x = u / (u.flatten(1).norm(dim=1)[:, None, None] + eps)
    a, b, c = NS
    for _ in range(steps):
        if x.shape[1] <= x.shape[2]:
            q = x @ x.mT
            x = a * x + (b * q + c * q @ q) @ x
        else:
            q = x.mT @ x
            x = a * x + x @ (b * q + c * q @ q)
    return w - lr * (scale * x + decay * w), m, x
