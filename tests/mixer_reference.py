"""Plain forms in 64 bits, on the CPU, of the layers that alternate with the recurrences: short convolution, selective scan, attention over latent rows;
gradients by differentiating these.  Each comes with what its errors are stated in: the sum of the magnitudes of all terms, and for the scan how far
relative errors of a step's factors are carried on."""
import torch


def d(t):
    return None if t is None else t.detach().double().cpu()


def spans(T, cu, B):
    """(first row, length) of the sequences on the flattened token axis."""
    if cu is None:
        return [(n * T, T) for n in range(B)]
    cu = [int(c) for c in cu]
    return [(a, b - a) for a, b in zip(cu, cu[1:])]


def silu(x):
    return x * torch.sigmoid(x)


# ---------------------------------------------------------------- short convolution

def conv(x, w, bias, h0, act, seqs):
    """x [tokens, C], h0 [N, K - 1, C] or None: y, hT, and the magnitude of the sums ahead of the activation."""
    K = w.shape[1]
    ys, last, mags = [], [], []
    for n, (a, m) in enumerate(seqs):
        full = torch.cat([torch.zeros(K - 1, x.shape[1], dtype=x.dtype) if h0 is None else h0[n], x[a:a + m]])
        last.append(full[len(full) - (K - 1):])
        if m == 0:
            continue
        win = full.unfold(0, K, 1)                           # [tokens, C, K]
        s, mag = (win * w).sum(-1), (win.abs() * w.abs()).sum(-1).detach()
        if bias is not None:
            s, mag = s + bias, mag + bias.abs().detach()
        ys.append(silu(s) if act else s)
        mags.append(mag)
    empty = torch.zeros(0, x.shape[1], dtype=torch.float64)
    return torch.cat([empty, *ys]), torch.stack(last), torch.cat([empty, *mags])


def conv_grads(dy, x, w, bias, h0, dhT, act, seqs):
    """{name: (gradient, magnitude)}; a relative error of 2^-24 in the sums moves e = dy act' by up to their magnitude times that."""
    x, w, dy, h0 = d(x), d(w), d(dy), d(h0)
    bias, dhT = d(bias), d(dhT)
    N, K, C = len(seqs), w.shape[1], x.shape[1]
    leaf = [t.clone().requires_grad_() for t in (x, w, torch.zeros(N, K - 1, C, dtype=torch.float64) if h0 is None else h0)]
    b = None if bias is None else bias.clone().requires_grad_()
    y, hT, mag = conv(leaf[0], leaf[1], b, leaf[2], act, seqs)
    out = [y] + ([hT] if dhT is not None else [])
    g = torch.autograd.grad(out, leaf + ([b] if b is not None else []), [dy] + ([dhT] if dhT is not None else []))
    # the same without an activation, of |dy| (1 + magnitude): all terms of all gradients
    e = dy.abs() * (1 + mag)
    pos = [t.abs().clone().requires_grad_() for t in (x, w, leaf[2].detach())]
    pb = None if bias is None else bias.abs().clone().requires_grad_()
    y, hT, _ = conv(pos[0], pos[1], pb, pos[2], False, seqs)
    m = torch.autograd.grad([y] + ([hT] if dhT is not None else []), pos + ([pb] if pb is not None else []), [e] + ([dhT.abs()] if dhT is not None else []))
    return dict(zip(["dx", "dw", "dh0", "db"], zip(g, m)))


# ---------------------------------------------------------------- selective scan

def steps(dt, dt_bias, softplus):
    v = dt if dt_bias is None else dt + dt_bias
    return torch.nn.functional.softplus(v, threshold=1e9) if softplus else v


def scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, seqs):
    """x, dt, z [tokens, ch], B, C [tokens, G, S]: y, hT, and errors E of the states and of y for a relative error of one in every factor of every step."""
    ch, S = A.shape
    of = torch.arange(ch) // (ch // B.shape[1])
    delta = steps(dt, dt_bias, softplus)
    ys, last, es, elast = [], [], [], []
    for n, (a, m) in enumerate(seqs):
        h = torch.zeros(ch, S, dtype=torch.float64) if h0 is None else h0[n]
        H, E = h.detach().abs(), torch.zeros(ch, S, dtype=torch.float64)
        for t in range(a, a + m):
            g = delta[t][:, None] * A
            u = (delta[t] * x[t])[:, None] * B[t][of]
            h = g.exp() * h + u
            with torch.no_grad():
                E = g.exp() * (E + (1 + g.abs()) * H) + u.abs()
                H = g.exp() * H + u.abs()
                E = E + H
                e = ((E + H) * C[t][of].abs()).sum(-1)
                if D is not None:
                    e = e + (D * x[t]).abs()
                es.append(e if z is None else e * silu(z[t]).abs())
            y = (h * C[t][of]).sum(-1)
            if D is not None:
                y = y + D * x[t]
            ys.append(y if z is None else y * silu(z[t]))
        last.append(h)
        elast.append(E)
    empty = torch.zeros(0, ch, dtype=torch.float64)
    return torch.stack(ys) if ys else empty, torch.stack(last), torch.stack(es) if es else empty, torch.stack(elast)


def scan_grads(dy, x, dt, A, B, C, D, z, dt_bias, softplus, h0, dhT, seqs):
    """{name: (gradient, error for a relative error of one in every factor)}"""
    t = {k: d(v) for k, v in dict(x=x, dt=dt, A=A, B=B, C=C, D=D, z=z, dt_bias=dt_bias, h0=h0).items() if v is not None}
    dy, dhT, ch, S, N = d(dy), d(dhT), A.shape[0], A.shape[1], len(seqs)
    if "h0" not in t:
        t["h0"] = torch.zeros(N, ch, S, dtype=torch.float64)
    leaf = {k: v.clone().requires_grad_() for k, v in t.items()}
    get = leaf.get
    y, hT, _, _ = scan(leaf["x"], leaf["dt"], leaf["A"], leaf["B"], leaf["C"], get("D"), get("z"), get("dt_bias"), softplus, leaf["h0"], seqs)
    got = torch.autograd.grad([y] + ([hT] if dhT is not None else []), list(leaf.values()), [dy] + ([dhT] if dhT is not None else []), allow_unused=True)
    grads = {"d" + k: torch.zeros_like(leaf[k]) if g is None else g for k, g in zip(leaf, got)}
    # errors: states forwards, their gradients backwards, each with what it carries on
    G, of = t["B"].shape[1], torch.arange(ch) // (ch // t["B"].shape[1])
    v = t["dt"] if "dt_bias" not in t else t["dt"] + t["dt_bias"]
    delta, slope = (torch.nn.functional.softplus(v, threshold=1e9), torch.sigmoid(v)) if softplus else (v, torch.ones_like(v))
    gate = torch.ones_like(dy) if "z" not in t else silu(t["z"]).abs()
    err = {k: torch.zeros_like(g) for k, g in grads.items()}
    group = lambda e: torch.zeros(G, S, dtype=torch.float64).index_add_(0, of, e)   # noqa: E731
    for n, (a, m) in enumerate(seqs):
        H, E = t["h0"][n].abs(), torch.zeros(ch, S, dtype=torch.float64)
        kept = []
        for i in range(a, a + m):
            g = (delta[i][:, None] * t["A"])
            u = (delta[i] * t["x"][i])[:, None].abs() * t["B"][i][of].abs()
            kept.append((H, E))
            E = g.exp() * (E + (1 + g.abs()) * H) + u
            H = g.exp() * H + u
            E = E + H
            kept[-1] += (H, E)
        Q = torch.zeros(ch, S, dtype=torch.float64) if dhT is None else dhT[n].abs()
        F = Q * 0
        for i in reversed(range(a, a + m)):
            g = delta[i][:, None] * t["A"]
            was, ewas, now, enow = kept.pop()
            gy = (dy[i].abs() * gate[i])[:, None]
            Q = Q + gy * t["C"][i][of].abs()
            F = F + Q
            u = (delta[i] * t["x"][i]).abs()[:, None]
            to_b = ((Q + F) * t["B"][i][of].abs()).sum(-1)
            flow = g.exp() * (F * was + Q * ewas + (2 + g.abs()) * Q * was)
            err["dx"][i] = delta[i] * to_b + (gy[:, 0] * t["D"].abs() if "D" in t else 0)
            ddelta = (flow * t["A"].abs()).sum(-1) + t["x"][i].abs() * to_b
            err["ddt"][i] = ddelta * slope[i]
            err["dA"] += flow * delta[i][:, None]
            err["dB"][i] = group((Q + F) * u)
            err["dC"][i] = group((now + enow) * gy)
            if "z" in t:
                p = ((now + enow) * t["C"][i][of].abs()).sum(-1) + (t["D"] * t["x"][i]).abs() if "D" in t else ((now + enow) * t["C"][i][of].abs()).sum(-1)
                err["dz"][i] = dy[i].abs() * p * 1.1
            if "D" in t:
                err["dD"] += gy[:, 0] * t["x"][i].abs()
            if "dt_bias" in t:
                err["ddt_bias"] += ddelta * slope[i]
            F = g.exp() * (F + (1 + g.abs()) * Q)
            Q = g.exp() * Q
        err["dh0"][n] = Q + F
    return {k: (grads[k], err[k] + grads[k].abs()) for k in grads}


# ---------------------------------------------------------------- attention

def attend(q, k, v, limit, scale):
    """q [rows, d], k [keys, d], v [keys, dv], limit [rows]: keys that each row sees.  o, lse, sum of weights times |v|, and the largest sum of
    magnitudes behind a score."""
    s = q @ k.T * scale
    mag = (q.abs() @ k.abs().T * abs(scale))
    hidden = torch.arange(len(k)) >= limit[:, None]
    s = s.masked_fill(hidden, -torch.inf)
    lse = torch.logsumexp(s, -1) if len(k) else torch.full((len(q),), -torch.inf, dtype=torch.float64)
    p = torch.where(hidden, torch.zeros_like(s), torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None]))
    top = mag.masked_fill(hidden, 0).amax(-1) if len(k) else torch.zeros(len(q), dtype=torch.float64)
    clean = torch.where((~hidden).any(0)[:, None], v, torch.zeros_like(v))
    return p @ clean, lse, p @ clean.abs(), top
