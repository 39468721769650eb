"""Plain forms in 64 bits, on the CPU, of what stands next to the delta-rule recurrence: gated linear attention token by token, its
gradients by the chain rule through the same steps, and the norms.  Each also with absolute values in place of the inputs: the sum
of the magnitudes of all terms, which error bounds are stated in."""
import torch


def d(t):
    return None if t is None else t.detach().double().cpu()


def lengths(q, cu):
    """(first row, length) of the sequences; rows are those of the token axis of the flattened [B, T]."""
    if cu is None:
        return [(n * q.shape[1], q.shape[1]) for n in range(q.shape[0])]
    cu = cu.tolist()
    return [(a, b - a) for a, b in zip(cu, cu[1:])]


def gla(q, k, v, g, h0=None, cu=None, scale=1.0, magnitude=False):
    """o [B, T, HV, d], hT [N, HV, d, d]."""
    q, k, v, g, h0 = d(q), d(k), d(v), d(g), d(h0)
    if magnitude:
        q, k, v, h0, scale = q.abs(), k.abs(), v.abs(), None if h0 is None else h0.abs(), abs(scale)
    seqs, (HK, D), HV = lengths(q, cu), q.shape[2:], v.shape[2]
    of = torch.arange(HV) // (HV // HK)
    fq, fk, fv, fg = (x.reshape(-1, *x.shape[2:]) for x in (q, k, v, g))
    o, hT = torch.zeros_like(fv), torch.zeros(len(seqs), HV, D, D, dtype=torch.float64)
    for n, (t0, L) in enumerate(seqs):
        h = hT[n] if h0 is None else h0.reshape(len(seqs), HV, D, D)[n].clone()
        for t in range(t0, t0 + L):
            h = fg[t].exp()[:, None, None] * h + fk[t][of][:, :, None] * fv[t][:, None, :]
            o[t] = scale * torch.einsum("hkv,hk->hv", h, fq[t][of])
        hT[n] = h
    return o.reshape(v.shape), hT


def gla_backward(do, q, k, v, g, h0=None, dhT=None, cu=None, scale=1.0, magnitude=False):
    """dq, dk (per V-head: [.., HV, d]), dv, dg, dh0."""
    do, q, k, v, g, h0, dhT = (d(t) for t in (do, q, k, v, g, h0, dhT))
    if magnitude:
        do, q, k, v, h0, dhT = (None if t is None else t.abs() for t in (do, q, k, v, h0, dhT))
        scale = abs(scale)
    seqs, (HK, D), HV = lengths(q, cu), q.shape[2:], v.shape[2]
    of = torch.arange(HV) // (HV // HK)
    fo, fq, fk, fv, fg = (x.reshape(-1, *x.shape[2:]) for x in (do, q, k, v, g))
    dq, dk, dv, dg = torch.zeros_like(fv), torch.zeros_like(fv), torch.zeros_like(fv), torch.zeros_like(fg)
    dh0 = torch.zeros(len(seqs), HV, D, D, dtype=torch.float64)
    for n, (t0, L) in enumerate(seqs):
        h = dh0[n].clone() if h0 is None else h0.reshape(len(seqs), HV, D, D)[n]
        hs = [h]
        for t in range(t0, t0 + L):
            h = fg[t].exp()[:, None, None] * h + fk[t][of][:, :, None] * fv[t][:, None, :]
            hs.append(h)
        dh = torch.zeros_like(h) if dhT is None else dhT.reshape(len(seqs), HV, D, D)[n]
        for t in reversed(range(t0, t0 + L)):
            a = fg[t].exp()[:, None, None]
            dh = dh + scale * fq[t][of][:, :, None] * fo[t][:, None, :]
            dv[t] = torch.einsum("hkv,hk->hv", dh, fk[t][of])
            dk[t] = torch.einsum("hkv,hv->hk", dh, fv[t])
            dq[t] = scale * torch.einsum("hkv,hv->hk", hs[t - t0 + 1], fo[t])
            dh = a * dh
            dg[t] = (dh * hs[t - t0]).sum((-1, -2))
        dh0[n] = dh
    return dq.reshape(v.shape), dk.reshape(v.shape), dv.reshape(v.shape), dg.reshape(g.shape), dh0


def heads_sum(x, HK):
    """[.., HV, d] -> [.., HK, d]: the sum over the V-heads of a q/k head."""
    return x.reshape(*x.shape[:-2], HK, -1, x.shape[-1]).sum(-2)


def rms_scale(x, eps):
    return 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()


def act(z, name):
    """Value and slope."""
    if z is None:
        return torch.ones(1, dtype=torch.float64), None
    s = torch.sigmoid(z)
    return (z * s, s * (1 + z * (1 - s))) if name == "silu" else (s, s * (1 - s))


def gated_norm(x, w, z, name, eps):
    x, w, z = d(x), d(w), d(z)
    return x * rms_scale(x, eps) * w * act(z, name)[0]


def norm_backward(x, rs, dn):
    n = x * rs
    return rs * (dn - n * (dn * n).mean(-1, keepdim=True)), rs * (dn.abs() + n.abs() * (dn * n).abs().mean(-1, keepdim=True))


def gated_norm_backward(dy, x, w, z, name, eps):
    """{name: (gradient, magnitude of its terms)}"""
    dy, x, w, z = d(dy), d(x), d(w), d(z)
    a, slope = act(z, name)
    rs = rms_scale(x, eps)
    t = dy * x * rs * a
    out = {"dx": norm_backward(x, rs, dy * w * a), "dw": (t.sum(0), t.abs().sum(0))}
    if z is not None:
        dz = dy * x * rs * w * slope
        s = torch.sigmoid(z)                               # (the slope of silu is a sum of two terms)
        out["dz"] = (dz, (dy * x * rs * w).abs() * (s * (1 + (z * (1 - s)).abs()) if name == "silu" else slope))
    return out


def add_norm(x, r, w, w_post, scale, eps):
    """y, r_out, and the magnitude of r_out's terms."""
    x, r, w, w_post = d(x), d(r), d(w), d(w_post)
    f = x if w_post is None else x * rms_scale(x, eps) * w_post
    out = r + scale * f
    return out * rms_scale(out, eps) * w, out, r.abs() + abs(scale) * f.abs()


def add_norm_backward(dy, dr_out, x, r_out, w, w_post, scale, eps):
    dy, dr_out, x, r, w, w_post = (d(t) for t in (dy, dr_out, x, r_out, w, w_post))
    rs = rms_scale(r, eps)
    t = dy * r * rs
    dr, mag = norm_backward(r, rs, dy * w)
    if dr_out is not None:
        dr, mag = dr + dr_out, mag + dr_out.abs()
    out = {"dr": (dr, mag), "dw": (t.sum(0), t.abs().sum(0))}
    if w_post is None:
        out["dx"] = (scale * dr, abs(scale) * mag)
        return out
    rx = rms_scale(x, eps)
    dx, _ = norm_backward(x, rx, scale * dr * w_post)
    _, m = norm_backward(x.abs(), rx, abs(scale) * mag * w_post.abs())
    out["dx"] = (dx, m)
    out["dw_post"] = ((scale * dr * x * rx).sum(0), (abs(scale) * mag * x.abs() * rx).sum(0))
    return out
