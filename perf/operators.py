"""What stands around the delta-rule recurrence in a hybrid model, as cases that can be timed and compared.

Four operators:

  gla_decode   one token per sequence of a gated linear attention head: h <- e^g h + k v^T, o = scale h^T q
  gla          the same recurrence over whole sequences, forward (outputs, final state) and backward (gradients of q, k, v,
               the log-gates and the start state)
  gated_norm   y = x / rms(x) * w * act(z) over the channels of a head, behind the recurrence; forward and backward
  add_norm     at the border of two blocks: f = x, or x / rms(x) * w_post; r' = r + scale * f; y = r' / rms(r') * w;
               forward and backward

Values: unit-norm q and k, v and gradients ~ N(0, 1), log-gate = -softplus(N(0, 1) + gate_shift), states ~ N(0, std 0.5); rows
of the norms ~ N(0, 1), weights ~ 1 + N(0, 0.1).  q, k, v and rows in bf16 or fp32; gates, states and weights fp32.

`own` false: plain torch operations in 32 bits (cumulative gates in 64); `own` true: the library's entry points.
"""
import math
import random

import torch

own = False

EPS = 1e-6
BLOCK = 64                                                   # tokens that the plain recurrence takes together


# ---------------------------------------------------------------------------------------------------------------- the cases

def _gla(name, back, hk, hv, d=128, dtype="bf16", rows=1, tokens=0, packed=0, lo=0, hi=0, len_seed=0, h0=False, gate_shift=2.0):
    """`rows` sequences of `tokens` tokens each, or, with `packed` > 0, that many of lo..hi tokens end to end."""
    c = dict(op="gla", back=back, dtype=dtype, d=d, hk=hk, hv=hv, rows=rows, tokens=tokens, packed=packed, lo=lo, hi=hi,
             len_seed=len_seed, h0=h0, gate_shift=gate_shift)
    return dict(c, name=name) if name else c


def _decode(name, n, hk, hv, d=128, dtype="bf16"):
    c = dict(op="gla_decode", back=False, dtype=dtype, d=d, hk=hk, hv=hv, n=n, gate_shift=2.0)
    return dict(c, name=name) if name else c


def _norm(name, op, back, rows, cols, dtype="bf16", act="silu", post=False, scale=1.0):
    c = dict(op=op, back=back, rows=rows, cols=cols, dtype=dtype, act=act, post=post, scale=scale)
    return dict(c, name=name) if name else c


def listed():
    return [
        # interactive decoding of one sequence: called for every token of every layer, latency is all of it
        _decode("gla_decode_n1", 1, 16, 16),
        # the decoding step of a full batch, two V-heads to a q/k head: 420 MB of states
        _decode("gla_decode_n200", 200, 16, 32),
        # two short fp32 sequences with small heads, one token over four chunks: a layer checked against a float64 reference
        _gla("gla_fp32_t257", False, 4, 4, d=64, dtype="fp32", rows=2, tokens=257, h0=True, gate_shift=0.0),
        # the layer of a ~2B hybrid model on a 4k prompt
        _gla("gla_t4096", False, 16, 16, tokens=4096),
        # prompts of 512 to 16384 tokens, each continued from a state: the largest call of serving
        _gla("gla_packed_8", False, 16, 16, packed=8, lo=512, hi=16384, len_seed=11, h0=True),
        # a fine-tuning step on one short ragged example
        _gla("gla_back_t333", True, 16, 16, tokens=333),
        # a training step on packed documents of uneven lengths, two V-heads to a q/k head, states carried between windows
        _gla("gla_back_packed_6", True, 8, 16, packed=6, lo=300, hi=5000, len_seed=5, h0=True),
        # a training step of that layer: four rows of 4096 tokens
        _gla("gla_back_b4_t4096", True, 16, 16, rows=4, tokens=4096),
        # the gated norm of a decoding batch: 37 tokens of 16 heads
        _norm("gated_norm_37", "gated_norm", False, 37 * 16, 128),
        # its backward pass in training, 8192 tokens of 32 heads
        _norm("gated_norm_back_8k", "gated_norm", True, 8192 * 32, 128),
        # block border while decoding one sequence
        _norm("add_norm_1", "add_norm", False, 1, 2048),
        # block border in training with a norm behind the block and a scaled residual, 16384 tokens
        _norm("add_norm_back_16k", "add_norm", True, 16384, 2048, post=True, scale=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.random()
    if kind < 0.15:                                          # decoding: 1 to 200 sequences
        hk = rng.choice([1, 2, 4, 8, 16, 32])
        hv = hk * rng.choice([1, 1, 2, 4])
        return _decode(None, _log_int(rng, 1, 200 * 32 // max(32, hv)), hk, hv, d=rng.choice([128, 128, 64]), dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if kind < 0.65:
        back = rng.random() < 0.5
        shift = rng.choice([2.0, 2.0, 0.0, 4.0])
        h0 = rng.random() < 0.5
        if rng.random() < 0.3:                               # fp32 inputs or small heads: short and medium sequences
            dtype, d = rng.choice([("fp32", 64), ("fp32", 128), ("bf16", 64)])
            hk = rng.choice([1, 2, 4, 8])
            hv = hk * rng.choice([1, 1, 2])
            top = 1500 if d == 64 else 600
        else:
            dtype, d = "bf16", 128
            hk = rng.choice([1, 2, 4, 8, 16])
            hv = hk * rng.choice([1, 1, 2])
            top = min(16384, (1 << (18 if back else 19)) // hv)
        if rng.random() < 0.4:
            n = _log_int(rng, 2, 24)
            hi = max(32, top // n)
            return _gla(None, back, hk, hv, d=d, dtype=dtype, packed=n, lo=rng.choice([1, max(1, hi // 8)]), hi=hi, len_seed=rng.randrange(1 << 20),
                        h0=h0, gate_shift=shift)
        rows = rng.choice([1, 1, 2, 4])
        return _gla(None, back, hk, hv, d=d, dtype=dtype, rows=rows, tokens=_log_int(rng, 8, top // rows), h0=h0, gate_shift=shift)
    back, dtype = rng.random() < 0.5, rng.choice(["bf16", "bf16", "fp32"])
    most = (1 << 24) if dtype == "fp32" else (1 << 25)       # elements of one tensor
    if kind < 0.82:
        cols = rng.choice([64, 128, 128, 256, rng.randint(40, 200)])
        return _norm(None, "gated_norm", back, _log_int(rng, 1, most // cols), cols, dtype=dtype, act=rng.choice(["silu", "silu", "sigmoid"]))
    cols = rng.choice([1024, 2048, 4096, rng.randint(300, 6000)])
    return _norm(None, "add_norm", back, _log_int(rng, 1, most // cols), cols, dtype=dtype, post=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 0.5]))


# ---------------------------------------------------------------------------------------------------------------- the inputs

def _lengths(c):
    if c["packed"]:
        r = random.Random(c["len_seed"])
        return [r.randint(c["lo"], c["hi"]) for _ in range(c["packed"])]
    return [c["tokens"]] * c["rows"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, dt = case, torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if c["op"] in ("gated_norm", "add_norm"):
        n, d = c["rows"], c["cols"]
        s = dict(c, x=normal(n, d).to(dt), w=1 + 0.1 * normal(d), w_post=1 + 0.1 * normal(d) if c["post"] else None)
        if c["op"] == "gated_norm":
            s["z"] = normal(n, d).to(dt)
        else:
            s["r"] = normal(n, d).to(dt)                     # (backward: the residual stream behind the addition)
        if c["back"]:
            s["dy"], s["dr"] = normal(n, d).to(dt), normal(n, d).to(dt) if c["op"] == "add_norm" else None
        return s

    def unit(*shape):
        return torch.nn.functional.normalize(normal(*shape), dim=-1).to(dt).contiguous()

    d, hk, hv = c["d"], c["hk"], c["hv"]
    lens = [1] * c["n"] if c["op"] == "gla_decode" else _lengths(c)
    lead = (c["n"],) if c["op"] == "gla_decode" else (1, sum(lens)) if c["packed"] else (c["rows"], c["tokens"])
    s = dict(c, q=unit(*lead, hk, d), k=unit(*lead, hk, d), v=normal(*lead, hv, d).to(dt),
             g=-torch.nn.functional.softplus(normal(*lead, hv) + c["gate_shift"]))
    if c["op"] == "gla_decode":
        s["state"] = 0.5 * normal(c["n"], hv, d, d)
        return s
    s["h0"] = 0.5 * normal(len(lens), hv, d, d) if c["h0"] else None
    if c["back"]:
        s["do"] = normal(*lead, hv, d).to(dt)
        s["dhT"] = 0.5 * normal(len(lens), hv, d, d) if c["h0"] else None
    s["cu_seqlens"], s["max_seqlen"] = None, 0
    if c["packed"]:
        s["cu_seqlens"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
        s["max_seqlen"] = max(lens)
    # where the tokens of each sequence's blocks are: [sequences, blocks of 64, 64] rows of the token axis, and which are none
    at = torch.arange(-(-max(lens) // BLOCK) * BLOCK)
    start = torch.tensor([sum(lens[:i]) for i in range(len(lens))])
    none = at[None] >= torch.tensor(lens)[:, None]
    s["rows_of"] = torch.where(none, torch.zeros_like(at), start[:, None] + at[None]).reshape(len(lens), -1, BLOCK).cuda()
    s["none"] = none.reshape(len(lens), -1, BLOCK).cuda()
    return s


# ---------------------------------------------------------------------------------------------------------------- one pass

def run(s):
    if s["op"] == "gla_decode":
        return _own_decode(s) if own else _plain_decode(s)
    if s["op"] == "gla":
        if s["back"]:
            return _own_gla_back(s) if own else _plain_gla_back(s)
        return _own_gla(s) if own else _plain_gla(s)
    if s["op"] == "gated_norm":
        if s["back"]:
            return _own_gated_norm_back(s) if own else _plain_gated_norm_back(s)
        return _own_gated_norm(s) if own else _plain_gated_norm(s)
    if s["back"]:
        return _own_add_norm_back(s) if own else _plain_add_norm_back(s)
    return _own_add_norm(s) if own else _plain_add_norm(s)


# ... by the library

def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def _own_decode(s):
    """To another state, so that every pass starts from the same one; that buffer is kept."""
    if "state_out" not in s:
        s["state_out"] = torch.empty_like(s["state"])
    o, state = _ha().ha_la_gla_decode(s["q"], s["k"], s["v"], s["g"], s["state"], state_out=s["state_out"])
    return {"o": o, "state": state}


def _own_gla(s):
    """The scratch workspace and the status word are kept from call to call, as a serving program does."""
    o, hT, s["status_word"], s["workspace"] = _ha().ha_la_gla_prefill(
        s["q"], s["k"], s["v"], s["g"], h0=s["h0"], cu_seqlens=s["cu_seqlens"], max_seqlen=s["max_seqlen"],
        workspace=s.get("workspace"), status_word=s.get("status_word"))
    return {"o": o, "hT": hT}


def _own_gla_back(s):
    dq, dk, dv, dg, dh0, s["status_word"], s["workspace"] = _ha().ha_la_gla_backward(
        s["do"], s["q"], s["k"], s["v"], s["g"], h0=s["h0"], dhT=s["dhT"], cu_seqlens=s["cu_seqlens"], max_seqlen=s["max_seqlen"],
        workspace=s.get("workspace"), status_word=s.get("status_word"))
    return {"dq": dq, "dk": dk, "dv": dv, "dg": dg, "dh0": dh0}


def _own_gated_norm(s):
    return {"y": _ha().ha_la_gated_norm(s["x"], s["w"], s["z"], activation=s["act"], eps=EPS)}


def _own_gated_norm_back(s):
    dx, dw, dz = _ha().ha_la_gated_norm_backward(s["dy"], s["x"], s["w"], s["z"], activation=s["act"], eps=EPS)
    return {"dx": dx, "dw": dw, "dz": dz}


def _own_add_norm(s):
    y, r = _ha().ha_la_add_norm(s["x"], s["r"], s["w"], w_post=s["w_post"], scale=s["scale"], eps=EPS)
    return {"y": y, "r": r}


def _own_add_norm_back(s):
    dx, dr, dw, dw_post = _ha().ha_la_add_norm_backward(s["dy"], s["dr"], s["x"], s["r"], s["w"], w_post=s["w_post"],
                                                        scale=s["scale"], eps=EPS)
    return {"dx": dx, "dr": dr, "dw": dw, **({"dw_post": dw_post} if s["post"] else {})}


# ... in plain operations

def _plain_decode(s):
    dt, r = s["q"].dtype, s["hv"] // s["hk"]
    q, k = (s[x].float().repeat_interleave(r, 1) for x in "qk")
    h = torch.exp(s["g"])[..., None, None] * s["state"] + k[..., :, None] * s["v"].float()[..., None, :]
    return {"o": (h * q[..., :, None]).sum(-2).to(dt), "state": h}


def _blocks(s, x, heads):
    """x [.., heads, ..] in blocks of tokens, [sequences, heads of v, blocks, 64, ..], zeros where there is no token."""
    x = x.reshape(-1, *x.shape[2:])[s["rows_of"]]
    x = x.masked_fill(s["none"].reshape(*s["none"].shape, *[1] * (x.dim() - 3)), 0)
    if heads != s["hv"]:
        x = x.repeat_interleave(s["hv"] // heads, 3)
    return x.movedim(3, 1)


def _rows(s, x, like):
    """... and back: [sequences, heads, blocks, 64, ..] in the layout and type of `like`."""
    out = torch.empty(like.shape[0] * like.shape[1], *x.movedim(1, 3).shape[3:], dtype=x.dtype, device=x.device)
    keep = ~s["none"]
    out[s["rows_of"][keep]] = x.movedim(1, 3)[keep]
    return out


def _gates(s):
    """Cumulative log-gates in 64 bits: G within a block, its total, and the decay between blocks in both directions."""
    G = _blocks(s, s["g"].double(), s["hv"]).cumsum(-1)      # [N, H, C, 64]
    total = G[..., -1]
    ends = total.cumsum(-1)                                  # log-gate from the start to the end of block c
    starts = ends - total
    c = torch.arange(total.shape[-1], device=G.device)
    before = c[:, None] > c[None]                            # block of the row behind block of the column
    carry = torch.exp((starts[..., :, None] - ends[..., None, :]).masked_fill(~before, -math.inf)).float()
    i = torch.arange(BLOCK, device=G.device)
    decay = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(i[:, None] < i[None], -math.inf)).float()
    return G, total, starts, ends, carry, decay


def _states_before(s, k, v, G, total, starts, carry, h0):
    """State at the start of each block, and what each block adds to it."""
    add = (k * torch.exp(total[..., None] - G).float()[..., None]).transpose(-1, -2) @ v
    N, H, C, d, _ = add.shape
    h = (carry @ add.reshape(N, H, C, d * d)).reshape(N, H, C, d, d)
    if h0 is not None:
        h = h + torch.exp(starts).float()[..., None, None] * h0[:, :, None]
    return h, add


def _plain_gla(s):
    q, k, v = _blocks(s, s["q"].float(), s["hk"]), _blocks(s, s["k"].float(), s["hk"]), _blocks(s, s["v"].float(), s["hv"])
    G, total, starts, ends, carry, decay = _gates(s)
    h, add = _states_before(s, k, v, G, total, starts, carry, s["h0"])
    o = ((q @ k.transpose(-1, -2)) * decay) @ v + torch.exp(G).float()[..., None] * (q @ h)
    hT = torch.exp(total[..., -1]).float()[..., None, None] * h[:, :, -1] + add[:, :, -1]
    return {"o": _rows(s, o, s["v"]).to(s["v"].dtype).reshape(s["v"].shape), "hT": hT}


def _plain_gla_back(s):
    q, k, v, do = (_blocks(s, s[x].float(), s[x].shape[2]) for x in ("q", "k", "v", "do"))
    G, total, starts, ends, carry, decay = _gates(s)
    h, _ = _states_before(s, k, v, G, total, starts, carry, s["h0"])
    # gradient of the state behind each block, from later blocks' outputs and the final state
    give = (q * torch.exp(G).float()[..., None]).transpose(-1, -2) @ do
    N, H, C, d, _ = give.shape
    dh = (carry.transpose(-1, -2) @ give.reshape(N, H, C, d * d)).reshape(N, H, C, d, d)
    if s["dhT"] is not None:
        dh = dh + torch.exp(ends[..., -1:] - ends).float()[..., None, None] * s["dhT"][:, :, None]
    dh0 = torch.exp(total[..., 0]).float()[..., None, None] * dh[:, :, 0] + give[:, :, 0]
    S, dP = q @ k.transpose(-1, -2), do @ v.transpose(-1, -2)
    from_start, to_end = torch.exp(G).float()[..., None], torch.exp(total[..., None] - G).float()[..., None]
    dq1, dk1 = from_start * (do @ h.transpose(-1, -2)), to_end * (v @ dh.transpose(-1, -2))
    dS = dP * decay
    dq, dk = dS @ k + dq1, dS.transpose(-1, -2) @ q + dk1
    dv = (S * decay).transpose(-1, -2) @ do + to_end * (k @ dh)
    # gate t scales everything that goes from before it to t or later
    E = (S * dS).tril(-1).double()
    x, y = (q * dq1).sum(-1).double(), (k * dk1).sum(-1).double()
    later = lambda e: e.flip(-1).cumsum(-1).flip(-1)         # noqa: E731
    dg = later(x + E.sum(-1) - E.sum(-2)) + (y.cumsum(-1) - y) + torch.exp(total)[..., None] * (h * dh).sum((-1, -2)).double()[..., None]

    def heads(e, like):                                      # (shared q/k heads: the sum over their V-heads)
        e = _rows(s, e, like)
        return e.reshape(e.shape[0], s["hk"], -1, d).sum(2).to(like.dtype).reshape(like.shape)

    return {"dq": heads(dq, s["q"]), "dk": heads(dk, s["k"]), "dv": _rows(s, dv, s["v"]).to(s["v"].dtype).reshape(s["v"].shape),
            "dg": _rows(s, dg, s["g"]).float().reshape(s["g"].shape), "dh0": dh0}


def _rms(x):
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _act(s):
    """The gate's value and slope."""
    z = s["z"].float()
    e = torch.sigmoid(z)
    return (e * z, e * (1 + z * (1 - e))) if s["act"] == "silu" else (e, e * (1 - e))


def _plain_gated_norm(s):
    x = s["x"].float()
    return {"y": (x * _rms(x) * s["w"] * _act(s)[0]).to(s["x"].dtype)}


def _norm_back(x, rs, dn):
    n = x * rs
    return rs * (dn - n * (dn * n).mean(-1, keepdim=True))


def _plain_gated_norm_back(s):
    x, dy = s["x"].float(), s["dy"].float()
    a, slope = _act(s)
    rs = _rms(x)
    n = x * rs
    return {"dx": _norm_back(x, rs, dy * s["w"] * a).to(s["x"].dtype), "dw": (dy * n * a).double().sum(0).float(),
            "dz": (dy * n * s["w"] * slope).to(s["x"].dtype)}


def _plain_add_norm(s):
    f = s["x"].float()
    if s["post"]:
        f = f * _rms(f) * s["w_post"]
    r = s["r"].float() + s["scale"] * f
    return {"y": (r * _rms(r) * s["w"]).to(s["x"].dtype), "r": r.to(s["x"].dtype)}


def _plain_add_norm_back(s):
    x, r, dy = s["x"].float(), s["r"].float(), s["dy"].float()
    rs = _rms(r)
    dr = s["dr"].float() + _norm_back(r, rs, dy * s["w"])
    out = {"dr": dr.to(s["x"].dtype), "dw": (dy * r * rs).double().sum(0).float()}
    df = s["scale"] * dr
    if s["post"]:
        rx = _rms(x)
        out["dw_post"] = (df * x * rx).double().sum(0).float()
        df = _norm_back(x, rx, df * s["w_post"])
    return {"dx": df.to(s["x"].dtype), **out}


# ---------------------------------------------------------------------------------------------------------------- how much work

def work(case):
    """Each input read once, each output written once; multiply-adds counted as two operations."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] in ("gated_norm", "add_norm"):
        tensors = {("gated_norm", False): 3, ("gated_norm", True): 5, ("add_norm", False): 4, ("add_norm", True): 6}[c["op"], c["back"]]
        vectors = (1 + c["post"]) * (2 if c["back"] else 1)
        per = {("gated_norm", False): 9, ("gated_norm", True): 20, ("add_norm", False): 8, ("add_norm", True): 16}[c["op"], c["back"]]
        return {"bytes": c["rows"] * c["cols"] * e * tensors + 4 * c["cols"] * vectors, "flops": float(c["rows"] * c["cols"] * per)}
    d, hk, hv = c["d"], c["hk"], c["hv"]
    state = hv * d * d * 4
    if c["op"] == "gla_decode":
        return {"bytes": c["n"] * (2 * (hk + hv) * d * e + 4 * hv + 2 * state), "flops": c["n"] * hv * 5.0 * d * d}
    lens = _lengths(c)
    tokens, n = sum(lens), len(lens)
    # blocks of 64 tokens, half of a block's pairs: 2 products of pairs and 2 of the state forward; 5 and 5 backward
    pairs, wide = (5, 5) if c["back"] else (2, 2)
    flops = tokens * hv * 2.0 * (pairs * 32 * d + wide * d * d)
    if c["back"]:
        return {"bytes": tokens * ((4 * hk + 3 * hv) * d * e + 8 * hv) + (3 if c["h0"] else 1) * n * state, "flops": flops}
    return {"bytes": tokens * (2 * (hk + hv) * d * e + 4 * hv) + (2 if c["h0"] else 1) * n * state, "flops": flops}


# ---------------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """From the definitions: the recurrence token by token, its gradients by the chain rule backwards through the same steps,
    the norms as written above and theirs by differentiating the formulas."""
    s = prepare(case, seed)
    c = case
    if c["op"] == "gla_decode":
        share = torch.arange(c["hv"], device="cuda") // (c["hv"] // c["hk"])
        h = s["state"].double() * s["g"].double().exp()[:, :, None, None]
        h += torch.einsum("nhk,nhv->nhkv", s["k"].double()[:, share], s["v"].double())
        return {"o": torch.einsum("nhk,nhkv->nhv", s["q"].double()[:, share], h), "state": h}
    return _exact_gla(s) if c["op"] == "gla" else _exact_norm(s)


def _exact_gla(s):
    c, back, d, hk, hv = s, s["back"], s["d"], s["hk"], s["hv"]
    lens = torch.tensor(_lengths(c), device="cuda")
    N, longest = len(lens), int(lens.max())
    start = torch.cumsum(lens, 0) - lens
    flat = {x: s[x].reshape(-1, *s[x].shape[2:]).double() for x in ("q", "k", "v", "g", "do") if x in s}
    zeros = lambda x: torch.zeros_like(flat[x])              # noqa: E731
    out = {"dq": zeros("q"), "dk": zeros("k"), "dv": zeros("v"), "dg": zeros("g")} if back else {"o": zeros("v")}
    last = torch.zeros(N, hv, d, d, dtype=torch.float64, device="cuda")
    R = hv // hk
    many = hv if not back else max(R, int(16e9 / (N * longest * d * d * 8)) // R * R)   # V-heads at once: states kept for the way back
    for j0 in range(0, hv, many):
        j1 = min(hv, j0 + many)
        heads, of = slice(j0, j1), torch.arange(j0, j1, device="cuda") // R
        h = s["h0"][:, heads].double() if s["h0"] is not None else torch.zeros(N, j1 - j0, d, d, dtype=torch.float64, device="cuda")
        kept = []
        for t in range(longest):
            m = (t < lens).nonzero()[:, 0] if int(lens.min()) <= t else slice(None)
            i = (start + t)[m]
            if back:
                kept.append(h[m])
            new = flat["g"][i][:, heads].exp()[:, :, None, None] * h[m]
            new = torch.baddbmm(new.flatten(0, 1), flat["k"][i][:, of].reshape(-1, d, 1), flat["v"][i][:, heads].reshape(-1, 1, d)).view_as(new)
            h = new if isinstance(m, slice) else h.index_copy(0, m, new)
            if not back:
                out["o"][i, heads] = (flat["q"][i][:, of].unsqueeze(-2) @ new).squeeze(-2)
        if not back:
            last[:, heads] = h
            continue
        dh = s["dhT"][:, heads].double() if s["dhT"] is not None else torch.zeros_like(h)
        for t in reversed(range(longest)):
            m = (t < lens).nonzero()[:, 0] if int(lens.min()) <= t else slice(None)
            i = (start + t)[m]
            q, k, v, do = flat["q"][i][:, of], flat["k"][i][:, of], flat["v"][i][:, heads], flat["do"][i][:, heads]
            a = flat["g"][i][:, heads].exp()[:, :, None, None]
            was = kept.pop()
            now = a * was + k.unsqueeze(-1) * v.unsqueeze(-2)
            d1 = dh[m] + q.unsqueeze(-1) * do.unsqueeze(-2)
            out["dv"][i, heads] = (k.unsqueeze(-2) @ d1).squeeze(-2)
            dk, dq = (d1 @ v.unsqueeze(-1)).squeeze(-1), (now @ do.unsqueeze(-1)).squeeze(-1)
            out["dk"][i] += torch.zeros_like(flat["k"][i]).index_add_(1, of, dk)
            out["dq"][i] += torch.zeros_like(flat["q"][i]).index_add_(1, of, dq)
            d1 = d1 * a
            out["dg"][i, heads] = (d1 * was).sum((-1, -2))
            dh = d1 if isinstance(m, slice) else dh.index_copy(0, m, d1)
        last[:, heads] = dh
    for x in out:
        out[x] = out[x].reshape(s[x[-1] if x != "o" else "v"].shape)
    return {**out, ("dh0" if back else "hT"): last}


def _exact_norm(s):
    leaves = {x: s[x].double().requires_grad_(s["back"]) for x in ("x", "w", "z", "r", "w_post") if s.get(x) is not None}
    if not s["back"]:
        y, r = _exact_forward(s, leaves)
        return {"y": y} if r is None else {"y": y, "r": r}
    if s["op"] == "gated_norm":
        y, _ = _exact_forward(s, leaves)
        dx, dw, dz = torch.autograd.grad(y, [leaves["x"], leaves["w"], leaves["z"]], s["dy"].double())
        return {"dx": dx, "dw": dw, "dz": dz}
    # r is the stream behind the addition here: its own gradient goes to x by way of f alone
    y = leaves["r"] / (leaves["r"].square().mean(-1, keepdim=True) + EPS).sqrt() * leaves["w"]
    via, dw = torch.autograd.grad(y, [leaves["r"], leaves["w"]], s["dy"].double())
    dr = via + s["dr"].double()
    out = {"dr": dr, "dw": dw}
    f = s["scale"] * _exact_f(leaves)
    got = torch.autograd.grad(f, [leaves["x"]] + ([leaves["w_post"]] if s["post"] else []), dr)
    if s["post"]:
        out["dw_post"] = got[1]
    return {"dx": got[0], **out}


def _exact_f(t):
    x = t["x"]
    return x * t["w_post"] / (x.square().mean(-1, keepdim=True) + EPS).sqrt() if "w_post" in t else x * 1.0


def _exact_forward(s, t):
    if s["op"] == "add_norm":
        r = t["r"] + s["scale"] * _exact_f(t)
        return r / (r.square().mean(-1, keepdim=True) + EPS).sqrt() * t["w"], r
    a = 1 / (1 + torch.exp(-t["z"]))
    a = a * t["z"] if s["act"] == "silu" else a
    return t["x"] / (t["x"].square().mean(-1, keepdim=True) + EPS).sqrt() * t["w"] * a, None
