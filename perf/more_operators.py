"""The layers that alternate with delta-rule layers in a hybrid model, as cases that can be timed and compared.

Three operators, each for whole sequences and for single tokens:

  conv    short causal convolution per channel, in front of a recurrence: y_t = act(bias + sum_j w_j x_(t-K+1+j)), K = 2, 3, 4;
          forward, backward, one token on a state of the last K - 1 inputs
  scan    selective state space scan: step delta_t = softplus(dt_t + dt_bias) per channel, h <- e^(delta A) h + delta B_t x_t,
          y_t = (<C_t, h> + D x_t) silu(z_t); forward, backward, one token on the states
  latent  attention whose keys and values come of one latent vector a token.  Expanded, for prompts: q [192] against a head's
          key [128] and a positional key [64] that all heads share, values [128], causal.  Absorbed, for one to four new tokens a
          sequence: all heads' q [576] against the cached rows [512 + 64] themselves, whose first 512 are the values, in pages

Values: x, z, B, C, q and gradients ~ N(0, 1); dt ~ N(0, 0.5), dt_bias so that steps are 0.001 to 0.1 in the middle, A = -(1 .. S)
with some spread; latent rows ~ N(0, 1), and q of a size that gives scores of a standard deviation of about 2.  bf16 or fp32;
weights, A, D, dt_bias and the scan's states fp32.

`own` false: plain torch operations in 32 bits; `own` true: the library's entry points.
"""
import math
import random

import torch

own = False

LATENT, ROPE, NOPE, VALUE = 512, 64, 128, 128
BLOCK = 32                                                   # tokens whose decays the plain scan makes together


# ---------------------------------------------------------------------------------------------------------------- the cases

def _lens(rows=1, tokens=0, packed=0, lo=0, hi=0, len_seed=0):
    """`rows` sequences of `tokens` tokens each, or, with `packed` > 0, that many of lo..hi tokens end to end."""
    return dict(rows=rows, tokens=tokens, packed=packed, lo=lo, hi=hi, len_seed=len_seed)


def _named(name, c):
    return dict(c, name=name) if name else c


def _conv(name, form, channels, taps=4, dtype="bf16", act="silu", bias=False, h0=False, n=0, **lens):
    return _named(name, dict(op="conv", form=form, channels=channels, taps=taps, dtype=dtype, act=act, bias=bias, h0=h0, n=n, **_lens(**lens)))


def _scan(name, form, channels, states=16, groups=1, dtype="bf16", gate=True, skip=True, h0=False, n=0, **lens):
    return _named(name, dict(op="scan", form=form, channels=channels, states=states, groups=groups, dtype=dtype, gate=gate, skip=skip, h0=h0, n=n,
                             **_lens(**lens)))


def _latent(name, heads, dtype="bf16", past=0, **lens):
    """past: tokens of each sequence that are in front of the queries (a prompt that goes on from a cached beginning)."""
    return _named(name, dict(op="latent", form="prompt", heads=heads, dtype=dtype, past=past, **_lens(**lens)))


def _latent_token(name, n, heads, lo, hi, len_seed=0, new=1, page=64, dtype="bf16"):
    return _named(name, dict(op="latent", form="token", heads=heads, dtype=dtype, n=n, new=new, page=page, lo=lo, hi=hi, len_seed=len_seed))


def listed():
    return [
        # interactive decoding of one sequence, the q, k and v channels of 16 heads of 128: latency is all of it
        _conv("conv_token_n1", "token", 6144, n=1),
        # prompts end to end in front of a layer with 16 q/k heads and 32 v heads, each continued from a state
        _conv("conv_packed_8", "forward", 8192, packed=8, lo=512, hi=8192, len_seed=3, h0=True),
        # a training step, four rows of 4096 tokens, with a bias
        _conv("conv_back_b4_t4096", "backward", 4096, rows=4, tokens=4096, bias=True),
        # the decoding step of a full batch: 134 MB of states
        _scan("scan_token_n256", "token", 4096, n=256),
        # two short fp32 sequences, odd lengths and channels: a layer checked against a float64 reference
        _scan("scan_fp32_t257", "forward", 390, dtype="fp32", rows=2, tokens=257, h0=True),
        # a 4k prompt
        _scan("scan_t4096", "forward", 4096, tokens=4096),
        # a batch of prompts of very uneven lengths, each continued from a state
        _scan("scan_packed_8", "forward", 4096, packed=8, lo=100, hi=8000, len_seed=9, h0=True),
        # a training step: two rows of 2048 tokens
        _scan("scan_back_b2_t2048", "backward", 4096, rows=2, tokens=2048),
        # one short ragged prompt
        _latent("latent_t333", 16, tokens=333),
        # a long prompt, 32 heads
        _latent("latent_t8192", 32, tokens=8192),
        # interactive decoding on a long context: one sequence, split over the whole chip
        _latent_token("latent_token_n1", 1, 16, 20011, 20011),
        # the decoding step of a full batch of uneven contexts
        _latent_token("latent_token_n64", 64, 32, 500, 16000, len_seed=7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _draw_lens(rng, top):
    """Sequences of `top` tokens in all at the most."""
    if rng.random() < 0.5:
        n = _log_int(rng, 2, 24)
        hi = max(16, top // n)
        return dict(packed=n, lo=rng.choice([1, max(1, hi // 8)]), hi=hi, len_seed=rng.randrange(1 << 20))
    rows = rng.choice([1, 1, 2, 4])
    return dict(rows=rows, tokens=_log_int(rng, 1, max(1, top // rows)))


def draw(rng):
    kind = rng.random()
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind < 0.3:
        form = rng.choice(["token", "forward", "backward"])
        channels = rng.choice([2048, 4096, 6144, 8192, rng.randint(100, 6000)])
        c = dict(taps=rng.choice([4, 4, 3, 2]), dtype=dtype, act=rng.choice(["silu", "silu", "none"]), bias=rng.random() < 0.5)
        if form == "token":
            return _conv(None, form, channels, n=_log_int(rng, 1, 256), **c)
        return _conv(None, form, channels, h0=rng.random() < 0.5, **c, **_draw_lens(rng, min(32768, (1 << 26) // channels)))
    if kind < 0.65:
        form = rng.choice(["token", "forward", "forward", "backward"])
        states = rng.choice([16, 16, 16, 8, 32, 64, rng.randint(5, 40)])
        channels = rng.choice([1024, 2048, 4096, rng.randint(60, 3000)])
        groups = rng.choice([1, 1, 2, 4]) if channels % 4 == 0 else 1
        c = dict(states=states, groups=groups, dtype=dtype, gate=rng.random() < 0.7, skip=rng.random() < 0.7)
        if form == "token":
            return _scan(None, form, channels, n=_log_int(rng, 1, (1 << 24) // (channels * states)), **c)
        top = min(8192, (1 << (28 if form == "backward" else 30)) // (channels * states))
        return _scan(None, form, channels, h0=rng.random() < 0.5, **c, **_draw_lens(rng, top))
    if kind < 0.82:
        heads = rng.choice([1, 4, 8, 16, 32])
        top = 8192 if dtype == "bf16" else 512
        past = rng.choice([0, 0, _log_int(rng, 1, 2048 if dtype == "bf16" else 200)])
        return _latent(None, heads, dtype=dtype, past=past, **_draw_lens(rng, top if not past else top // 4))
    heads = rng.choice([8, 16, 32, 64, 128])
    n = _log_int(rng, 1, 64)
    hi = _log_int(rng, 16, min(16000, 500000 // n) * 32 // max(32, heads)) if dtype == "bf16" else _log_int(rng, 16, 3000 // n + 16)
    return _latent_token(None, n, heads, rng.choice([1, max(1, hi // 16), hi]), hi, len_seed=rng.randrange(1 << 20), new=rng.choice([1, 1, 1, 2, 4]),
                         page=rng.choice([16, 32, 64, 64, 128]), dtype=dtype)


# ---------------------------------------------------------------------------------------------------------------- the inputs

def _lengths(c):
    if c.get("packed"):
        r = random.Random(c["len_seed"])
        return [r.randint(c["lo"], c["hi"]) for _ in range(c["packed"])]
    return [c["tokens"]] * c["rows"]


def _contexts(c):
    r = random.Random(c["len_seed"])
    return [max(c["new"], r.randint(c["lo"], c["hi"])) for _ in range(c["n"])]


def _ends(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)

    s = dict(c)
    if c["op"] == "latent":
        return _prepare_token(c, s, normal, gen, dt) if c["form"] == "token" else _prepare_prompt(c, s, normal, dt)
    token = c["form"] == "token"
    lens = [1] * c["n"] if token else _lengths(c)
    N, ch = len(lens), c["channels"]
    lead = (c["n"],) if token else (1, sum(lens)) if c["packed"] else (c["rows"], c["tokens"])
    s["cu_seqlens"], s["max_seqlen"] = None, 0
    if not token:
        if c["packed"]:
            s["cu_seqlens"], s["max_seqlen"] = _ends(lens), max(lens)
        s["lens"] = torch.tensor(lens, device="cuda")
        s["start"] = torch.cumsum(s["lens"], 0) - s["lens"]
        s["longest"] = max(lens)
        s["seq"] = torch.repeat_interleave(torch.arange(N, device="cuda"), s["lens"])
        s["pos"] = torch.arange(sum(lens), device="cuda") - s["start"][s["seq"]]
    s["x"] = normal(*lead, ch).to(dt)
    back = c["form"] == "backward"
    if back:
        s["dy"] = normal(*lead, ch).to(dt)
    if c["op"] == "conv":
        K = c["taps"]
        s["w"] = normal(ch, K, std=K ** -0.5)
        s["bias"] = normal(ch, std=0.1) if c["bias"] else None
        s["state"] = normal(N, K - 1, ch).to(dt) if token else None
        s["h0"] = normal(N, K - 1, ch).to(dt) if c["h0"] else None
        s["dhT"] = normal(N, K - 1, ch).to(dt) if back and c["h0"] else None
        return s
    S, G = c["states"], c["groups"]
    s["dt"] = normal(*lead, ch, std=0.5).to(dt)
    step = torch.exp(torch.rand(ch, generator=gen, device="cuda") * math.log(100.0) + math.log(0.001))
    s["dt_bias"] = torch.log(torch.expm1(step))
    s["A"] = -torch.arange(1, S + 1, device="cuda", dtype=torch.float32) * torch.exp(normal(ch, S, std=0.1))
    s["B"], s["C"] = normal(*lead, G, S).to(dt), normal(*lead, G, S).to(dt)
    s["D"] = 1 + normal(ch, std=0.1) if c["skip"] else None
    s["z"] = normal(*lead, ch).to(dt) if c["gate"] else None
    s["state"] = normal(N, ch, S, std=0.5) if token else None
    s["h0"] = normal(N, ch, S, std=0.5) if c["h0"] else None
    s["dhT"] = normal(N, ch, S, std=0.5) if back and c["h0"] else None
    return s


def _prepare_prompt(c, s, normal, dt):
    lens, past, H = _lengths(c), c["past"], c["heads"]
    full = [n + past for n in lens]
    rows = (1, sum(lens)) if c["packed"] else (c["rows"], c["tokens"])
    keys = (1, sum(full)) if c["packed"] else (c["rows"], c["tokens"] + past)
    s["q"] = normal(*rows, H, NOPE + ROPE, std=2.0).to(dt)
    # a head's key and value of one token lie side by side, as the product that expands the latent rows leaves them
    s["kv"] = normal(*keys, H, NOPE + VALUE).to(dt)
    s["kr"] = normal(*keys, ROPE).to(dt)
    s["scale"] = (NOPE + ROPE) ** -0.5
    s["cu_seqlens"] = s["cu_seqlens_k"] = None
    s["max_seqlen"] = 0
    if c["packed"]:
        s["cu_seqlens"], s["cu_seqlens_k"], s["max_seqlen"] = _ends(lens), _ends(full), max(lens)
    s["lens"] = lens
    return s


def _prepare_token(c, s, normal, gen, dt):
    lens, page = _contexts(c), c["page"]
    s["q"] = normal(c["n"], c["new"], c["heads"], LATENT + ROPE, std=2.0).to(dt)
    s["scale"] = (LATENT + ROPE) ** -0.5
    need = [-(-n // page) for n in lens]
    # pages of all sequences lie mixed in the cache
    order = torch.randperm(sum(need) + 3, generator=gen, device="cuda")[:sum(need)].to(torch.int32)
    s["page_table"] = torch.zeros(c["n"], max(need), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        s["page_table"][i, :n] = order[at:at + n]
        at += n
    s["cache"] = normal(sum(need) + 3, page, LATENT + ROPE).to(dt)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["longest"] = max(lens)
    return s


# ---------------------------------------------------------------------------------------------------------------- one pass

def run(s):
    return (_OWN if own else _PLAIN)[s["op"], s["form"]](s)


# ... by the library

def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def _act(s):
    return None if s["act"] == "none" else s["act"]


def _own_conv_token(s):
    """To another state, so that every pass starts from the same one; that buffer is kept."""
    if "state_out" not in s:
        s["state_out"] = torch.empty_like(s["state"])
    y, state = _ha().ha_la_conv_decode(s["x"], s["w"], s["state"], bias=s["bias"], activation=_act(s), state_out=s["state_out"])
    return {"y": y, "state": state}


def _own_conv(s):
    y, hT, s["status_word"] = _ha().ha_la_conv(s["x"], s["w"], bias=s["bias"], activation=_act(s), h0=s["h0"], cu_seqlens=s["cu_seqlens"],
                                               max_seqlen=s["max_seqlen"], status_word=s.get("status_word"))
    return {"y": y, "hT": hT}


def _own_conv_back(s):
    dx, dw, db, dh0, s["status_word"], s["workspace"] = _ha().ha_la_conv_backward(
        s["dy"], s["x"], s["w"], bias=s["bias"], activation=_act(s), h0=s["h0"], dhT=s["dhT"], cu_seqlens=s["cu_seqlens"],
        max_seqlen=s["max_seqlen"], status_word=s.get("status_word"), workspace=s.get("workspace"))
    return {"dx": dx, "dw": dw, "dh0": dh0, **({"db": db} if s["bias"] is not None else {})}


def _own_scan_token(s):
    if "state_out" not in s:
        s["state_out"] = torch.empty_like(s["state"])
    y, state = _ha().ha_la_scan_decode(s["x"], s["dt"], s["A"], s["B"], s["C"], s["state"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"],
                                       state_out=s["state_out"])
    return {"y": y, "state": state}


def _own_scan(s):
    """The scratch workspace and the status word are kept from call to call, as a serving program does."""
    y, hT, s["status_word"], s["workspace"] = _ha().ha_la_scan(
        s["x"], s["dt"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], h0=s["h0"], cu_seqlens=s["cu_seqlens"],
        max_seqlen=s["max_seqlen"], status_word=s.get("status_word"), workspace=s.get("workspace"))
    return {"y": y, "hT": hT}


def _own_scan_back(s):
    dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0, s["status_word"], s["workspace"] = _ha().ha_la_scan_backward(
        s["dy"], s["x"], s["dt"], s["A"], s["B"], s["C"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], h0=s["h0"], dhT=s["dhT"],
        cu_seqlens=s["cu_seqlens"], max_seqlen=s["max_seqlen"], status_word=s.get("status_word"), workspace=s.get("workspace"))
    return {"dx": dx, "ddt": ddt, "dA": dA, "dB": dB, "dC": dC, "ddt_bias": ddt_bias, "dh0": dh0,
            **({"dD": dD} if s["skip"] else {}), **({"dz": dz} if s["gate"] else {})}


def _own_prompt(s):
    o, lse, s["status_word"] = _ha().ha_la_latent_prefill(
        s["q"], s["kv"][..., :NOPE], s["kr"], s["kv"][..., NOPE:], scale=s["scale"], cu_seqlens=s["cu_seqlens"], cu_seqlens_k=s["cu_seqlens_k"],
        max_seqlen=s["max_seqlen"], status_word=s.get("status_word"))
    return {"o": o, "lse": lse}


def _own_token(s):
    o, lse, s["status_word"], s["workspace"] = _ha().ha_la_latent_decode(
        s["q"], s["cache"], s["page_table"], s["lengths"], scale=s["scale"], status_word=s.get("status_word"), workspace=s.get("workspace"))
    return {"o": o, "lse": lse}


# ... in plain operations

def _silu(z):
    return z * torch.sigmoid(z)


def _plain_conv_token(s):
    x = torch.cat([s["state"], s["x"][:, None]], 1).float()  # [N, K, channels], oldest first
    y = (x * s["w"].T).sum(1)
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": (_silu(y) if s["act"] == "silu" else y).to(s["x"].dtype), "state": x[:, 1:].to(s["x"].dtype)}


def _back_by(s, x, j):
    """The inputs j tokens in front of each one, [tokens, channels]; from h0, or zeros, in front of a sequence."""
    y = torch.roll(x, j, 0)
    first = (s["pos"] < j).nonzero()[:, 0]
    if s["h0"] is None:
        y[first] = 0
    else:
        y[first] = s["h0"][s["seq"][first], s["taps"] - 1 + s["pos"][first] - j].float()
    return y


def _tail(s, x):
    """The last K - 1 inputs of each sequence."""
    K, N = s["taps"], len(s["lens"])
    i = torch.arange(K - 1, device="cuda")
    at = s["lens"][:, None] - (K - 1) + i
    new = x[(s["start"][:, None] + at).clamp_min(0).clamp_max(len(x) - 1)]
    old = torch.zeros(N, K - 1, x.shape[-1], device="cuda") if s["h0"] is None else s["h0"].float()
    old = torch.gather(old, 1, (at + K - 1).clamp_max(K - 2)[..., None].expand_as(old))
    return torch.where((at >= 0)[..., None], new, old)


def _before_act(s, x):
    K = s["taps"]
    y = sum(_back_by(s, x, K - 1 - j) * s["w"][:, j] for j in range(K))
    return y if s["bias"] is None else y + s["bias"]


def _plain_conv(s):
    x = s["x"].reshape(-1, s["channels"]).float()
    y = _before_act(s, x)
    return {"y": (_silu(y) if s["act"] == "silu" else y).to(s["x"].dtype).reshape(s["x"].shape), "hT": _tail(s, x).to(s["x"].dtype)}


def _plain_conv_back(s):
    K, N, dt = s["taps"], len(s["lens"]), s["x"].dtype
    x, d = s["x"].reshape(-1, s["channels"]).float(), s["dy"].reshape(-1, s["channels"]).float()
    if s["act"] == "silu":
        y = _before_act(s, x)
        e = torch.sigmoid(y)
        d = d * e * (1 + y * (1 - e))
    dw = torch.stack([(d * _back_by(s, x, K - 1 - j)).double().sum(0).float() for j in range(K)], 1)
    # with K - 1 places in front of each sequence for the state's gradient
    at = s["start"][s["seq"]] + (s["seq"] + 1) * (K - 1) + s["pos"]
    full = torch.zeros(len(x) + N * (K - 1), x.shape[1], device="cuda")
    for j in range(K):
        full[at - (K - 1 - j)] += d * s["w"][:, j]
    ends = s["start"] + s["lens"] + (torch.arange(N, device="cuda") + 1) * (K - 1)
    if s["dhT"] is not None:
        for i in range(K - 1):
            full[ends - (K - 1) + i] += s["dhT"][:, i].float()
    front = (s["start"] + torch.arange(N, device="cuda") * (K - 1))[:, None] + torch.arange(K - 1, device="cuda")
    out = {"dx": full[at].to(dt).reshape(s["x"].shape), "dw": dw, "dh0": full[front].to(dt)}
    return out if s["bias"] is None else {**out, "db": d.double().sum(0).float()}


def _steps(s):
    """softplus(dt + bias) and its slope."""
    v = s["dt"].float() + s["dt_bias"]
    return torch.clamp_min(v, 0) + torch.log1p(torch.exp(-v.abs())), torch.sigmoid(v)


def _wide(s, b):
    """[.., groups, S] for each channel: [.., channels, S]."""
    return b.float().repeat_interleave(s["channels"] // s["groups"], -2)


def _plain_scan_token(s):
    x, (delta, _) = s["x"].float(), _steps(s)
    h = torch.exp(delta[..., None] * s["A"]) * s["state"] + (delta * x)[..., None] * _wide(s, s["B"])
    y = (h * _wide(s, s["C"])).sum(-1)
    if s["skip"]:
        y = y + s["D"] * x
    return {"y": (y * _silu(s["z"].float()) if s["gate"] else y).to(s["x"].dtype), "state": h}


def _flat(s, x):
    return x.reshape(-1, *x.shape[2:])


def _at(s, t, n):
    """Rows of the n tokens from position t on of each sequence, and which of them there are: [sequences, n]."""
    p = t + torch.arange(n, device="cuda")
    return (s["start"][:, None] + p).clamp_max(len(s["seq"]) - 1), p < s["lens"][:, None]


def _zeros_like_state(s):
    return torch.zeros(len(s["lens"]), s["channels"], s["states"], device="cuda")


def _plain_scan(s, keep=None):
    """The recurrence, blocks of tokens for the decays, token by token for the states, all sequences together."""
    x, delta = _flat(s, s["x"]).float(), _flat(s, _steps(s)[0])
    B, C = _flat(s, s["B"]), _flat(s, s["C"])
    h = _zeros_like_state(s) if s["h0"] is None else s["h0"].clone()
    y = torch.zeros_like(x)
    for t in range(0, s["longest"], BLOCK):
        n = min(BLOCK, s["longest"] - t)
        at, there = _at(s, t, n)
        d = delta[at] * there[..., None]                     # (no step where there is no token: the state stays)
        decay = torch.exp(d[..., None] * s["A"])
        add = (d * x[at])[..., None] * _wide(s, B[at])
        hs = torch.empty_like(decay)
        for i in range(n):
            h = decay[:, i] * h + add[:, i]
            hs[:, i] = h
        if keep is not None:
            keep.append((decay, hs))
        y[at[there]] = (hs * _wide(s, C[at])).sum(-1)[there]
    if s["skip"]:
        y = y + s["D"] * x
    if keep is not None:
        return y
    if s["gate"]:
        y = y * _silu(_flat(s, s["z"]).float())
    return {"y": y.to(s["x"].dtype).reshape(s["x"].shape), "hT": h}


def _plain_scan_back(s):
    keep = []
    y = _plain_scan(s, keep)
    dt, ch, S, G = s["x"].dtype, s["channels"], s["states"], s["groups"]
    x, dy = _flat(s, s["x"]).float(), _flat(s, s["dy"]).float()
    delta, slope = (_flat(s, e) for e in _steps(s))
    B, C = _flat(s, s["B"]), _flat(s, s["C"])
    out = {}
    if s["gate"]:
        z = _flat(s, s["z"]).float()
        e = torch.sigmoid(z)
        out["dz"] = (dy * y * e * (1 + z * (1 - e))).to(dt).reshape(s["x"].shape)
        dy = dy * z * e
    dx = torch.zeros_like(x)
    if s["skip"]:
        out["dD"] = (dy * x).double().sum(0).float()
        dx += dy * s["D"]
    ddelta = torch.zeros_like(x)
    dB, dC = torch.zeros(len(x), G, S, device="cuda"), torch.zeros(len(x), G, S, device="cuda")
    dA = torch.zeros(ch, S, dtype=torch.float64, device="cuda")
    dh = _zeros_like_state(s) if s["dhT"] is None else s["dhT"].clone()
    first = _zeros_like_state(s) if s["h0"] is None else s["h0"]
    per_group = lambda e: e.reshape(*e.shape[:-2], G, ch // G, S).sum(-2)    # noqa: E731
    for t in reversed(range(0, s["longest"], BLOCK)):
        decay, hs = keep.pop()
        n = hs.shape[1]
        at, there = _at(s, t, n)
        before = torch.cat([(keep[-1][1][:, -1] if keep else first)[:, None], hs[:, :-1]], 1)
        give = (dy[at] * there[..., None])[..., None] * _wide(s, C[at])
        dhs = torch.empty_like(hs)
        for i in reversed(range(n)):
            dh = dh + give[:, i]
            dhs[:, i] = dh
            dh = dh * decay[:, i]
        dhs = dhs * there[..., None, None]
        flow = dhs * decay * before                          # gradient of delta A
        here = at[there]
        u = (dhs * _wide(s, B[at])).sum(-1)                  # ... of delta x
        ddelta[here] = ((flow * s["A"]).sum(-1) + u * x[at])[there]
        dx[here] += (u * delta[at])[there]
        dA += (flow * delta[at][..., None]).sum(1).double().sum(0)
        dB[here] = per_group(dhs * (delta[at] * x[at])[..., None])[there]
        dC[here] = per_group(hs * dy[at][..., None])[there]
    ddt = ddelta * slope
    out.update(dx=dx.to(dt).reshape(s["x"].shape), ddt=ddt.to(dt).reshape(s["x"].shape), dA=dA.float(), dB=dB.to(dt).reshape(s["B"].shape),
               dC=dC.to(dt).reshape(s["C"].shape), ddt_bias=ddt.double().sum(0).float(), dh0=dh)
    return out


def _softmax(scores, there):
    """Of the last dimension's places that are there: weights and the logarithm of their sum; zeros and -inf where none is."""
    scores = scores.masked_fill(~there, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    e = torch.exp(scores - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    return e / total.clamp_min(1e-37), lse


def _plain_prompt(s):
    H, past = s["heads"], s["past"]
    q, kv, kr = (_flat(s, s[x]) for x in ("q", "kv", "kr"))
    o = torch.empty(len(q), H, VALUE, dtype=q.dtype, device="cuda")
    lse = torch.empty(len(q), H, device="cuda")
    a = b = 0
    for n in s["lens"]:
        m = n + past
        there = torch.arange(m, device="cuda") <= torch.arange(n, device="cuda")[:, None] + past
        for h in range(H):
            k = torch.cat([kv[b:b + m, h, :NOPE], kr[b:b + m]], -1).float()
            p, lse[a:a + n, h] = _softmax(q[a:a + n, h].float() @ k.T * s["scale"], there)
            o[a:a + n, h] = (p @ kv[b:b + m, h, NOPE:].float()).to(q.dtype)
        a, b = a + n, b + m
    return {"o": o.reshape(*s["q"].shape[:-1], VALUE), "lse": lse.reshape(s["q"].shape[:-1])}


def _plain_token(s):
    N, new, H = s["n"], s["new"], s["heads"]
    pos = torch.arange(s["longest"], device="cuda")
    at = s["page_table"].long()[:, pos // s["page"]] * s["page"] + pos % s["page"]
    limit = s["lengths"][:, None] - new + torch.arange(new, device="cuda")   # last position that a new token sees
    there = (pos <= limit[..., None])[:, :, None]
    rows = s["cache"].reshape(-1, LATENT + ROPE)
    o = torch.empty(N, new, H, LATENT, dtype=s["q"].dtype, device="cuda")
    lse = torch.empty(N, new, H, device="cuda")
    for n in range(0, N, 8):                                 # eight sequences at once
        kv = rows[at[n:n + 8]].float()
        scores = torch.einsum("nihd,ntd->niht", s["q"][n:n + 8].float(), kv) * s["scale"]
        p, lse[n:n + 8] = _softmax(scores, there[n:n + 8])
        o[n:n + 8] = torch.einsum("niht,ntd->nihd", p, kv[..., :LATENT]).to(o.dtype)
    return {"o": o, "lse": lse}


_OWN = {("conv", "token"): _own_conv_token, ("conv", "forward"): _own_conv, ("conv", "backward"): _own_conv_back,
        ("scan", "token"): _own_scan_token, ("scan", "forward"): _own_scan, ("scan", "backward"): _own_scan_back,
        ("latent", "prompt"): _own_prompt, ("latent", "token"): _own_token}
_PLAIN = {("conv", "token"): _plain_conv_token, ("conv", "forward"): _plain_conv, ("conv", "backward"): _plain_conv_back,
          ("scan", "token"): _plain_scan_token, ("scan", "forward"): _plain_scan, ("scan", "backward"): _plain_scan_back,
          ("latent", "prompt"): _plain_prompt, ("latent", "token"): _plain_token}


# ---------------------------------------------------------------------------------------------------------------- how much work

def work(case):
    """Each input read once, each output written once; multiply-adds counted as two operations, an exponential as one."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "latent":
        H = c["heads"]
        if c["form"] == "token":
            lens, rows = _contexts(c), c["n"] * c["new"] * H
            seen = sum(sum(n - i for i in range(c["new"])) for n in lens)
            return {"bytes": sum(lens) * (LATENT + ROPE) * e + rows * ((2 * LATENT + ROPE) * e + 4), "flops": 2.0 * H * seen * (2 * LATENT + ROPE)}
        lens = _lengths(c)
        seen = sum(n * c["past"] + n * (n + 1) // 2 for n in lens)
        q, k = sum(lens), sum(lens) + len(lens) * c["past"]
        return {"bytes": e * (q * H * (NOPE + ROPE + VALUE) + k * (H * (NOPE + VALUE) + ROPE)) + 4 * q * H,
                "flops": 2.0 * H * seen * (NOPE + ROPE + VALUE)}
    token, back, ch = c["form"] == "token", c["form"] == "backward", c["channels"]
    N = c["n"] if token else len(_lengths(c))
    tokens = N if token else sum(_lengths(c))
    if c["op"] == "conv":
        K = c["taps"]
        states = 2 if token else 1 + c["h0"] + (back and c["h0"])
        return {"bytes": e * ch * (tokens * (3 if back else 2) + states * N * (K - 1)) + 4 * ch * (K + c["bias"]) * (1 + back),
                "flops": float(tokens) * ch * (2 * K + 4) * (3 if back else 1)}
    S, G = c["states"], c["groups"]
    states = 2 if token else 1 + c["h0"] + (back and c["h0"])
    streams = (5 + 2 * c["gate"]) if back else 3 + c["gate"]
    return {"bytes": e * tokens * (ch * streams + 2 * G * S * (2 if back else 1)) + 4 * states * N * ch * S + 4 * ch * (S + 1 + c["skip"]) * (1 + back),
            "flops": float(tokens) * ch * S * (18 if back else 7)}


# ---------------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """From the definitions in 64 bits: convolutions over padded sequences and the recurrences token by token, their gradients by
    differentiating these, attention row by row."""
    s = prepare(case, seed)
    if s["op"] == "latent":
        return _exact_token(s) if s["form"] == "token" else _exact_prompt(s)
    if s["op"] == "conv":
        return _exact_conv(s)
    if s["form"] == "token":
        h, y = _exact_step(s, s["state"].double(), s["x"].double(), s["dt"].double(), s["B"].double(), s["C"].double(),
                           s["z"].double() if s["gate"] else None)
        return {"y": y, "state": h}
    return _exact_scan_back(s) if s["form"] == "backward" else _exact_scan(s)


def _exact_conv(s):
    K, ch, act = s["taps"], s["channels"], s["act"] == "silu"
    back = s["form"] == "backward"
    w = s["w"].double().requires_grad_(back)
    bias = s["bias"].double().requires_grad_(back) if s["bias"] is not None else None

    def apply(front, x):
        """front [.., K - 1, channels], x [.., T, channels]"""
        full = torch.cat([front, x], -2)
        y = full.unfold(-2, K, 1).mul(w).sum(-1)
        y = y if bias is None else y + bias
        return (y / (1 + torch.exp(-y)) if act else y), full[..., full.shape[-2] - (K - 1):, :]

    if s["form"] == "token":
        y, state = apply(s["state"].double(), s["x"].double()[:, None])
        return {"y": y[:, 0], "state": state}
    lens = s["lens"].tolist()
    x = s["x"].reshape(-1, ch)
    fronts, ys, lasts = [], [], []
    gx, gf = [], []
    dw, db = 0, 0
    at = 0
    for n, m in enumerate(lens):
        front = (s["h0"][n].double() if s["h0"] is not None else torch.zeros(K - 1, ch, dtype=torch.float64, device="cuda")).requires_grad_(back)
        xs = x[at:at + m].double().requires_grad_(back)
        y, last = apply(front, xs)
        if back:
            ends, grads = [y], [s["dy"].reshape(-1, ch)[at:at + m].double()]
            if s["dhT"] is not None:
                ends, grads = [y, last], [grads[0], s["dhT"][n].double()]
            got = torch.autograd.grad(ends, [xs, front, w] + ([bias] if bias is not None else []), grads)
            gx.append(got[0])
            gf.append(got[1])
            dw = dw + got[2]
            db = db + got[3] if bias is not None else 0
        else:
            ys.append(y)
            lasts.append(last)
        fronts.append(front)
        at += m
    if back:
        out = {"dx": torch.cat(gx).reshape(s["x"].shape), "dw": dw, "dh0": torch.stack(gf)}
        return out if bias is None else {**out, "db": db}
    return {"y": torch.cat(ys).reshape(s["x"].shape), "hT": torch.stack(lasts)}


def _exact_step(s, h, x, dt, B, C, z):
    """One token of each of the rows of h [n, channels, S]: the new states and outputs."""
    r, A = s["channels"] // s["groups"], s["A"].double()
    v = dt + s["dt_bias"].double()
    delta = torch.where(v > 40, v, torch.log1p(torch.exp(v.clamp_max(40))))
    g = torch.arange(s["channels"], device="cuda") // r
    h = torch.exp(delta.unsqueeze(-1) * A) * h + (delta * x).unsqueeze(-1) * B[:, g]
    y = torch.einsum("ncs,ncs->nc", h, C[:, g])
    if s["skip"]:
        y = y + s["D"].double() * x
    return h, y if z is None else y * z / (1 + torch.exp(-z))


def _exact_rows(s, t):
    """Which sequences have a token t, and its row."""
    m = (s["lens"] > t).nonzero()[:, 0]
    return m, (s["start"] + t)[m]


def _exact_scan(s):
    f = {k: _flat(s, s[k]) for k in ("x", "dt", "B", "C", "z") if s[k] is not None}
    h = _zeros_like_state(s).double() if s["h0"] is None else s["h0"].double()
    y = torch.zeros(f["x"].shape, dtype=torch.float64, device="cuda")
    for t in range(s["longest"]):
        m, i = _exact_rows(s, t)
        new, y[i] = _exact_step(s, h[m], *(f[k][i].double() for k in ("x", "dt", "B", "C")), f["z"][i].double() if s["gate"] else None)
        h = h.index_copy(0, m, new)
    return {"y": y.reshape(s["x"].shape), "hT": h}


def _exact_scan_back(s):
    """Backwards through one token after another, each step differentiated by itself."""
    names = ["x", "dt", "B", "C"] + (["z"] if s["gate"] else [])
    f = {k: _flat(s, s[k]) for k in names + ["dy"]}
    weights = {k: s[k] for k in ("A", "dt_bias", "D") if s[k] is not None}
    if s["longest"] > 4096 or s["longest"] * len(s["lens"]) * s["channels"] * s["states"] > 1 << 30:
        return None
    h = _zeros_like_state(s).double() if s["h0"] is None else s["h0"].double()
    kept = []
    for t in range(s["longest"]):
        m, i = _exact_rows(s, t)
        kept.append(h[m])
        new, _ = _exact_step(s, h[m], *(f[k][i].double() for k in ("x", "dt", "B", "C")), None)
        h = h.index_copy(0, m, new)
    dh = torch.zeros_like(h) if s["dhT"] is None else s["dhT"].double()
    grads = {k: torch.zeros(f[k].shape, dtype=torch.float64, device="cuda") for k in names}
    sums = {k: torch.zeros(v.shape, dtype=torch.float64, device="cuda") for k, v in weights.items()}
    for t in reversed(range(s["longest"])):
        m, i = _exact_rows(s, t)
        was = kept.pop().requires_grad_()
        leaf = {k: f[k][i].double().requires_grad_() for k in names}
        v = {k: e.double().requires_grad_() for k, e in weights.items()}
        with torch.enable_grad():
            new, y = _exact_step({**s, **v}, was, leaf["x"], leaf["dt"], leaf["B"], leaf["C"], leaf.get("z"))
            got = torch.autograd.grad([new, y], [was, *leaf.values(), *v.values()], [dh[m], f["dy"][i].double()])
        dh = dh.index_copy(0, m, got[0])
        for k, e in zip(names, got[1:]):
            grads[k][i] = e
        for k, e in zip(v, got[1 + len(names):]):
            sums[k] += e
    out = {"d" + k: grads[k].reshape(s[k].shape) for k in names}
    out.update({"d" + k: e for k, e in sums.items()}, dh0=dh)
    return out


def _exact_prompt(s):
    H, past = s["heads"], s["past"]
    if sum(n * (n + past) for n in s["lens"]) * H > 1 << 33:
        return None
    q, kv, kr = (_flat(s, s[x]) for x in ("q", "kv", "kr"))
    o = torch.zeros(len(q), H, VALUE, dtype=torch.float64, device="cuda")
    lse = torch.full((len(q), H), -math.inf, dtype=torch.float64, device="cuda")
    a = b = 0
    for n in s["lens"]:
        m = n + past
        shared = kr[b:b + m].double()
        for h in range(H):
            k, v = kv[b:b + m, h, :NOPE].double(), kv[b:b + m, h, NOPE:].double()
            for i in range(0, n, 1024):                      # rows i .. j see the first past + j keys at the most
                j = min(n, i + 1024)
                e = q[a + i:a + j, h].double()
                w = (e[:, :NOPE] @ k[:past + j].T + e[:, NOPE:] @ shared[:past + j].T) * s["scale"]
                w += torch.full_like(w, -math.inf).triu(past + i + 1)
                lse[a + i:a + j, h] = torch.logsumexp(w, -1)
                o[a + i:a + j, h] = torch.exp(w - lse[a + i:a + j, h, None]) @ v[:past + j]
        a, b = a + n, b + m
    return {"o": o.reshape(*s["q"].shape[:-1], VALUE), "lse": lse.reshape(s["q"].shape[:-1])}


def _exact_token(s):
    N, new, H = s["n"], s["new"], s["heads"]
    o = torch.zeros(N, new, H, LATENT, dtype=torch.float64, device="cuda")
    lse = torch.full((N, new, H), -math.inf, dtype=torch.float64, device="cuda")
    for n, length in enumerate(s["lengths"].tolist()):
        pages = s["page_table"][n, :-(-length // s["page"])].long()
        rows = s["cache"][pages].reshape(-1, LATENT + ROPE).double()
        for i in range(new):
            see = rows[:length - new + 1 + i]
            w = s["q"][n, i].double() @ see.T * s["scale"]
            lse[n, i] = torch.logsumexp(w, -1)
            o[n, i] = torch.exp(w - lse[n, i, :, None]) @ see[:, :LATENT]
    return {"o": o, "lse": lse}
