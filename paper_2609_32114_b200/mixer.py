"""Binding of the layers that alternate with the recurrences in a hybrid model (include/ha_la.h): short causal convolution, selective
state space scan, forward, backward and one token.

As in `layer`: marshalling only, torch CUDA tensors in and out, everything is computed by the library's kernels on the caller's
stream, nothing is synchronised, tensors whose type, layout, size or device does not fit raise ValueError before anything is launched,
and nothing is recorded for autograd.  Inputs with one row to a token may be rows of a wider tensor (slices of a fused projection's
output along the last dimension); outputs are contiguous.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import HA_LA_OK, HaLaError, _aligned_part, _check_room, _reachable
from .layer import _INT32_MAX, _On, _as, _bound, _cuda, _element, _ptr, _sizes

HA_LA_ACT_SILU, HA_LA_ACT_NONE = 0, 2
_ACTIVATIONS = {"silu": HA_LA_ACT_SILU, None: HA_LA_ACT_NONE}

_p, _i, _l = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class ha_la_conv_args(ctypes.Structure):
    _fields_ = [
        *((n, _i) for n in ("dtype", "batch", "seqlen", "channels", "taps", "activation")), ("x_stride", _l),
        *((n, _p) for n in ("x", "w", "bias", "h0", "cu_seqlens")), ("num_seqs", _i), ("max_seqlen", _i),
        *((n, _p) for n in ("y", "hT", "dy", "dhT", "dx", "dw", "db", "dh0", "workspace")), ("workspace_bytes", ctypes.c_size_t), ("status_word", _p),
    ]


class ha_la_scan_args(ctypes.Structure):
    _fields_ = [
        *((n, _i) for n in ("dtype", "batch", "seqlen", "channels", "states", "groups", "softplus", "num_seqs", "max_seqlen")), ("cu_seqlens", _p),
        *((n, _l) for n in ("x_stride", "dt_stride", "b_stride", "c_stride", "z_stride")),
        *((n, _p) for n in ("x", "dt", "B", "C", "z", "A", "D", "dt_bias", "h0", "y", "hT", "dy", "dhT", "dx", "ddt", "dB", "dC", "dz", "dA", "dD",
                            "ddt_bias", "dh0", "workspace")), ("workspace_bytes", ctypes.c_size_t), ("status_word", _p),
    ]


_STRUCTS = {"ha_la_conv": ha_la_conv_args, "ha_la_conv_backward": ha_la_conv_args, "ha_la_conv_decode": ha_la_conv_args,
            "ha_la_scan": ha_la_scan_args, "ha_la_scan_backward": ha_la_scan_args, "ha_la_scan_decode": ha_la_scan_args}


def declare(lib) -> None:
    """Argument and result types of the entry points, for ctypes."""
    for name, struct in _STRUCTS.items():
        getattr(lib, name).argtypes = [ctypes.POINTER(struct), ctypes.c_void_p]
        getattr(lib, name).restype = ctypes.c_int
    size = ctypes.POINTER(ctypes.c_size_t)
    lib.ha_la_conv_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_conv_args), size]
    lib.ha_la_scan_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_scan_args), ctypes.c_int, size]
    for name in ("conv", "scan"):
        getattr(lib, f"ha_la_{name}_workspace_bytes").restype = ctypes.c_int


# ---------------------------------------------------------------- calls

def ha_la_conv_workspace_bytes(args: ha_la_conv_args) -> int:
    """Of the backward pass."""
    n = ctypes.c_size_t(0)
    rc = binding.load_library().ha_la_conv_workspace_bytes(ctypes.byref(args), ctypes.byref(n))
    if rc != HA_LA_OK:
        raise HaLaError(rc, "ha_la_conv_workspace_bytes")
    return n.value


def ha_la_scan_workspace_bytes(args: ha_la_scan_args, backward: bool = False) -> int:
    n = ctypes.c_size_t(0)
    rc = binding.load_library().ha_la_scan_workspace_bytes(ctypes.byref(args), int(bool(backward)), ctypes.byref(n))
    if rc != HA_LA_OK:
        raise HaLaError(rc, "ha_la_scan_workspace_bytes")
    return n.value


def _rows(t, like, name, lead, inner):
    """Elements from a token of `t` to the next: rows of like's type and device, [*lead, *inner], contiguous within a token, tokens at one distance."""
    ok = _reachable(t, like) and t.dtype == like.dtype and tuple(t.shape) == (*lead, *inner)
    size = 1
    if ok:
        for n, s in zip(reversed(inner), reversed(t.stride()[len(lead):])):
            ok = ok and (n == 1 or s == size)
            size *= n
    if ok and t.numel() == 0:
        return size
    step = size
    if ok:
        tokens = 1                                           # tokens that the dimensions behind this one hold
        for n, s in zip(reversed(lead), reversed(t.stride()[:len(lead)])):
            if n > 1:
                if tokens == 1:
                    step = s
                ok = ok and s == step * tokens
            tokens *= n
    if not ok or step < size:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, strides {tuple(t.stride())}, on {t.device}; wanted is {like.dtype} "
                         f"{(*lead, *inner)} on {like.device}, contiguous but for one distance of at least {size} from token to token")
    return step


def _vector(t, like, name, shape):
    import torch

    if t is not None:
        _as(t, like, name, shape, torch.float32)


def _sequences(x, cu_seqlens, name):
    """(batch, tokens, sequences) of [B, T, ..] or [T, ..]."""
    import torch

    lead = tuple(x.shape[:-1])
    B, T = lead if len(lead) == 2 else (1, lead[0])
    if cu_seqlens is None:
        return lead, B, T, B
    if B != 1 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
        raise ValueError(f"cu_seqlens: {tuple(cu_seqlens.shape)} with {name} {tuple(x.shape)}; wanted are [N + 1], N >= 1, and a batch of one")
    _as(cu_seqlens, x, "cu_seqlens", cu_seqlens.shape, torch.int32)
    _sizes(cu_seqlens, "cu_seqlens")
    return lead, B, T, cu_seqlens.numel() - 1


def _first(what, x, dims):
    _cuda(x, what)
    if x.dim() not in dims:
        raise ValueError(f"x: {tuple(x.shape)}; wanted are {' or '.join({2: '[T, channels]', 3: '[B, T, channels]'}[d] for d in dims)}")
    if x.shape[-1] < 1:
        raise ValueError(f"x: {tuple(x.shape)}; wanted is at least one channel")
    _sizes(x, "x")
    return _element(x, "x")


def _workspace(on, args, workspace, nbytes):
    workspace = on.scratch(workspace, nbytes)
    args.workspace, args.workspace_bytes = _aligned_part(workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return workspace


def _status(on, args, status_word):
    import torch

    status_word = on.new(status_word, (1,), torch.int32, zeros=True)
    args.status_word = status_word.data_ptr()
    return status_word


# ---------------------------------------------------------------- short convolution

def _conv_args(what, x, w, bias, activation, cu_seqlens, max_seqlen, dims=(2, 3)):
    dtype = _first(what, x, dims)
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation: {activation!r}; wanted is 'silu' or None")
    C = x.shape[-1]
    if w.dim() != 2 or w.shape[1] not in (2, 3, 4):
        raise ValueError(f"w: {tuple(w.shape)}; wanted are [channels, taps] with 2, 3 or 4 taps")
    _vector(w, x, "w", (C, w.shape[1]))
    _vector(bias, x, "bias", (C,))
    lead, B, T, N = _sequences(x, cu_seqlens, "x")
    stride = _rows(x, x, "x", lead, (C,))
    args = ha_la_conv_args(dtype=dtype, batch=B, seqlen=T, channels=C, taps=w.shape[1], activation=_ACTIVATIONS[activation], x_stride=stride, x=_ptr(x),
                           w=_ptr(w), bias=_ptr(bias), cu_seqlens=_ptr(cu_seqlens), num_seqs=0 if cu_seqlens is None else N, max_seqlen=_bound(max_seqlen))
    return args, N, C, w.shape[1] - 1


def ha_la_conv(x, w, *, bias=None, activation="silu", h0=None, cu_seqlens=None, max_seqlen=0, y=None, hT=None, want_hT=True, status_word=None,
               stream=None):
    """y_t = act(bias + sum_j w[:, j] x_{t - taps + 1 + j}), every channel by itself; activation "silu" or None.

    x : [B, T, C] (or [T, C]) bf16 or fp32    w : fp32 [C, taps], taps 2, 3 or 4    bias : fp32 [C] or None
    h0 : [N, taps - 1, C], x's type, the inputs in front of each sequence, oldest first, or None (zeros)
    cu_seqlens : int32 [N+1] device tensor or None (packed sequences, B = 1); max_seqlen : bound on their lengths, 0 = T
    Returns (y, hT, status_word): hT the last taps - 1 inputs of each sequence (None if not wanted); a status word other than 0 reports lengths
    that do not fit.
    """
    import torch

    args, N, C, K = _conv_args("ha_la_conv", x, w, bias, activation, cu_seqlens, max_seqlen)
    for name, t, dt, n in (("h0", h0, x.dtype, N * K * C), ("y", y, x.dtype, x.numel()), ("hT", hT, x.dtype, N * K * C), ("status_word", status_word, torch.int32, 1)):
        _check_room(name, t, x, dt, n)
    with _On(stream, x) as on:
        y = on.new(y, x.shape, x.dtype)
        if want_hT or hT is not None:
            hT = on.new(hT, (N, K, C), x.dtype)
        args.h0, args.y, args.hT = _ptr(h0), _ptr(y), _ptr(hT)
        status_word = _status(on, args, status_word)
        on.call("ha_la_conv", args)
    return y, hT, status_word


def ha_la_conv_backward(dy, x, w, *, bias=None, activation="silu", h0=None, dhT=None, cu_seqlens=None, max_seqlen=0, dx=None, dw=None, db=None,
                        dh0=None, want_dh0=True, workspace=None, status_word=None, stream=None):
    """Gradients of ha_la_conv from dy (of y, contiguous) and dhT (of hT, or None: zeros).

    Returns (dx, dw, db, dh0, status_word, workspace); db is None without a bias, dh0 if it is not wanted.
    """
    import torch

    args, N, C, K = _conv_args("ha_la_conv_backward", x, w, bias, activation, cu_seqlens, max_seqlen)
    _as(dy, x, "dy", x.shape)
    for name, t, dt, n in (("h0", h0, x.dtype, N * K * C), ("dhT", dhT, x.dtype, N * K * C), ("dx", dx, x.dtype, x.numel()), ("dw", dw, torch.float32, C * (K + 1)),
                           ("db", db, torch.float32, C), ("dh0", dh0, x.dtype, N * K * C), ("workspace", workspace, None, 0),
                           ("status_word", status_word, torch.int32, 1)):
        _check_room(name, t, x, dt, n)
    with _On(stream, x) as on:
        dx, dw = on.new(dx, x.shape, x.dtype), on.new(dw, (C, K + 1), torch.float32)
        db = on.new(db, (C,), torch.float32) if bias is not None else None
        if want_dh0 or dh0 is not None:
            dh0 = on.new(dh0, (N, K, C), x.dtype)
        args.h0, args.dy, args.dhT, args.dx, args.dw, args.db, args.dh0 = (_ptr(t) for t in (h0, dy, dhT, dx, dw, db, dh0))
        workspace = _workspace(on, args, workspace, ha_la_conv_workspace_bytes(args))
        status_word = _status(on, args, status_word)
        on.call("ha_la_conv_backward", args)
    return dx, dw, db, dh0, status_word, workspace


def ha_la_conv_decode(x, w, state, *, bias=None, activation="silu", y=None, state_out=None, stream=None):
    """One token per sequence.

    x : [N, C]    state : [N, taps - 1, C], the last inputs, oldest first, or None (zeros)
    The new state goes to state_out (default: in place into state; allocated when that is None).  Returns (y, new state).
    """
    args, _, C, K = _conv_args("ha_la_conv_decode", x, w, bias, activation, None, 0, (2,))
    N = x.shape[0]
    for name, t, n in (("state", state, N * K * C), ("state_out", state_out, N * K * C), ("y", y, x.numel())):
        _check_room(name, t, x, x.dtype, n)
    args.batch, args.seqlen = N, 1
    with _On(stream, x) as on:
        y = on.new(y, x.shape, x.dtype)
        if state_out is None:
            state_out = on.new(state, (N, K, C), x.dtype)
        args.h0, args.y, args.hT = _ptr(state), _ptr(y), _ptr(state_out)
        on.call("ha_la_conv_decode", args)
    return y, state_out


# ---------------------------------------------------------------- selective scan

def _scan_args(what, x, dt, A, B, C, D, z, dt_bias, softplus, cu_seqlens, max_seqlen, dims=(2, 3)):
    dtype = _first(what, x, dims)
    ch = x.shape[-1]
    lead, batch, T, N = _sequences(x, cu_seqlens, "x")
    if A.dim() != 2 or B.dim() != len(lead) + 2:
        raise ValueError(f"A: {tuple(A.shape)}, B: {tuple(B.shape)}; wanted are [channels, states] and {'[N' if dims == (2,) else '[B, T'}, groups, states]")
    G, S = B.shape[-2:]
    if not 1 <= S <= 64 or G < 1 or ch % G:
        raise ValueError(f"B: {tuple(B.shape)} with {ch} channels; wanted are 1 to 64 states, and groups that divide the channels")
    _vector(A, x, "A", (ch, S))
    _vector(D, x, "D", (ch,))
    _vector(dt_bias, x, "dt_bias", (ch,))
    strides = {"x_stride": _rows(x, x, "x", lead, (ch,)), "dt_stride": _rows(dt, x, "dt", lead, (ch,)), "b_stride": _rows(B, x, "B", lead, (G, S)),
               "c_stride": _rows(C, x, "C", lead, (G, S)), "z_stride": _rows(z, x, "z", lead, (ch,)) if z is not None else 0}
    return ha_la_scan_args(dtype=dtype, batch=batch, seqlen=T, channels=ch, states=S, groups=G, softplus=int(bool(softplus)),
                           num_seqs=0 if cu_seqlens is None else N, max_seqlen=_bound(max_seqlen), cu_seqlens=_ptr(cu_seqlens), x=_ptr(x), dt=_ptr(dt),
                           B=_ptr(B), C=_ptr(C), z=_ptr(z), A=_ptr(A), D=_ptr(D), dt_bias=_ptr(dt_bias), **strides), N, ch, S


def ha_la_scan(x, dt, A, B, C, *, D=None, z=None, dt_bias=None, softplus=True, h0=None, cu_seqlens=None, max_seqlen=0, y=None, hT=None, want_hT=True,
               workspace=None, status_word=None, stream=None):
    """delta = softplus(dt + dt_bias); h <- e^(delta A) h + delta B_t x_t; y_t = (<C_t, h> + D x_t) silu(z_t), every channel by itself.

    x, dt, z : [B, T, channels] (or [T, channels]) bf16 or fp32, z None: no gate    B, C : [B, T, groups, S] (or [T, groups, S]), S <= 64; channel c
    reads group c / (channels / groups)    A : fp32 [channels, S], <= 0    D, dt_bias : fp32 [channels] or None    softplus False: delta = dt + dt_bias,
    which has to be >= 0    h0 : fp32 [N, channels, S] or None (zeros)    cu_seqlens, max_seqlen : as in ha_la_conv
    Returns (y, hT, status_word, workspace); hT is None if not wanted.  workspace and status_word may be handed in again, for one call at a time.
    """
    import torch

    args, N, ch, S = _scan_args("ha_la_scan", x, dt, A, B, C, D, z, dt_bias, softplus, cu_seqlens, max_seqlen)
    for name, t, dt_, n in (("h0", h0, torch.float32, N * ch * S), ("y", y, x.dtype, x.numel()), ("hT", hT, torch.float32, N * ch * S),
                            ("workspace", workspace, None, 0), ("status_word", status_word, torch.int32, 1)):
        _check_room(name, t, x, dt_, n)
    with _On(stream, x) as on:
        y = on.new(y, x.shape, x.dtype)
        if want_hT or hT is not None:
            hT = on.new(hT, (N, ch, S), torch.float32)
        args.h0, args.y, args.hT = _ptr(h0), _ptr(y), _ptr(hT)
        workspace = _workspace(on, args, workspace, ha_la_scan_workspace_bytes(args))
        status_word = _status(on, args, status_word)
        on.call("ha_la_scan", args)
    return y, hT, status_word, workspace


def ha_la_scan_backward(dy, x, dt, A, B, C, *, D=None, z=None, dt_bias=None, softplus=True, h0=None, dhT=None, cu_seqlens=None, max_seqlen=0, dx=None,
                        ddt=None, dA=None, dB=None, dC=None, dD=None, dz=None, ddt_bias=None, dh0=None, want_dh0=True, workspace=None, status_word=None,
                        stream=None):
    """Gradients of ha_la_scan from dy (of y, contiguous) and dhT (of hT, fp32, or None: zeros); dh0 may be dhT itself.

    Returns (dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0, status_word, workspace); dD, dz and ddt_bias are None without D, z and dt_bias, dh0 if it is
    not wanted.
    """
    import torch

    args, N, ch, S = _scan_args("ha_la_scan_backward", x, dt, A, B, C, D, z, dt_bias, softplus, cu_seqlens, max_seqlen)
    _as(dy, x, "dy", x.shape)
    f32 = torch.float32
    for name, t, dt_, n in (("h0", h0, f32, N * ch * S), ("dhT", dhT, f32, N * ch * S), ("dx", dx, x.dtype, x.numel()), ("ddt", ddt, x.dtype, x.numel()),
                            ("dA", dA, f32, ch * S), ("dB", dB, x.dtype, B.numel()), ("dC", dC, x.dtype, B.numel()), ("dD", dD, f32, ch),
                            ("dz", dz, x.dtype, x.numel()), ("ddt_bias", ddt_bias, f32, ch), ("dh0", dh0, f32, N * ch * S), ("workspace", workspace, None, 0),
                            ("status_word", status_word, torch.int32, 1)):
        _check_room(name, t, x, dt_, n)
    with _On(stream, x) as on:
        dx, ddt = on.new(dx, x.shape, x.dtype), on.new(ddt, x.shape, x.dtype)
        dB, dC = on.new(dB, B.shape, x.dtype), on.new(dC, B.shape, x.dtype)
        dA = on.new(dA, A.shape, f32)
        dD = on.new(dD, (ch,), f32) if D is not None else None
        dz = on.new(dz, x.shape, x.dtype) if z is not None else None
        ddt_bias = on.new(ddt_bias, (ch,), f32) if dt_bias is not None else None
        if want_dh0 or dh0 is not None:
            dh0 = on.new(dh0, (N, ch, S), f32)
        for name, t in (("h0", h0), ("dy", dy), ("dhT", dhT), ("dx", dx), ("ddt", ddt), ("dA", dA), ("dB", dB), ("dC", dC), ("dD", dD), ("dz", dz),
                        ("ddt_bias", ddt_bias), ("dh0", dh0)):
            setattr(args, name, _ptr(t))
        workspace = _workspace(on, args, workspace, ha_la_scan_workspace_bytes(args, True))
        status_word = _status(on, args, status_word)
        on.call("ha_la_scan_backward", args)
    return dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0, status_word, workspace


def ha_la_scan_decode(x, dt, A, B, C, state, *, D=None, z=None, dt_bias=None, softplus=True, y=None, state_out=None, stream=None):
    """One token per sequence.

    x, dt, z : [N, channels]    B, C : [N, groups, S]    state : fp32 [N, channels, S] or None (zeros)
    The new state goes to state_out (default: in place into state; allocated when that is None).  Returns (y, new state).
    """
    import torch

    args, _, ch, S = _scan_args("ha_la_scan_decode", x, dt, A, B, C, D, z, dt_bias, softplus, None, 0, (2,))
    N = x.shape[0]
    for name, t, dt_, n in (("state", state, torch.float32, N * ch * S), ("state_out", state_out, torch.float32, N * ch * S), ("y", y, x.dtype, x.numel())):
        _check_room(name, t, x, dt_, n)
    args.batch, args.seqlen = N, 1
    with _On(stream, x) as on:
        y = on.new(y, x.shape, x.dtype)
        if state_out is None:
            state_out = on.new(state, (N, ch, S), torch.float32)
        args.h0, args.y, args.hT = _ptr(state), _ptr(y), _ptr(state_out)
        on.call("ha_la_scan_decode", args)
    return y, state_out
