"""Binding of the layers that alternate with the recurrences in a hybrid model (include/ha_la.h): short causal convolution, selective
state space scan, forward, backward and one token; attention over latent rows, for prompts and for single tokens.

As in `layer`: marshalling only, torch CUDA tensors in and out, everything is computed by the library's kernels on the caller's
stream, nothing is synchronised, tensors whose type, layout, size or device does not fit raise ValueError before anything is launched,
and nothing is recorded for autograd.  Inputs with one row to a token may be rows of a wider tensor (slices of a fused projection's
output along the last dimension); outputs are contiguous.  States, outputs and their gradients that a caller hands in have the shape that is
written beside them, outer dimensions taken together if that suits the caller (up to a flat buffer), and may hold more behind it; one whose inner
dimensions are others is refused, however many elements it has.
"""
from __future__ import annotations

import ctypes
import math

from . import binding
from .binding import HA_LA_OK, HaLaError, _aligned_part, _check_room, _reachable
from .layer import _On, _as, _bound, _cuda, _element, _float, _ptr, _sizes

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


class ha_la_latent_prefill_args(ctypes.Structure):
    _fields_ = [
        *((n, _i) for n in ("dtype", "batch", "seqlen", "seqlen_k", "num_heads", "d_nope", "d_rope", "d_v")), ("scale", ctypes.c_float),
        ("num_seqs", _i), ("max_seqlen", _i), ("cu_seqlens", _p), ("cu_seqlens_k", _p),
        *((n, _l) for n in ("q_stride", "kn_stride", "kr_stride", "v_stride", "kn_head_stride", "v_head_stride")),
        *((n, _p) for n in ("q", "kn", "kr", "v", "o", "lse", "status_word")),
    ]


class ha_la_latent_decode_args(ctypes.Structure):
    _fields_ = [
        *((n, _i) for n in ("dtype", "num_seqs", "new_tokens", "num_heads", "d_latent", "d_rope", "page_size", "num_pages", "max_pages")),
        ("scale", ctypes.c_float), *((n, _p) for n in ("q", "cache", "page_table", "lengths", "o", "lse", "workspace")),
        ("workspace_bytes", ctypes.c_size_t), ("status_word", _p),
    ]


_STRUCTS = {"ha_la_conv": ha_la_conv_args, "ha_la_conv_backward": ha_la_conv_args, "ha_la_conv_decode": ha_la_conv_args,
            "ha_la_scan": ha_la_scan_args, "ha_la_scan_backward": ha_la_scan_args, "ha_la_scan_decode": ha_la_scan_args,
            "ha_la_latent_prefill": ha_la_latent_prefill_args, "ha_la_latent_decode": ha_la_latent_decode_args}


def declare(lib) -> None:
    """Argument and result types of the entry points, for ctypes."""
    for name, struct in _STRUCTS.items():
        getattr(lib, name).argtypes = [ctypes.POINTER(struct), ctypes.c_void_p]
        getattr(lib, name).restype = ctypes.c_int
    size = ctypes.POINTER(ctypes.c_size_t)
    lib.ha_la_conv_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_conv_args), size]
    lib.ha_la_scan_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_scan_args), ctypes.c_int, size]
    lib.ha_la_latent_decode_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_latent_decode_args), size]
    for name in ("conv", "scan", "latent_decode"):
        getattr(lib, f"ha_la_{name}_workspace_bytes").restype = ctypes.c_int
    for name in ("prefill", "decode"):
        f = getattr(lib, f"ha_la_latent_{name}_path")
        f.argtypes, f.restype = [ctypes.POINTER(_STRUCTS[f"ha_la_latent_{name}"])], ctypes.c_char_p


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


def ha_la_latent_decode_workspace_bytes(args: ha_la_latent_decode_args) -> int:
    n = ctypes.c_size_t(0)
    rc = binding.load_library().ha_la_latent_decode_workspace_bytes(ctypes.byref(args), ctypes.byref(n))
    if rc != HA_LA_OK:
        raise HaLaError(rc, "ha_la_latent_decode_workspace_bytes")
    return n.value


def ha_la_latent_prefill_path(args: ha_la_latent_prefill_args):
    r = binding.load_library().ha_la_latent_prefill_path(ctypes.byref(args))
    return None if r is None else r.decode()


def ha_la_latent_decode_path(args: ha_la_latent_decode_args):
    r = binding.load_library().ha_la_latent_decode_path(ctypes.byref(args))
    return None if r is None else r.decode()


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


def _laid_out(name, t, like, dtype, shape):
    """A tensor (or None) that the kernels take by its address: contiguous, and its elements in that shape's order as far as its own shape tells.  From the last one on
    dimensions agree, but for the outermost (in front of which there are only ones): it has at least what the wanted ones that are left come to."""
    if t is None:
        return
    have, shape = tuple(t.shape), tuple(shape)
    i, j = len(have) - 1, len(shape) - 1
    while i > 0 and j >= 0 and have[i] == shape[j]:
        i, j = i - 1, j - 1
    fits = i >= 0 and math.prod(have) >= math.prod(shape) and (j < 0 or all(n == 1 for n in have[:i]) and have[i] >= math.prod(shape[:j + 1]))
    if not (_reachable(t, like) and t.is_contiguous() and t.dtype == dtype and fits):
        raise ValueError(f"{name}: {t.dtype} {have}, strides {tuple(t.stride())}, on {t.device}; wanted is {dtype} {shape}, contiguous, on {like.device}")


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
    r = binding._native().conv(x, w, bias, _ACTIVATIONS.get(activation), h0, cu_seqlens, max_seqlen, y, hT, want_hT, status_word, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_conv")
    import torch

    args, N, C, K = _conv_args("ha_la_conv", x, w, bias, activation, cu_seqlens, max_seqlen)
    for name, t, shape in (("h0", h0, (N, K, C)), ("y", y, x.shape), ("hT", hT, (N, K, C))):
        _laid_out(name, t, x, x.dtype, shape)
    _check_room("status_word", status_word, x, torch.int32, 1)
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
    r = binding._native().conv_backward(dy, x, w, bias, _ACTIVATIONS.get(activation), h0, dhT, cu_seqlens, max_seqlen, dx, dw, db, dh0, want_dh0,
                                        workspace, status_word, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_conv_backward")
    import torch

    args, N, C, K = _conv_args("ha_la_conv_backward", x, w, bias, activation, cu_seqlens, max_seqlen)
    _as(dy, x, "dy", x.shape)
    for name, t, dt, shape in (("h0", h0, x.dtype, (N, K, C)), ("dhT", dhT, x.dtype, (N, K, C)), ("dx", dx, x.dtype, x.shape), ("dw", dw, torch.float32, (C, K + 1)),
                               ("db", db, torch.float32, (C,)), ("dh0", dh0, x.dtype, (N, K, C))):
        _laid_out(name, t, x, dt, shape)
    _check_room("workspace", workspace, x, None, 0)
    _check_room("status_word", status_word, x, torch.int32, 1)
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
    r = binding._native().conv_decode(x, w, state, bias, _ACTIVATIONS.get(activation), y, state_out, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_conv_decode")
    args, _, C, K = _conv_args("ha_la_conv_decode", x, w, bias, activation, None, 0, (2,))
    N = x.shape[0]
    for name, t, shape in (("state", state, (N, K, C)), ("state_out", state_out, (N, K, C)), ("y", y, x.shape)):
        _laid_out(name, t, x, x.dtype, shape)
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
    r = binding._native().scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, cu_seqlens, max_seqlen, y, hT, want_hT, workspace, status_word, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_scan")
    import torch

    args, N, ch, S = _scan_args("ha_la_scan", x, dt, A, B, C, D, z, dt_bias, softplus, cu_seqlens, max_seqlen)
    for name, t, dt_, shape in (("h0", h0, torch.float32, (N, ch, S)), ("y", y, x.dtype, x.shape), ("hT", hT, torch.float32, (N, ch, S))):
        _laid_out(name, t, x, dt_, shape)
    _check_room("workspace", workspace, x, None, 0)
    _check_room("status_word", status_word, x, torch.int32, 1)
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
    r = binding._native().scan_backward(dy, x, dt, A, B, C, D, z, dt_bias, softplus, h0, dhT, cu_seqlens, max_seqlen, dx, ddt, dA, dB, dC, dD, dz,
                                        ddt_bias, dh0, want_dh0, workspace, status_word, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_scan_backward")
    import torch

    args, N, ch, S = _scan_args("ha_la_scan_backward", x, dt, A, B, C, D, z, dt_bias, softplus, cu_seqlens, max_seqlen)
    _as(dy, x, "dy", x.shape)
    f32 = torch.float32
    for name, t, dt_, shape in (("h0", h0, f32, (N, ch, S)), ("dhT", dhT, f32, (N, ch, S)), ("dx", dx, x.dtype, x.shape), ("ddt", ddt, x.dtype, x.shape),
                                ("dA", dA, f32, (ch, S)), ("dB", dB, x.dtype, B.shape), ("dC", dC, x.dtype, B.shape), ("dD", dD, f32, (ch,)),
                                ("dz", dz, x.dtype, x.shape), ("ddt_bias", ddt_bias, f32, (ch,)), ("dh0", dh0, f32, (N, ch, S))):
        _laid_out(name, t, x, dt_, shape)
    _check_room("workspace", workspace, x, None, 0)
    _check_room("status_word", status_word, x, torch.int32, 1)
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
    r = binding._native().scan_decode(x, dt, A, B, C, state, D, z, dt_bias, softplus, y, state_out, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_scan_decode")
    import torch

    args, _, ch, S = _scan_args("ha_la_scan_decode", x, dt, A, B, C, D, z, dt_bias, softplus, None, 0, (2,))
    N = x.shape[0]
    for name, t, dt_, shape in (("state", state, torch.float32, (N, ch, S)), ("state_out", state_out, torch.float32, (N, ch, S)), ("y", y, x.dtype, x.shape)):
        _laid_out(name, t, x, dt_, shape)
    args.batch, args.seqlen = N, 1
    with _On(stream, x) as on:
        y = on.new(y, x.shape, x.dtype)
        if state_out is None:
            state_out = on.new(state, (N, ch, S), torch.float32)
        args.h0, args.y, args.hT = _ptr(state), _ptr(y), _ptr(state_out)
        on.call("ha_la_scan_decode", args)
    return y, state_out


# ---------------------------------------------------------------- attention over latent rows

def _heads(t, like, name, lead, H):
    """(elements from a token to the next, from a head to the next, head size) of [*lead, H, d]: contiguous within a head, else at any distances."""
    if t.dim() != len(lead) + 2:
        raise ValueError(f"{name}: {tuple(t.shape)}; wanted are {(*lead, H, 'd')}")
    d = t.shape[-1]
    ok = _reachable(t, like) and t.dtype == like.dtype and tuple(t.shape) == (*lead, H, d) and d >= 1
    if ok and t.numel() == 0:
        return H * d, d, d
    head = t.stride(-2) if H > 1 else d
    step, tokens = H * d, 1
    if ok:
        ok = (d == 1 or t.stride(-1) == 1) and head >= d
        for n, s in zip(reversed(lead), reversed(t.stride()[:len(lead)])):
            if n > 1:
                if tokens == 1:
                    step = s
                ok = ok and s == step * tokens
            tokens *= n
    if not ok or step < d:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, strides {tuple(t.stride())}, on {t.device}; wanted is {like.dtype} {(*lead, H, 'd')} "
                         f"on {like.device}, contiguous within a head, with one distance from token to token and one from head to head")
    return step, head, d


def ha_la_latent_prefill(q, kn, kr, v, *, scale=1.0, cu_seqlens=None, cu_seqlens_k=None, max_seqlen=0, o=None, lse=None, status_word=None, stream=None):
    """Causal attention of a prompt on expanded keys and values: s_ij = scale (q_i[..d_nope] . kn_j + q_i[d_nope..] . kr_j) per head, kr shared by
    all heads.  A sequence's queries are its last tokens: query i sees the keys up to i + (keys - queries).

    q  : [B, T, H, d_nope + d_rope] (or [T, H, ..]) bf16 or fp32, may be rows of a wider tensor    kn : [B, Tk, H, d_nope]    kr : [B, Tk, d_rope]
    v  : [B, Tk, H, d_v]; kn and v may be slices of one tensor    cu_seqlens : int32 [N+1] or None (packed, B = 1), cu_seqlens_k the same of the keys
    (None: the queries')    max_seqlen : bound on a sequence's queries, 0 = T
    Returns (o, lse, status_word): o [B, T, H, d_v], lse fp32 [B, T, H], the logarithm of the sum of e^s; a query without a key has 0 and -infinity.
    """
    r = binding._native().latent_prefill(q, kn, kr, v, scale, cu_seqlens, cu_seqlens_k, max_seqlen, o, lse, status_word, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_latent_prefill")
    import torch

    _cuda(q, "ha_la_latent_prefill")
    if q.dim() not in (3, 4):
        raise ValueError(f"q: {tuple(q.shape)}; wanted are [B, T, heads, d] or [T, heads, d]")
    _sizes(q, "q")
    dtype, lead, H, dq = _element(q, "q"), tuple(q.shape[:-2]), q.shape[-2], q.shape[-1]
    if kr.dim() != len(lead) + 1 or kr.shape[-1] >= dq or H < 1:
        raise ValueError(f"kr: {tuple(kr.shape)}; wanted are {len(lead) + 1} dimensions and less than q's {dq} channels")
    _sizes(kr, "kr")
    keys, dr = (*lead[:-1], kr.shape[-2]), kr.shape[-1]
    B, T = lead if len(lead) == 2 else (1, lead[0])
    N = 0
    if cu_seqlens is None and cu_seqlens_k is not None:
        raise ValueError("cu_seqlens_k without cu_seqlens")
    if cu_seqlens is not None:
        _, _, _, N = _sequences(q.flatten(-2) if q.is_contiguous() else q[..., 0], cu_seqlens, "q")
        if cu_seqlens_k is None:
            if keys != lead:
                raise ValueError(f"kr: {tuple(kr.shape)} for {T} queries; cu_seqlens_k is wanted")
            cu_seqlens_k = cu_seqlens
        _as(cu_seqlens_k, q, "cu_seqlens_k", (N + 1,), torch.int32)
    q_stride = _rows(q, q, "q", lead, (H, dq))
    kr_stride = _rows(kr, q, "kr", keys, (dr,))
    kn_stride, kn_head, dn = _heads(kn, q, "kn", keys, H)
    v_stride, v_head, dv = _heads(v, q, "v", keys, H)
    if dn + dr != dq:
        raise ValueError(f"q: {tuple(q.shape)}; wanted are kn's {dn} and kr's {dr} channels together")
    _laid_out("o", o, q, q.dtype, (*lead, H, dv))
    _laid_out("lse", lse, q, torch.float32, (*lead, H))
    _check_room("status_word", status_word, q, torch.int32, 1)
    args = ha_la_latent_prefill_args(dtype=dtype, batch=B, seqlen=T, seqlen_k=keys[-1], num_heads=H, d_nope=dn, d_rope=dr, d_v=dv, scale=_float(scale, "scale"),
                                     num_seqs=N, max_seqlen=_bound(max_seqlen), cu_seqlens=_ptr(cu_seqlens), cu_seqlens_k=_ptr(cu_seqlens_k),
                                     q_stride=q_stride, kn_stride=kn_stride, kr_stride=kr_stride, v_stride=v_stride, kn_head_stride=kn_head,
                                     v_head_stride=v_head, q=_ptr(q), kn=_ptr(kn), kr=_ptr(kr), v=_ptr(v))
    with _On(stream, q) as on:
        o, lse = on.new(o, (*lead, H, dv), q.dtype), on.new(lse, (*lead, H), torch.float32)
        args.o, args.lse = _ptr(o), _ptr(lse)
        status_word = _status(on, args, status_word)
        on.call("ha_la_latent_prefill", args)
    return o, lse, status_word


def ha_la_latent_decode(q, cache, page_table, lengths, *, scale=1.0, o=None, lse=None, d_latent=None, workspace=None, status_word=None, stream=None):
    """Attention of one or a few new tokens a sequence to the cached latent rows themselves (absorbed form): s_ij = scale q_i . c_j per head,
    o_i = sum of softmax weights times c_j[..d_latent].

    q : [N, new, H, d_latent + d_rope] bf16 or fp32    cache : [pages, page_size, d_latent + d_rope], q's type, page_size a power of two
    page_table : int32 [N, max_pages]    lengths : int32 [N], cached rows of each sequence, the new tokens' among them; token i of the new ones sees
    the rows up to its own    d_latent : default the row size - 64
    Returns (o, lse, status_word, workspace): o [N, new, H, d_latent], lse fp32 [N, new, H]; a token without a row has 0 and -infinity.
    A status word other than 0 reports a length or a page that does not exist.
    """
    r = binding._native().latent_decode(q, cache, page_table, lengths, scale, o, lse, d_latent, workspace, status_word, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_latent_decode")
    import torch

    _cuda(q, "ha_la_latent_decode")
    if q.dim() != 4 or cache.dim() != 3 or page_table.dim() != 2:
        raise ValueError(f"q: {tuple(q.shape)}, cache: {tuple(cache.shape)}, page_table: {tuple(page_table.shape)}; wanted are [N, new, heads, d], "
                         "[pages, page_size, d] and [N, max_pages]")
    for t, name in ((q, "q"), (cache, "cache"), (page_table, "page_table")):
        _sizes(t, name)
    dtype, (N, new, H, d) = _element(q, "q"), q.shape
    dl = d - 64 if d_latent is None else int(d_latent)
    if not 1 <= dl <= d:
        raise ValueError(f"d_latent: {dl} of {d} channels")
    if new < 1 or H < 1 or cache.shape[1] < 1 or cache.shape[1] & (cache.shape[1] - 1):
        raise ValueError(f"q: {tuple(q.shape)}, cache: {tuple(cache.shape)}; wanted are at least one token and head, and pages of a power of two")
    _as(q, q, "q", q.shape)
    _as(cache, q, "cache", (*cache.shape[:2], d))
    _as(page_table, q, "page_table", (N, page_table.shape[1]), torch.int32)
    _as(lengths, q, "lengths", (N,), torch.int32)
    _laid_out("o", o, q, q.dtype, (N, new, H, dl))
    _laid_out("lse", lse, q, torch.float32, (N, new, H))
    _check_room("workspace", workspace, q, None, 0)
    _check_room("status_word", status_word, q, torch.int32, 1)
    args = ha_la_latent_decode_args(dtype=dtype, num_seqs=N, new_tokens=new, num_heads=H, d_latent=dl, d_rope=d - dl, page_size=cache.shape[1],
                                    num_pages=cache.shape[0], max_pages=page_table.shape[1], scale=_float(scale, "scale"), q=_ptr(q), cache=_ptr(cache),
                                    page_table=_ptr(page_table), lengths=_ptr(lengths))
    with _On(stream, q) as on:
        o, lse = on.new(o, (N, new, H, dl), q.dtype), on.new(lse, (N, new, H), torch.float32)
        args.o, args.lse = _ptr(o), _ptr(lse)
        workspace = _workspace(on, args, workspace, ha_la_latent_decode_workspace_bytes(args))
        status_word = _status(on, args, status_word)
        on.call("ha_la_latent_decode", args)
    return o, lse, status_word, workspace
