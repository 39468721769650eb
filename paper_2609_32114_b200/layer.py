"""Binding of what stands next to the delta-rule recurrence in a hybrid model (include/ha_la.h): gated linear attention, forward,
backward and one token, and the norms on both sides of a block, forward and backward.

As in `binding`: marshalling only, torch CUDA tensors in and out, everything is computed by the library's kernels on the caller's
stream, nothing is synchronised, and tensors whose type, layout, size or device does not fit raise ValueError before anything is
launched.  The backward passes are plain calls that return gradients; nothing is recorded for autograd.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import binding
from .binding import HA_LA_BF16, HA_LA_FP32, HA_LA_OK, HaLaError, _aligned_part, _check_room, _reachable, ha_la_decode_args

HA_LA_ACT_SILU, HA_LA_ACT_SIGMOID = 0, 1
_ACTIVATIONS = {"silu": HA_LA_ACT_SILU, "sigmoid": HA_LA_ACT_SIGMOID}


class ha_la_gla_args(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("seqlen", ctypes.c_int32),
        ("num_qk_heads", ctypes.c_int32),
        ("num_v_heads", ctypes.c_int32),
        ("d_k", ctypes.c_int32),
        ("d_v", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("q", ctypes.c_void_p),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("g", ctypes.c_void_p),
        ("h0", ctypes.c_void_p),
        ("cu_seqlens", ctypes.c_void_p),
        ("num_seqs", ctypes.c_int32),
        ("max_seqlen", ctypes.c_int32),
        ("o", ctypes.c_void_p),
        ("hT", ctypes.c_void_p),
        ("do_", ctypes.c_void_p),
        ("dhT", ctypes.c_void_p),
        ("dq", ctypes.c_void_p),
        ("dk", ctypes.c_void_p),
        ("dv", ctypes.c_void_p),
        ("dg", ctypes.c_void_p),
        ("dh0", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
        ("status_word", ctypes.c_void_p),
    ]


class ha_la_gated_norm_args(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("activation", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("x", ctypes.c_void_p),
        ("w", ctypes.c_void_p),
        ("z", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("dy", ctypes.c_void_p),
        ("dx", ctypes.c_void_p),
        ("dz", ctypes.c_void_p),
        ("dw", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
    ]


class ha_la_add_norm_args(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int32),
        ("cols", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("scale", ctypes.c_float),
        ("eps", ctypes.c_float),
        ("x", ctypes.c_void_p),
        ("r", ctypes.c_void_p),
        ("w", ctypes.c_void_p),
        ("w_post", ctypes.c_void_p),
        ("y", ctypes.c_void_p),
        ("r_out", ctypes.c_void_p),
        ("dy", ctypes.c_void_p),
        ("dr_out", ctypes.c_void_p),
        ("dx", ctypes.c_void_p),
        ("dr", ctypes.c_void_p),
        ("dw", ctypes.c_void_p),
        ("dw_post", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p),
        ("workspace_bytes", ctypes.c_size_t),
    ]


_STRUCTS = {"ha_la_gla_prefill": ha_la_gla_args, "ha_la_gla_backward": ha_la_gla_args, "ha_la_gla_decode": ha_la_decode_args,
            "ha_la_gated_norm": ha_la_gated_norm_args, "ha_la_gated_norm_backward": ha_la_gated_norm_args,
            "ha_la_add_norm": ha_la_add_norm_args, "ha_la_add_norm_backward": ha_la_add_norm_args}


def declare(lib) -> None:
    """Argument and result types of the entry points, for ctypes."""
    for name, struct in _STRUCTS.items():
        getattr(lib, name).argtypes = [ctypes.POINTER(struct), ctypes.c_void_p]
        getattr(lib, name).restype = ctypes.c_int
    size = ctypes.POINTER(ctypes.c_size_t)
    lib.ha_la_gla_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_gla_args), ctypes.c_int, size]
    lib.ha_la_gated_norm_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_gated_norm_args), size]
    lib.ha_la_add_norm_workspace_bytes.argtypes = [ctypes.POINTER(ha_la_add_norm_args), size]
    for name in ("gla", "gated_norm", "add_norm"):
        getattr(lib, f"ha_la_{name}_workspace_bytes").restype = ctypes.c_int
    lib.ha_la_gla_path.argtypes = [ctypes.POINTER(ha_la_gla_args)]
    lib.ha_la_gla_path.restype = ctypes.c_char_p


# ---------------------------------------------------------------- calls

def ha_la_gla_workspace_bytes(args: ha_la_gla_args, backward: bool = False) -> int:
    n = ctypes.c_size_t(0)
    rc = binding.load_library().ha_la_gla_workspace_bytes(ctypes.byref(args), int(bool(backward)), ctypes.byref(n))
    if rc != HA_LA_OK:
        raise HaLaError(rc, "ha_la_gla_workspace_bytes")
    return n.value


def ha_la_gla_path(args: ha_la_gla_args) -> Optional[str]:
    r = binding.load_library().ha_la_gla_path(ctypes.byref(args))
    return None if r is None else r.decode()


def _norm_bytes(name, args) -> int:
    n = ctypes.c_size_t(0)
    rc = getattr(binding.load_library(), name)(ctypes.byref(args), ctypes.byref(n))
    if rc != HA_LA_OK:
        raise HaLaError(rc, name)
    return n.value


def ha_la_gated_norm_workspace_bytes(args: ha_la_gated_norm_args) -> int:
    return _norm_bytes("ha_la_gated_norm_workspace_bytes", args)


def ha_la_add_norm_workspace_bytes(args: ha_la_add_norm_args) -> int:
    return _norm_bytes("ha_la_add_norm_workspace_bytes", args)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _element(t, name):
    import torch

    if t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{name}: {t.dtype}; wanted is bfloat16 or float32")
    return HA_LA_BF16 if t.dtype == torch.bfloat16 else HA_LA_FP32


def _cuda(t, what):
    if not t.is_cuda:
        raise ValueError(f"{what} needs CUDA tensors (there is no CPU path)")


def _as(t, like, name, shape, dtype=None):
    """`t` has to be a contiguous tensor of that shape on like's device, or within its reach."""
    dtype = like.dtype if dtype is None else dtype
    if not (_reachable(t, like) and t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous()):
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)}, strides {tuple(t.stride())}, on {t.device}; wanted is {dtype} {tuple(shape)}, "
                         f"contiguous, on {like.device}")


_INT32_MAX = 2 ** 31 - 1                                     # the structs' sizes are 32-bit; ctypes would cut a larger one down to its low bits


def _sizes(t, name):
    if any(n > _INT32_MAX for n in t.shape):
        raise ValueError(f"{name}: {tuple(t.shape)}; a dimension has at most {_INT32_MAX}")


def _bound(v):
    """A bound on lengths: no sequence is longer than 32 bits count, so a larger one is that one."""
    return max(-_INT32_MAX - 1, min(int(v), _INT32_MAX))


def _float(v, name):
    v = float(v)
    if v != v:
        raise ValueError(f"{name}: {v}")
    return v


class _On:
    """A call's stream: the caller's (a cudaStream_t) or torch's current one of the tensors' device, which is the current device meanwhile.
    Where the caller names another stream than the current one, what the call allocates and fills is that stream's, and recorded
    on the current one as well, where the caller reads it once it has waited."""

    def __init__(self, stream, t):
        import torch

        self.device = torch.cuda.device(t.device)
        self.current = torch.cuda.current_stream(t.device)
        self.handle = self.current.cuda_stream if stream is None else stream
        other = self.handle != self.current.cuda_stream
        self.guard = torch.cuda.stream(torch.cuda.ExternalStream(stream, device=t.device)) if other else None
        self.t = t

    def __enter__(self):
        self.device.__enter__()
        if self.guard:
            self.guard.__enter__()
        return self

    def __exit__(self, *e):
        if self.guard:
            self.guard.__exit__(*e)
        self.device.__exit__(*e)

    def new(self, given, shape, dtype, zeros=False):
        import torch

        if given is not None:
            return given
        t = (torch.zeros if zeros else torch.empty)(shape, dtype=dtype, device=self.t.device)
        if self.guard:
            t.record_stream(self.current)
        return t

    def scratch(self, given, nbytes):
        import torch

        return self.new(given, (nbytes + 256,), torch.uint8)

    def call(self, name, args):
        rc = getattr(binding.load_library(), name)(ctypes.byref(args), ctypes.c_void_p(self.handle) if self.handle else None)
        if rc != HA_LA_OK:
            raise HaLaError(rc, name)


# ---------------------------------------------------------------- gated linear attention

def _gla_args(what, q, k, v, g, h0, cu_seqlens, max_seqlen, scale):
    """Checked sizes and inputs of a call: (args, V-heads, d, sequences)."""
    import torch

    _cuda(q, what)
    if q.dim() not in (3, 4) or v.dim() != q.dim():
        raise ValueError(f"q: {tuple(q.shape)}, v: {tuple(v.shape)}; wanted are [B, T, heads, d] or [T, heads, d]")
    dtype = _element(q, "q")
    _sizes(q, "q")
    _sizes(v, "v")
    lead, (HK, d), HV = tuple(q.shape[:-2]), q.shape[-2:], v.shape[-2]
    B, T = lead if len(lead) == 2 else (1, lead[0])
    _as(q, q, "q", q.shape)
    _as(k, q, "k", (*lead, HK, d))
    _as(v, q, "v", (*lead, HV, d))
    _as(g, q, "g", (*lead, HV), torch.float32)
    N = B
    if cu_seqlens is not None:
        if B != 1 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
            raise ValueError(f"cu_seqlens: {tuple(cu_seqlens.shape)} with q {tuple(q.shape)}; wanted are [N + 1], N >= 1, and a batch of one")
        _as(cu_seqlens, q, "cu_seqlens", cu_seqlens.shape, torch.int32)
        _sizes(cu_seqlens, "cu_seqlens")
        N = cu_seqlens.numel() - 1
    _check_room("h0", h0, q, torch.float32, N * HV * d * d)
    args = ha_la_gla_args(dtype=dtype, batch=B, seqlen=T, num_qk_heads=HK, num_v_heads=HV, d_k=d, d_v=d, scale=_float(scale, "scale"),
                          q=_ptr(q), k=_ptr(k), v=_ptr(v), g=_ptr(g), h0=_ptr(h0), cu_seqlens=_ptr(cu_seqlens),
                          num_seqs=0 if cu_seqlens is None else N, max_seqlen=_bound(max_seqlen))
    return args, HV, d, N


def _take_workspace(on, args, workspace, status_word, backward):
    import torch

    workspace = on.scratch(workspace, ha_la_gla_workspace_bytes(args, backward))
    status_word = on.new(status_word, (1,), torch.int32, zeros=True)
    args.workspace, args.workspace_bytes = _aligned_part(workspace.data_ptr(), workspace.numel() * workspace.element_size())
    args.status_word = status_word.data_ptr()
    return workspace, status_word


def ha_la_gla_prefill(q, k, v, g, *, h0=None, cu_seqlens=None, max_seqlen=0, scale=1.0, o=None, hT=None, want_hT=True, workspace=None,
                      status_word=None, stream=None):
    """h <- exp(g_t) h + k_t v_t^T, o_t = scale h^T q_t over whole sequences.

    q, k : [B, T, HK, d] (or [T, HK, d])    v : [B, T, HV, d]    bf16 or fp32, contiguous, d = 64 or 128, HV a multiple of HK
    g    : fp32 [B, T, HV], log-gates <= 0  h0 : fp32 [N, HV, d, d] or None (zeros)
    cu_seqlens : int32 [N+1] device tensor or None (packed sequences, B = 1); max_seqlen : bound on their lengths, 0 = T
    Returns (o, hT, status_word, workspace); hT is None if not wanted.  workspace and status_word may be handed in again, for one
    call at a time; a status word other than 0 reports lengths that do not fit.
    """
    r = binding._native().gla_prefill(q, k, v, g, h0, cu_seqlens, max_seqlen, stream, scale, o, hT, want_hT, workspace, status_word)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_gla_prefill")
    import torch

    args, HV, d, N = _gla_args("ha_la_gla_prefill", q, k, v, g, h0, cu_seqlens, max_seqlen, scale)
    state = N * HV * d * d
    for name, t, dt, n in (("o", o, q.dtype, v.numel()), ("hT", hT, torch.float32, state), ("workspace", workspace, None, 0),
                           ("status_word", status_word, None, 4)):
        _check_room(name, t, q, dt, n)
    with _On(stream, q) as on:
        o = on.new(o, v.shape, v.dtype)
        if want_hT or hT is not None:
            hT = on.new(hT, (N, HV, d, d), torch.float32)
        args.o, args.hT = _ptr(o), _ptr(hT)
        workspace, status_word = _take_workspace(on, args, workspace, status_word, False)
        on.call("ha_la_gla_prefill", args)
    return o, hT, status_word, workspace


def ha_la_gla_backward(do, q, k, v, g, *, h0=None, dhT=None, cu_seqlens=None, max_seqlen=0, scale=1.0, dq=None, dk=None, dv=None, dg=None,
                       dh0=None, want_dh0=True, workspace=None, status_word=None, stream=None):
    """Gradients of ha_la_gla_prefill from do (of o, like v) and dhT (of hT, fp32 [N, HV, d, d] or None: zeros).

    Returns (dq, dk, dv, dg, dh0, status_word, workspace); dh0 is None if not wanted.  dq and dk of a head that several V-heads share
    are the sums over them.
    """
    r = binding._native().gla_backward(do, q, k, v, g, h0, dhT, cu_seqlens, max_seqlen, stream, scale, dq, dk, dv, dg, dh0, want_dh0, workspace,
                                       status_word)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_gla_backward")
    import torch

    args, HV, d, N = _gla_args("ha_la_gla_backward", q, k, v, g, h0, cu_seqlens, max_seqlen, scale)
    _as(do, q, "do", v.shape)
    state = N * HV * d * d
    for name, t, dt, n in (("dhT", dhT, torch.float32, state), ("dq", dq, q.dtype, q.numel()), ("dk", dk, q.dtype, k.numel()),
                           ("dv", dv, q.dtype, v.numel()), ("dg", dg, torch.float32, g.numel()), ("dh0", dh0, torch.float32, state),
                           ("workspace", workspace, None, 0), ("status_word", status_word, None, 4)):
        _check_room(name, t, q, dt, n)
    with _On(stream, q) as on:
        dq, dk, dv = on.new(dq, q.shape, q.dtype), on.new(dk, k.shape, q.dtype), on.new(dv, v.shape, q.dtype)
        dg = on.new(dg, g.shape, torch.float32)
        if want_dh0 or dh0 is not None:
            dh0 = on.new(dh0, (N, HV, d, d), torch.float32)
        args.do_, args.dhT, args.dq, args.dk, args.dv, args.dg, args.dh0 = (_ptr(t) for t in (do, dhT, dq, dk, dv, dg, dh0))
        workspace, status_word = _take_workspace(on, args, workspace, status_word, True)
        on.call("ha_la_gla_backward", args)
    return dq, dk, dv, dg, dh0, status_word, workspace


def ha_la_gla_decode(q, k, v, g, state, *, scale=1.0, o=None, state_out=None, stream=None):
    """One token per sequence: state <- exp(g) state + k v^T, o = scale state^T q.

    q, k : [N, HK, d]   v : [N, HV, d]   g : fp32 [N, HV]   state : fp32 [N, HV, d, d] or None (zeros)
    The new state goes to state_out (default: in place into state; allocated when that is None).  Returns (o, new state).
    """
    r = binding._native().gla_decode(q, k, v, g, state, stream, scale, o, state_out)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_gla_decode")
    import torch

    _cuda(q, "ha_la_gla_decode")
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError(f"q: {tuple(q.shape)}, v: {tuple(v.shape)}; wanted are [N, heads, d]")
    _sizes(q, "q")
    _sizes(v, "v")
    dtype, (N, HK, d), HV = _element(q, "q"), q.shape, v.shape[1]
    _as(q, q, "q", q.shape)
    _as(k, q, "k", (N, HK, d))
    _as(v, q, "v", (N, HV, d))
    _as(g, q, "g", (N, HV), torch.float32)
    for name, t, dt, n in (("state", state, torch.float32, N * HV * d * d), ("state_out", state_out, torch.float32, N * HV * d * d), ("o", o, q.dtype, v.numel())):
        _check_room(name, t, q, dt, n)
    scale = _float(scale, "scale")
    with _On(stream, q) as on:
        o = on.new(o, v.shape, q.dtype)
        if state_out is None:
            state_out = on.new(state, (N, HV, d, d), torch.float32)
        args = ha_la_decode_args(variant=0, dtype=dtype, num_seqs=N, num_qk_heads=HK, num_v_heads=HV, d_k=d, d_v=d, scale=scale,
                                 q=_ptr(q), k=_ptr(k), v=_ptr(v), g=_ptr(g), h_in=_ptr(state), h_out=_ptr(state_out), o=_ptr(o))
        on.call("ha_la_gla_decode", args)
    return o, state_out


# ---------------------------------------------------------------- norms

def _rows_of(what, x, w):
    """Checked rows [.., cols] and their weight: (dtype, rows, cols)."""
    import torch

    _cuda(x, what)
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"x: {tuple(x.shape)}; wanted are rows of at least one value")
    dtype = _element(x, "x")
    if x.shape[-1] > _INT32_MAX:
        raise ValueError(f"x: {tuple(x.shape)}; a row has at most {_INT32_MAX} values")
    _as(x, x, "x", x.shape)
    _as(w, x, "w", (x.shape[-1],), torch.float32)
    return dtype, x.numel() // x.shape[-1], x.shape[-1]


def _out(t, x, name):
    _check_room(name, t, x, x.dtype, x.numel())


def _activation(name):
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation: {name!r}; wanted is one of {sorted(_ACTIVATIONS)}")
    return _ACTIVATIONS[name]


def _eps(v):
    v = _float(v, "eps")
    if v < 0:
        raise ValueError(f"eps: {v}")
    return v


def ha_la_gated_norm(x, w, z=None, *, activation="silu", eps=1e-6, y=None, stream=None):
    """y = x / sqrt(mean(x^2) + eps) * w * act(z) over the last dimension; z None: no gate; act "silu" or "sigmoid".

    x, z : [.., cols] bf16 or fp32, contiguous    w : fp32 [cols]    Returns y.
    """
    r = binding._native().gated_norm(x, w, z, _ACTIVATIONS.get(activation), eps, y, stream)
    if r.__class__ is not int and r is not None:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_gated_norm")
    act, eps = _activation(activation), _eps(eps)
    dtype, rows, cols = _rows_of("ha_la_gated_norm", x, w)
    if z is not None:
        _as(z, x, "z", x.shape)
    _out(y, x, "y")
    with _On(stream, x) as on:
        y = on.new(y, x.shape, x.dtype)
        on.call("ha_la_gated_norm", ha_la_gated_norm_args(dtype=dtype, activation=act, rows=rows, cols=cols, eps=eps, x=_ptr(x), w=_ptr(w),
                                                          z=_ptr(z), y=_ptr(y)))
    return y


def ha_la_gated_norm_backward(dy, x, w, z=None, *, activation="silu", eps=1e-6, dx=None, dw=None, dz=None, workspace=None, stream=None):
    """Gradients of ha_la_gated_norm from dy (like x).  Returns (dx, dw, dz); dz is None without a gate."""
    r = binding._native().gated_norm_backward(dy, x, w, z, _ACTIVATIONS.get(activation), eps, dx, dw, dz, workspace, stream)
    if r.__class__ is tuple:
        return r
    if r is not None:
        raise HaLaError(r, "ha_la_gated_norm_backward")
    import torch

    act, eps = _activation(activation), _eps(eps)
    dtype, rows, cols = _rows_of("ha_la_gated_norm_backward", x, w)
    _as(dy, x, "dy", x.shape)
    if z is not None:
        _as(z, x, "z", x.shape)
    for t, name in ((dx, "dx"), (dz, "dz")):
        _out(t, x, name)
    _check_room("dw", dw, x, torch.float32, cols)
    _check_room("workspace", workspace, x, None, 0)
    with _On(stream, x) as on:
        dx = on.new(dx, x.shape, x.dtype)
        dw = on.new(dw, (cols,), torch.float32)
        dz = on.new(dz, x.shape, x.dtype) if z is not None else None
        args = ha_la_gated_norm_args(dtype=dtype, activation=act, rows=rows, cols=cols, eps=eps, x=_ptr(x), w=_ptr(w), z=_ptr(z), dy=_ptr(dy),
                                     dx=_ptr(dx), dz=_ptr(dz), dw=_ptr(dw))
        ws = on.scratch(workspace, ha_la_gated_norm_workspace_bytes(args))
        args.workspace, args.workspace_bytes = _aligned_part(ws.data_ptr(), ws.numel() * ws.element_size())
        on.call("ha_la_gated_norm_backward", args)
    return dx, dw, dz


def ha_la_add_norm(x, r, w, *, w_post=None, scale=1.0, eps=1e-6, y=None, r_out=None, stream=None):
    """f = x, or x / rms(x) * w_post; r_out = r + scale * f; y = r_out / rms(r_out) * w, over the last dimension.

    x, r : [.., cols] bf16 or fp32, contiguous    w, w_post : fp32 [cols]    r_out may be r itself.  Returns (y, r_out).
    """
    res = binding._native().add_norm(x, r, w, w_post, scale, eps, y, r_out, stream)
    if res.__class__ is tuple:
        return res
    if res is not None:
        raise HaLaError(res, "ha_la_add_norm")
    import torch

    scale, eps = _float(scale, "scale"), _eps(eps)
    dtype, rows, cols = _rows_of("ha_la_add_norm", x, w)
    _as(r, x, "r", x.shape)
    if w_post is not None:
        _as(w_post, x, "w_post", (cols,), torch.float32)
    for t, name in ((y, "y"), (r_out, "r_out")):
        _out(t, x, name)
    with _On(stream, x) as on:
        y, r_out = on.new(y, x.shape, x.dtype), on.new(r_out, x.shape, x.dtype)
        on.call("ha_la_add_norm", ha_la_add_norm_args(dtype=dtype, cols=cols, rows=rows, scale=scale, eps=eps, x=_ptr(x), r=_ptr(r),
                                                      w=_ptr(w), w_post=_ptr(w_post), y=_ptr(y), r_out=_ptr(r_out)))
    return y, r_out


def ha_la_add_norm_backward(dy, dr_out, x, r_out, w, *, w_post=None, scale=1.0, eps=1e-6, dx=None, dr=None, dw=None, dw_post=None, workspace=None,
                            stream=None):
    """Gradients of ha_la_add_norm from dy and dr_out (what r_out has from elsewhere, or None), with x and r_out as the forward pass left
    them.  Returns (dx, dr, dw, dw_post); dw_post is None without w_post."""
    res = binding._native().add_norm_backward(dy, dr_out, x, r_out, w, w_post, scale, eps, dx, dr, dw, dw_post, workspace, stream)
    if res.__class__ is tuple:
        return res
    if res is not None:
        raise HaLaError(res, "ha_la_add_norm_backward")
    import torch

    scale, eps = _float(scale, "scale"), _eps(eps)
    dtype, rows, cols = _rows_of("ha_la_add_norm_backward", x, w)
    for t, name in ((dy, "dy"), (r_out, "r_out")):
        _as(t, x, name, x.shape)
    if dr_out is not None:
        _as(dr_out, x, "dr_out", x.shape)
    if w_post is not None:
        _as(w_post, x, "w_post", (cols,), torch.float32)
    for t, name in ((dx, "dx"), (dr, "dr")):
        _out(t, x, name)
    _check_room("dw", dw, x, torch.float32, cols)
    _check_room("dw_post", dw_post, x, torch.float32, cols)
    _check_room("workspace", workspace, x, None, 0)
    with _On(stream, x) as on:
        dx, dr = on.new(dx, x.shape, x.dtype), on.new(dr, x.shape, x.dtype)
        dw = on.new(dw, (cols,), torch.float32)
        dw_post = on.new(dw_post, (cols,), torch.float32) if w_post is not None else None
        args = ha_la_add_norm_args(dtype=dtype, cols=cols, rows=rows, scale=scale, eps=eps, x=_ptr(x), w=_ptr(w), w_post=_ptr(w_post),
                                   r_out=_ptr(r_out), dy=_ptr(dy), dr_out=_ptr(dr_out), dx=_ptr(dx), dr=_ptr(dr), dw=_ptr(dw), dw_post=_ptr(dw_post))
        ws = on.scratch(workspace, ha_la_add_norm_workspace_bytes(args))
        args.workspace, args.workspace_bytes = _aligned_part(ws.data_ptr(), ws.numel() * ws.element_size())
        on.call("ha_la_add_norm_backward", args)
    return dx, dr, dw, dw_post
