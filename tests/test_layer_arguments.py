"""What the entry points next to the delta rule's refuse, and the host-only answers.  No GPU: tensors with nothing behind them, in one
process of its own, and plain structs."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

import paper_2609_32114_b200 as ha
from paper_2609_32114_b200 import binding, build, layer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

REFUSED = {
    "gla.q_fp16": "gla(q=e(2, 70, 2, 128).half())", "gla.q_strided": "gla(q=e(2, 70, 2, 256)[..., ::2])", "gla.k_heads": "gla(k=e(2, 70, 1, 128))",
    "gla.k_fp32": "gla(k=f(2, 70, 2, 128))", "gla.k_tokens": "gla(k=e(2, 71, 2, 128))", "gla.v_tokens": "gla(v=e(2, 69, 4, 128))", "gla.v_dim": "gla(v=e(2, 70, 4, 64))",
    "gla.g_heads": "gla(g=f(2, 70, 2))", "gla.g_bf16": "gla(g=e(2, 70, 4))", "gla.g_cpu": "gla(g=f(2, 70, 4, device='cpu'))",
    "gla.h0_short": "gla(h0=f(1, 4, 128, 128))", "gla.h0_bf16": "gla(h0=e(2, 4, 128, 128))", "gla.h0_transposed": "gla(h0=f(2, 4, 128, 128).transpose(2, 3))",
    "gla.o_short": "gla(o=e(2, 69, 4, 128))", "gla.o_fp32": "gla(o=f(2, 70, 4, 128))", "gla.hT_short": "gla(hT=f(2, 3, 128, 128))",
    "gla.cu_seqlens_int64": "gla(batch=1, cu_seqlens=torch.zeros(3, dtype=torch.int64, device='cuda'))",
    "gla.cu_seqlens_rows": "gla(cu_seqlens=torch.zeros(3, dtype=torch.int32, device='cuda'))",
    "gla.cu_seqlens_one": "gla(batch=1, cu_seqlens=torch.zeros(1, dtype=torch.int32, device='cuda'))",
    "gla.status_word_short": "gla(status_word=torch.zeros(3, dtype=torch.uint8, device='cuda'))",
    "gla.workspace_strided": "gla(workspace=torch.empty(1 << 23, dtype=torch.uint8, device='cuda')[::2])", "gla.scale_nan": "gla(scale=float('nan'))",
    "back.do_short": "back(do=e(2, 69, 4, 128))", "back.do_fp32": "back(do=f(2, 70, 4, 128))", "back.dhT_short": "back(dhT=f(1, 4, 128, 128))",
    "back.dq_short": "back(dq=e(1, 70, 2, 128))", "back.dk_fp32": "back(dk=f(2, 70, 2, 128))", "back.dv_strided": "back(dv=e(2, 70, 8, 128)[:, :, ::2])",
    "back.dg_bf16": "back(dg=e(2, 70, 4))", "back.dh0_short": "back(dh0=f(2, 4, 64, 128))", "back.k_heads": "back(k=e(2, 70, 1, 128))",
    "step.q_strided": "step(q=e(3, 4, 128)[:, ::2])", "step.k_rows": "step(k=e(2, 2, 128))", "step.v_dim": "step(v=e(3, 4, 64))", "step.g_heads": "step(g=f(3, 2))",
    "step.state_short": "step(state=f(2, 4, 128, 128))", "step.state_bf16": "step(state=e(3, 4, 128, 128))", "step.state_out_short": "step(state_out=f(3, 2, 128, 128))",
    "step.o_fp32": "step(o=f(3, 4, 128))", "step.scale_nan": "step(scale=float('nan'))",
    "gated.x_fp16": "gated(x=e(5, 64).half())", "gated.x_strided": "gated(x=e(5, 128)[:, ::2])", "gated.w_short": "gated(w=f(63))", "gated.w_bf16": "gated(w=e(64))",
    "gated.z_fp32": "gated(z=f(5, 64))", "gated.z_rows": "gated(z=e(4, 64))", "gated.y_short": "gated(y=e(4, 64))", "gated.eps_negative": "gated(eps=-1.0)",
    "gated.eps_nan": "gated(eps=float('nan'))", "gated.activation": "gated(activation='relu')",
    "gated_back.dy_rows": "gated_back(dy=e(4, 64))", "gated_back.dx_fp32": "gated_back(dx=f(5, 64))", "gated_back.dw_short": "gated_back(dw=f(63))",
    "gated_back.dz_short": "gated_back(dz=e(5, 63))", "gated_back.activation": "gated_back(activation=None)",
    "add.r_fp32": "add(r=f(5, 64))", "add.r_rows": "add(r=e(6, 64))", "add.w_post_short": "add(w_post=f(32))", "add.y_strided": "add(y=e(5, 128)[:, ::2])",
    "add.r_out_short": "add(r_out=e(4, 64))", "add.scale_nan": "add(scale=float('nan'))",
    "add_back.dr_out_fp32": "add_back(dr_out=f(5, 64))", "add_back.r_out_rows": "add_back(r_out=e(4, 64))", "add_back.dr_short": "add_back(dr=e(4, 64))",
    "add_back.dw_bf16": "add_back(dw=e(64))", "add_back.dw_post_short": "add_back(w_post=f(64), dw_post=f(63))",
    "cpu.gla": "gla(**{n: torch.zeros(1, 3, 1, 64) for n in 'qkv'}, g=torch.zeros(1, 3, 1))", "cpu.gated": "gated(x=torch.zeros(2, 64), z=None)",
}
CODE = """
import sys, torch
import paper_2609_32114_b200 as ha
from torch._subclasses.fake_tensor import FakeTensorMode
ha.binding._native()
def e(*s, device="cuda"): return torch.empty(*s, dtype=torch.bfloat16, device=device)
def f(*s, device="cuda"): return torch.empty(*s, dtype=torch.float32, device=device)
def gla(batch=2, **kw):
    a = dict(q=e(batch, 70, 2, 128), k=e(batch, 70, 2, 128), v=e(batch, 70, 4, 128), g=f(batch, 70, 4)) | kw
    return ha.ha_la_gla_prefill(*[a.pop(n) for n in "qkvg"], **a)
def back(**kw):
    a = dict(do=e(2, 70, 4, 128), q=e(2, 70, 2, 128), k=e(2, 70, 2, 128), v=e(2, 70, 4, 128), g=f(2, 70, 4)) | kw
    return ha.ha_la_gla_backward(a.pop("do"), *[a.pop(n) for n in "qkvg"], **a)
def step(**kw):
    a = dict(q=e(3, 2, 128), k=e(3, 2, 128), v=e(3, 4, 128), g=f(3, 4), state=f(3, 4, 128, 128)) | kw
    return ha.ha_la_gla_decode(*[a.pop(n) for n in ("q", "k", "v", "g", "state")], **a)
def gated(**kw):
    a = dict(x=e(5, 64), w=f(64), z=e(5, 64)) | kw
    return ha.ha_la_gated_norm(a.pop("x"), a.pop("w"), a.pop("z"), **a)
def gated_back(**kw):
    a = dict(dy=e(5, 64), x=e(5, 64), w=f(64), z=e(5, 64)) | kw
    return ha.ha_la_gated_norm_backward(a.pop("dy"), a.pop("x"), a.pop("w"), a.pop("z"), **a)
def add(**kw):
    a = dict(x=e(5, 64), r=e(5, 64), w=f(64)) | kw
    return ha.ha_la_add_norm(a.pop("x"), a.pop("r"), a.pop("w"), **a)
def add_back(**kw):
    a = dict(dy=e(5, 64), dr_out=e(5, 64), x=e(5, 64), r_out=e(5, 64), w=f(64)) | kw
    return ha.ha_la_add_norm_backward(*[a.pop(n) for n in ("dy", "dr_out", "x", "r_out", "w")], **a)
with FakeTensorMode():
    for line in sys.stdin.read().splitlines():
        name, call = line.split("|")
        try:
            eval(call)
            print(name, "returned")
        except Exception as x:
            print(name, type(x).__name__, str(x).splitlines()[0][:200])
"""


@pytest.fixture(scope="module")
def outcomes():
    plain = ["plain.%s|%s()" % (n, n) for n in ("gla", "back", "step", "gated", "gated_back", "add", "add_back")]
    calls = [f"{n}|{c}" for n, c in REFUSED.items()] + plain
    r = subprocess.run([sys.executable, "-c", CODE], input="\n".join(calls), cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return dict(line.split(" ", 1) for line in r.stdout.splitlines())


@pytest.mark.parametrize("name", list(REFUSED))
def test_refused(outcomes, name):
    what = name.split(".")[1]
    if name.startswith("cpu."):
        assert "needs CUDA tensors" in outcomes[name]
        return
    known = ("cu_seqlens", "status_word", "state_out", "r_out", "dr_out", "w_post", "dw_post")
    what = next((k for k in known if what.startswith(k)), what.split("_")[0])
    assert outcomes[name].startswith(f"ValueError {what}:"), outcomes[name]


@pytest.mark.parametrize("name", ["gla", "back", "step", "gated", "gated_back", "add", "add_back"])
def test_the_plain_call_gets_as_far_as_the_driver(outcomes, name):
    """What the refused calls are changes of is not refused for its arguments: an error of torch's or the library's, not the process's end."""
    assert "ValueError" not in outcomes[f"plain.{name}"], outcomes[f"plain.{name}"]


@pytest.fixture(scope="module")
def lib():
    build.build()
    return ha.load_library()


def _fields(struct):
    """(name, pointer / 64-bit?) of a struct of the header, in order."""
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ha_la.h")).read(), flags=re.S)
    body = hdr[:hdr.index("} " + struct + ";")].rsplit("typedef struct {", 1)[1]
    out = []
    for decl in body.split(";"):
        decl = decl.strip()
        if decl:
            kind, names = re.match(r"((?:const )?\w+\s*\**)\s*(.*)", decl, re.S).groups()
            out += [(n.strip().lstrip("*"), "*" in kind or "64" in kind or "size_t" in kind) for n in names.split(",")]
    return out


@pytest.mark.parametrize("struct", ["ha_la_gla_args", "ha_la_gated_norm_args", "ha_la_add_norm_args", "ha_la_decode_args"])
def test_structs_are_those_of_the_header(struct):
    want = _fields(struct)
    have = [(n, ctypes.sizeof(t) == 8) for n, t in getattr(layer, struct)._fields_]
    assert have == want


def _gla(**kw):
    return layer.ha_la_gla_args(**{**dict(dtype=0, batch=2, seqlen=300, num_qk_heads=2, num_v_heads=4, d_k=128, d_v=128, scale=1.0), **kw})


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 1), (dict(batch=0), 1), (dict(seqlen=-1), 1), (dict(num_v_heads=3), 1), (dict(num_qk_heads=0), 1),
                                       (dict(d_k=0), 1), (dict(d_v=64), 2), (dict(d_k=96, d_v=96), 2), (dict(scale=float("nan")), 1), (dict(num_seqs=3), 1),
                                       (dict(batch=1, num_seqs=-1, cu_seqlens=16), 1), (dict(batch=1, num_seqs=2, max_seqlen=-1), 1),
                                       (dict(batch=1 << 20, seqlen=1 << 20), 2), (dict(batch=1 << 20, seqlen=1000, num_qk_heads=4096, num_v_heads=4096), 2)])
def test_shapes_that_the_library_refuses(lib, kw, status):
    n = ctypes.c_size_t(0)
    assert lib.ha_la_gla_workspace_bytes(ctypes.byref(_gla(**kw)), 0, ctypes.byref(n)) == status
    assert lib.ha_la_gla_path(ctypes.byref(_gla(**kw))) is None
    assert lib.ha_la_gla_prefill(ctypes.byref(_gla(**kw)), None) == status == lib.ha_la_gla_backward(ctypes.byref(_gla(**kw)), None)


@pytest.mark.parametrize("kw,status", [(dict(), 1), (dict(q=8), 1), (dict(q=16, k=16, v=16, g=16), 1), (dict(q=16, k=16, v=16, g=16, o=16, do_=16, dq=16, dk=16, dv=16, dg=16), 3),
                                       (dict(q=16, k=16, v=16, g=18, o=16, do_=16, dq=16, dk=16, dv=16, dg=16), 1),
                                       (dict(q=16, k=16, v=24, g=16, o=16, do_=16, dq=16, dk=16, dv=16, dg=16), 1),
                                       (dict(q=16, k=16, v=16, g=16, o=16, do_=16, dq=16, dk=16, dv=16, dg=16, workspace=256, workspace_bytes=100), 3),
                                       (dict(q=16, k=16, v=16, g=16, o=16, do_=16, dq=16, dk=16, dv=16, dg=16, workspace=128, workspace_bytes=1 << 40), 3)])
def test_pointers_that_the_library_refuses(lib, kw, status):
    """(addresses that nothing follows: the calls return before they launch)"""
    assert lib.ha_la_gla_prefill(ctypes.byref(_gla(**kw)), None) == status == lib.ha_la_gla_backward(ctypes.byref(_gla(**kw)), None)


def test_workspace_of_the_recurrence(lib):
    small, large = ha.ha_la_gla_workspace_bytes(_gla()), ha.ha_la_gla_workspace_bytes(_gla(), backward=True)
    assert 0 < small < large and small % 256 == 0
    assert ha.ha_la_gla_workspace_bytes(_gla(seqlen=0)) <= small and ha.ha_la_gla_workspace_bytes(_gla(seqlen=0), backward=True) < large
    packed = _gla(batch=1, seqlen=600, num_seqs=2)
    assert ha.ha_la_gla_workspace_bytes(packed) > 0 and ha.ha_la_gla_path(packed) in ("tc", "simt")
    for d in (dict(dtype=1), dict(d_k=64, d_v=64)):
        assert ha.ha_la_gla_path(_gla(**d)) == "simt"


def _gated(**kw):
    return layer.ha_la_gated_norm_args(**{**dict(dtype=0, rows=5, cols=64, eps=1e-6, x=16, w=16, y=16, dy=16, dx=16, dw=16, z=16, dz=16), **kw})


def _add(**kw):
    return layer.ha_la_add_norm_args(**{**dict(dtype=0, rows=5, cols=64, eps=1e-6, scale=1.0, x=16, r=16, w=16, y=16, r_out=16, dy=16, dx=16, dr=16, dw=16), **kw})


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 1), (dict(rows=-1), 1), (dict(cols=0), 1), (dict(cols=16385), 2), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
                                       (dict(rows=1 << 45), 2), (dict(x=17), 1), (dict(w=18), 1), (dict(x=0), 1), (dict(w=0), 1), (dict(dx=0, y=0), 1)])
def test_norms_that_the_library_refuses(lib, kw, status):
    for make, name in ((_gated, "gated"), (_add, "add")):
        if make is _add and "x" in kw:
            kw = {**kw, "r_out": kw["x"], "r": kw["x"]}
        a = make(**kw)
        assert getattr(lib, f"ha_la_{name}_norm")(ctypes.byref(a), None) == status, name
        assert getattr(lib, f"ha_la_{name}_norm_backward")(ctypes.byref(a), None) == status, name


def test_norms_without_their_own_arguments(lib):
    assert lib.ha_la_gated_norm(ctypes.byref(_gated(activation=2)), None) == 1
    assert lib.ha_la_gated_norm_backward(ctypes.byref(_gated(dz=0)), None) == 1
    assert lib.ha_la_gated_norm_backward(ctypes.byref(_gated()), None) == 3
    assert lib.ha_la_add_norm(ctypes.byref(_add(scale=float("nan"))), None) == 1
    assert lib.ha_la_add_norm_backward(ctypes.byref(_add(w_post=16)), None) == 1
    assert lib.ha_la_add_norm_backward(ctypes.byref(_add(dr=0)), None) == 1
    assert lib.ha_la_add_norm_backward(ctypes.byref(_add(workspace=16, workspace_bytes=1 << 30)), None) == 3
    assert lib.ha_la_gated_norm(ctypes.byref(_gated(rows=0, x=0, w=0, y=0)), None) == 0
    for name in ("gla_prefill", "gla_backward", "gla_decode", "gated_norm", "gated_norm_backward", "add_norm", "add_norm_backward"):
        assert getattr(lib, f"ha_la_{name}")(None, None) == 1


def test_workspace_of_the_norms(lib):
    a = ha.ha_la_gated_norm_workspace_bytes(_gated(rows=1 << 20, cols=128))
    assert a % 256 == 0 and a >= 148 * 128 * 4
    assert ha.ha_la_add_norm_workspace_bytes(_add(rows=1 << 20, cols=2048, w_post=16)) == 2 * ha.ha_la_add_norm_workspace_bytes(_add(rows=1 << 20, cols=2048))
