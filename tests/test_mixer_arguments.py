"""What the mixers' entry points refuse, and the host-only answers.  No GPU: tensors with nothing behind them, in one process of its own, and plain structs."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_2609_32114_b200 as ha
from paper_2609_32114_b200 import build, mixer
from tests.test_layer_arguments import _fields

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

REFUSED = {
    "conv.x_fp16": "conv(x=e(2, 70, 64).half())", "conv.x_every_other": "conv(x=e(2, 70, 128)[..., ::2])", "conv.x_expanded": "conv(x=e(2, 1, 64).expand(2, 70, 64))",
    "conv.x_padded_rows": "conv(x=e(2, 80, 64)[:, :70])", "conv.x_no_channel": "conv(x=e(2, 70, 0), w=f(0, 4), bias=None)", "conv.x_four_dims": "conv(x=e(2, 7, 10, 64))",
    "conv.w_bf16": "conv(w=e(64, 4))", "conv.w_taps": "conv(w=f(64, 5))", "conv.w_one_tap": "conv(w=f(64, 1))", "conv.w_short": "conv(w=f(63, 4))", "conv.w_transposed": "conv(w=f(4, 64).t())",
    "conv.bias_short": "conv(bias=f(63))", "conv.bias_cpu": "conv(bias=f(64, device='cpu'))", "conv.activation": "conv(activation='sigmoid')",
    "conv.h0_short": "conv(h0=e(2, 2, 64))", "conv.h0_fp32": "conv(h0=f(2, 3, 64))", "conv.y_short": "conv(y=e(2, 69, 64))", "conv.hT_fp32": "conv(hT=f(2, 3, 64))",
    "conv.cu_seqlens_rows": "conv(cu_seqlens=i(3))", "conv.cu_seqlens_int64": "conv(x=e(1, 70, 64), cu_seqlens=i(3).long())", "conv.cu_seqlens_one": "conv(x=e(1, 70, 64), cu_seqlens=i(1))",
    "conv.status_word_short": "conv(status_word=torch.zeros(1, dtype=torch.uint8, device='cuda'))",
    "conv_back.dy_strided": "conv_back(dy=e(2, 70, 128)[..., :64])", "conv_back.dy_short": "conv_back(dy=e(2, 69, 64))", "conv_back.dx_fp32": "conv_back(dx=f(2, 70, 64))",
    "conv_back.dw_short": "conv_back(dw=f(64, 3))", "conv_back.db_bf16": "conv_back(db=e(64))", "conv_back.dh0_short": "conv_back(dh0=e(1, 3, 64))", "conv_back.dhT_fp32": "conv_back(dhT=f(2, 3, 64))",
    "conv_back.workspace_strided": "conv_back(workspace=torch.empty(1 << 20, dtype=torch.uint8, device='cuda')[::2])",
    "conv_step.x_rows": "conv_step(x=e(1, 5, 64))", "conv_step.state_fp32": "conv_step(state=f(5, 3, 64))", "conv_step.state_short": "conv_step(state=e(4, 3, 64))",
    "conv_step.state_out_short": "conv_step(state_out=e(5, 2, 64))", "conv_step.y_short": "conv_step(y=e(4, 64))",
    "scan.x_fp16": "scan(x=e(2, 70, 64).half())", "scan.dt_fp32": "scan(dt=f(2, 70, 64))", "scan.dt_tokens": "scan(dt=e(2, 69, 64))", "scan.dt_padded_rows": "scan(dt=e(2, 80, 64)[:, :70])",
    "scan.A_bf16": "scan(A=e(64, 16))", "scan.A_states": "scan(A=f(64, 15))", "scan.B_states": "scan(B=e(2, 70, 1, 65))", "scan.B_no_state": "scan(B=e(2, 70, 1, 0))",
    "scan.B_groups": "scan(B=e(2, 70, 3, 16))", "scan.C_groups": "scan(C=e(2, 70, 2, 16))", "scan.C_transposed": "scan(C=e(2, 70, 16, 1).transpose(2, 3)[..., ::1].expand(2, 70, 1, 16)[:, ::1].flip(1)[..., ::2])",
    "scan.D_short": "scan(D=f(63))", "scan.z_fp32": "scan(z=f(2, 70, 64))", "scan.dt_bias_bf16": "scan(dt_bias=e(64))", "scan.h0_short": "scan(h0=f(1, 64, 16))", "scan.h0_bf16": "scan(h0=e(2, 64, 16))",
    "scan.hT_transposed": "scan(hT=f(2, 16, 64).transpose(1, 2))", "scan.y_fp32": "scan(y=f(2, 70, 64))", "scan.cu_seqlens_rows": "scan(cu_seqlens=i(3))",
    "scan_back.dy_strided": "scan_back(dy=e(2, 70, 128)[..., :64])", "scan_back.dx_short": "scan_back(dx=e(1, 70, 64))", "scan_back.ddt_fp32": "scan_back(ddt=f(2, 70, 64))",
    "scan_back.dA_short": "scan_back(dA=f(64, 15))", "scan_back.dB_fp32": "scan_back(dB=f(2, 70, 1, 16))", "scan_back.dC_short": "scan_back(dC=e(2, 70, 1, 15))", "scan_back.dD_bf16": "scan_back(dD=e(64))",
    "scan_back.dz_short": "scan_back(dz=e(2, 70, 63))", "scan_back.ddt_bias_short": "scan_back(ddt_bias=f(63))", "scan_back.dh0_bf16": "scan_back(dh0=e(2, 64, 16))", "scan_back.dhT_short": "scan_back(dhT=f(2, 64, 15))",
    "scan_step.x_rows": "scan_step(x=e(1, 5, 64))", "scan_step.state_bf16": "scan_step(state=e(5, 64, 16))", "scan_step.state_out_short": "scan_step(state_out=f(4, 64, 16))", "scan_step.dt_rows": "scan_step(dt=e(4, 64))",
    "prompt.q_fp16": "prompt(q=e(2, 70, 4, 192).half())", "prompt.q_heads_apart": "prompt(q=e(2, 70, 8, 192)[:, :, ::2])", "prompt.kr_wide": "prompt(kr=e(2, 70, 192))", "prompt.kr_fp32": "prompt(kr=f(2, 70, 64))",
    "prompt.kr_padded_rows": "prompt(kr=e(2, 80, 64)[:, :70])", "prompt.kn_heads": "prompt(kn=e(2, 70, 3, 128))", "prompt.kn_fp32": "prompt(kn=f(2, 70, 4, 128))",
    "prompt.kn_every_other": "prompt(kn=e(2, 70, 4, 256)[..., ::2])", "prompt.v_tokens": "prompt(v=e(2, 69, 4, 128))", "prompt.q_channels": "prompt(kn=e(2, 70, 4, 64))", "prompt.o_short": "prompt(o=e(2, 69, 4, 128))",
    "prompt.lse_bf16": "prompt(lse=e(2, 70, 4))", "prompt.scale_nan": "prompt(scale=float('nan'))", "prompt.cu_seqlens_rows": "prompt(cu_seqlens=i(3))", "prompt.cu_seqlens_k_alone": "prompt(cu_seqlens_k=i(3))",
    "prompt.cu_seqlens_k_short": "packed(cu_seqlens=i(3), cu_seqlens_k=i(4))", "prompt.kr_tokens": "packed(cu_seqlens=i(3), kr=e(1, 80, 64))",
    "token.cache_beside_fp32": "token(q=f(3, 1, 16, 576))", "token.q_strided": "token(q=e(3, 2, 16, 576)[:, ::2])", "token.cache_fp32": "token(cache=f(9, 64, 576))", "token.cache_row": "token(cache=e(9, 64, 512))",
    "token.q_page_of_48": "token(cache=e(9, 48, 576))", "token.cache_strided": "token(cache=e(9, 64, 640)[..., :576])", "token.page_table_int64": "token(page_table=i(3, 4).long())",
    "token.page_table_rows": "token(page_table=i(2, 4))", "token.lengths_short": "token(lengths=i(2))", "token.lengths_float": "token(lengths=f(3))", "token.d_latent_zero": "token(d_latent=0)",
    "token.d_latent_wide": "token(d_latent=577)", "token.o_short": "token(o=e(3, 1, 15, 512))", "token.lse_short": "token(lse=f(3, 1, 15))", "token.scale_nan": "token(scale=float('nan'))",
    "token.workspace_strided": "token(workspace=torch.empty(1 << 20, dtype=torch.uint8, device='cuda')[::2])",
    "cpu.conv": "conv(x=torch.zeros(1, 3, 64))", "cpu.scan": "scan(x=torch.zeros(1, 3, 64))", "cpu.prompt": "prompt(q=torch.zeros(1, 3, 4, 192))", "cpu.token": "token(q=torch.zeros(3, 1, 16, 576))",
}
CODE = """
import sys, torch
import paper_2609_32114_b200 as ha
from torch._subclasses.fake_tensor import FakeTensorMode
ha.binding._native()
def e(*s, device="cuda"): return torch.empty(*s, dtype=torch.bfloat16, device=device)
def f(*s, device="cuda"): return torch.empty(*s, dtype=torch.float32, device=device)
def i(*s): return torch.zeros(*s, dtype=torch.int32, device="cuda")
def conv(**kw):
    a = dict(x=e(2, 70, 64), w=f(64, 4), bias=f(64)) | kw
    return ha.ha_la_conv(a.pop("x"), a.pop("w"), **a)
def conv_back(**kw):
    a = dict(dy=e(2, 70, 64), x=e(2, 70, 64), w=f(64, 4), bias=f(64)) | kw
    return ha.ha_la_conv_backward(a.pop("dy"), a.pop("x"), a.pop("w"), **a)
def conv_step(**kw):
    a = dict(x=e(5, 64), w=f(64, 4), state=e(5, 3, 64)) | kw
    return ha.ha_la_conv_decode(a.pop("x"), a.pop("w"), a.pop("state"), **a)
S = ("x", "dt", "A", "B", "C")
def scan_args(*lead): return dict(x=e(*lead, 64), dt=e(*lead, 64), A=f(64, 16), B=e(*lead, 1, 16), C=e(*lead, 1, 16), D=f(64), z=e(*lead, 64), dt_bias=f(64))
def scan(**kw):
    a = scan_args(2, 70) | kw
    return ha.ha_la_scan(*[a.pop(n) for n in S], **a)
def scan_back(**kw):
    a = scan_args(2, 70) | dict(dy=e(2, 70, 64)) | kw
    return ha.ha_la_scan_backward(a.pop("dy"), *[a.pop(n) for n in S], **a)
def scan_step(**kw):
    a = scan_args(5) | dict(state=f(5, 64, 16)) | kw
    return ha.ha_la_scan_decode(*[a.pop(n) for n in S], a.pop("state"), **a)
def prompt(B=2, **kw):
    a = dict(q=e(B, 70, 4, 192), kn=e(B, 70, 4, 128), kr=e(B, 70, 64), v=e(B, 70, 4, 128)) | kw
    return ha.ha_la_latent_prefill(*[a.pop(n) for n in ("q", "kn", "kr", "v")], **a)
def packed(**kw): return prompt(B=1, **kw)
def token(**kw):
    a = dict(q=e(3, 1, 16, 576), cache=e(9, 64, 576), page_table=i(3, 4), lengths=i(3)) | kw
    return ha.ha_la_latent_decode(*[a.pop(n) for n in ("q", "cache", "page_table", "lengths")], **a)
with FakeTensorMode():
    for line in sys.stdin.read().splitlines():
        name, call = line.split("|")
        try:
            eval(call)
            print(name, "returned")
        except Exception as x:
            print(name, type(x).__name__, str(x).splitlines()[0][:200])
"""
PLAIN = ["conv", "conv_back", "conv_step", "scan", "scan_back", "scan_step", "prompt", "packed", "token"]


@pytest.fixture(scope="module")
def outcomes():
    calls = [f"{n}|{c}" for n, c in REFUSED.items()] + [f"plain.{n}|{n}()" for n in PLAIN]
    r = subprocess.run([sys.executable, "-c", CODE], input="\n".join(calls), cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return dict(line.split(" ", 1) for line in r.stdout.splitlines())


@pytest.mark.parametrize("name", list(REFUSED))
def test_refused(outcomes, name):
    if name.startswith("cpu."):
        assert "needs CUDA tensors" in outcomes[name]
        return
    what = name.split(".")[1]
    if what == "cu_seqlens_k_alone":
        assert outcomes[name] == "ValueError cu_seqlens_k without cu_seqlens"
        return
    known = ("cu_seqlens_k", "cu_seqlens", "status_word", "state_out", "dt_bias", "ddt_bias", "page_table", "d_latent")
    what = next((k for k in known if what.startswith(k)), what.split("_")[0])
    assert outcomes[name].startswith(f"ValueError {what}:"), outcomes[name]


@pytest.mark.parametrize("name", PLAIN)
def test_the_plain_call_gets_as_far_as_the_driver(outcomes, name):
    """What the refused calls are changes of is not refused for its arguments: an error of torch's or the library's, not the process's end."""
    assert "ValueError" not in outcomes[f"plain.{name}"], outcomes[f"plain.{name}"]


@pytest.fixture(scope="module")
def lib():
    build.build()
    return ha.load_library()


@pytest.mark.parametrize("struct", ["ha_la_conv_args", "ha_la_scan_args", "ha_la_latent_prefill_args", "ha_la_latent_decode_args"])
def test_structs_are_those_of_the_header(struct):
    assert [(n, ctypes.sizeof(t) == 8) for n, t in getattr(mixer, struct)._fields_] == _fields(struct)


def _conv(**kw):
    return mixer.ha_la_conv_args(**{**dict(dtype=0, batch=2, seqlen=70, channels=64, taps=4, activation=0, x=16, w=16, y=16, dy=16, dx=16, dw=16), **kw})


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 1), (dict(batch=0), 1), (dict(seqlen=-1), 1), (dict(channels=0), 1), (dict(taps=0), 1), (dict(taps=1), 2), (dict(taps=5), 2),
                                       (dict(activation=1), 1), (dict(activation=3), 1), (dict(x_stride=-1), 1), (dict(x_stride=63), 1), (dict(num_seqs=3), 1),
                                       (dict(batch=1, num_seqs=-1, cu_seqlens=16), 1), (dict(batch=1, num_seqs=2, cu_seqlens=16, max_seqlen=-1), 1), (dict(batch=1 << 20, seqlen=1 << 20), 2),
                                       (dict(channels=(1 << 24) + 1), 2)])
def test_convolutions_that_the_library_refuses(lib, kw, status):
    n = ctypes.c_size_t(0)
    assert lib.ha_la_conv_workspace_bytes(ctypes.byref(_conv(**kw)), ctypes.byref(n)) == status
    assert lib.ha_la_conv(ctypes.byref(_conv(**kw)), None) == status == lib.ha_la_conv_backward(ctypes.byref(_conv(**kw)), None)


@pytest.mark.parametrize("kw", [dict(x=0), dict(x=17), dict(w=0), dict(w=18), dict(y=0, dx=0), dict(bias=17), dict(batch=1, num_seqs=2)])
def test_convolutions_with_pointers_that_do_not_fit(lib, kw):
    assert lib.ha_la_conv(ctypes.byref(_conv(**kw)), None) == 1 == lib.ha_la_conv_backward(ctypes.byref(_conv(**kw)), None)


def test_convolutions_on_their_own(lib):
    assert lib.ha_la_conv(ctypes.byref(_conv(h0=16, hT=16)), None) == 1
    assert lib.ha_la_conv_backward(ctypes.byref(_conv()), None) == 3
    assert lib.ha_la_conv_backward(ctypes.byref(_conv(dw=0)), None) == 1
    assert lib.ha_la_conv_decode(ctypes.byref(_conv()), None) == 1 == lib.ha_la_conv_decode(ctypes.byref(_conv(seqlen=1)), None)
    assert lib.ha_la_conv_decode(ctypes.byref(_conv(batch=0, seqlen=1)), None) == 0
    for name in ("conv", "conv_backward", "conv_decode", "scan", "scan_backward", "scan_decode", "latent_prefill", "latent_decode"):
        assert getattr(lib, f"ha_la_{name}")(None, None) == 1
    a, b = (ha.ha_la_conv_workspace_bytes(_conv(seqlen=n, channels=4096)) for n in (1, 8192))
    assert a % 256 == 0 and a <= b and b >= 5 * 4096 * 4


def _scan(**kw):
    return mixer.ha_la_scan_args(**{**dict(dtype=0, batch=2, seqlen=70, channels=64, states=16, groups=2, softplus=1, x=16, dt=16, B=16, C=16, A=16, y=16, dy=16, dx=16, ddt=16, dB=16,
                                           dC=16, dA=16), **kw})


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 1), (dict(batch=0), 1), (dict(seqlen=-1), 1), (dict(channels=0), 1), (dict(states=0), 1), (dict(states=65), 2), (dict(groups=0), 1),
                                       (dict(groups=3), 1), (dict(softplus=2), 1), (dict(x_stride=63), 1), (dict(dt_stride=-1), 1), (dict(z_stride=1), 1), (dict(b_stride=31), 1), (dict(c_stride=31), 1),
                                       (dict(num_seqs=3), 1), (dict(batch=1, num_seqs=2, cu_seqlens=16, max_seqlen=-1), 1), (dict(batch=1 << 20, seqlen=1 << 20), 2)])
def test_scans_that_the_library_refuses(lib, kw, status):
    n = ctypes.c_size_t(0)
    assert lib.ha_la_scan_workspace_bytes(ctypes.byref(_scan(**kw)), 0, ctypes.byref(n)) == status == lib.ha_la_scan_workspace_bytes(ctypes.byref(_scan(**kw)), 1, ctypes.byref(n))
    assert lib.ha_la_scan(ctypes.byref(_scan(**kw)), None) == status == lib.ha_la_scan_backward(ctypes.byref(_scan(**kw)), None)


@pytest.mark.parametrize("kw,status", [(dict(), 3), (dict(x=0), 1), (dict(x=17), 1), (dict(dt=0), 1), (dict(B=0), 1), (dict(C=0), 1), (dict(A=0), 1), (dict(A=18), 1), (dict(h0=18), 1), (dict(y=0, dx=0), 1),
                                       (dict(workspace=128, workspace_bytes=1 << 40), 3), (dict(workspace=256, workspace_bytes=100), 3), (dict(batch=1, num_seqs=2), 1)])
def test_scans_with_pointers_that_do_not_fit(lib, kw, status):
    assert lib.ha_la_scan(ctypes.byref(_scan(**kw)), None) == status == lib.ha_la_scan_backward(ctypes.byref(_scan(**kw)), None)


def test_scans_on_their_own(lib):
    assert lib.ha_la_scan_backward(ctypes.byref(_scan(z=16)), None) == 1 == lib.ha_la_scan_backward(ctypes.byref(_scan(D=16)), None) == lib.ha_la_scan_backward(ctypes.byref(_scan(dt_bias=16)), None)
    assert lib.ha_la_scan_decode(ctypes.byref(_scan()), None) == 1 == lib.ha_la_scan_decode(ctypes.byref(_scan(seqlen=1)), None)
    assert lib.ha_la_scan_decode(ctypes.byref(_scan(batch=0, seqlen=1)), None) == 0
    small, large = ha.ha_la_scan_workspace_bytes(_scan()), ha.ha_la_scan_workspace_bytes(_scan(), backward=True)
    assert small % 256 == 0 and small < large and large >= 140 // 8 * 64 * 16 * 4
    # a workspace asked for without its offsets is enough for the call with them
    long = dict(batch=1, seqlen=5000, num_seqs=3)
    assert ha.ha_la_scan_workspace_bytes(_scan(**long)) == ha.ha_la_scan_workspace_bytes(_scan(**long, cu_seqlens=16)) > 4096


def _prompt(**kw):
    return mixer.ha_la_latent_prefill_args(**{**dict(dtype=0, batch=2, seqlen=70, seqlen_k=70, num_heads=4, d_nope=128, d_rope=64, d_v=128, scale=1.0, q=16, kn=16, kr=16, v=16, o=16), **kw})


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 1), (dict(batch=0), 1), (dict(seqlen=-1), 1), (dict(seqlen_k=-1), 1), (dict(num_heads=0), 1), (dict(num_heads=65536), 2), (dict(d_nope=0), 1),
                                       (dict(d_nope=257), 2), (dict(d_rope=-1), 1), (dict(d_rope=129), 2), (dict(d_v=0), 1), (dict(d_v=257), 2), (dict(scale=float("nan")), 1), (dict(q_stride=767), 1),
                                       (dict(kn_stride=127), 1), (dict(kr_stride=63), 1), (dict(v_head_stride=127), 1), (dict(num_seqs=3), 1), (dict(batch=1 << 20, seqlen=1 << 20), 2)])
def test_prompts_that_the_library_refuses(lib, kw, status):
    assert ha.ha_la_latent_prefill_path(_prompt(**kw)) is None
    assert lib.ha_la_latent_prefill(ctypes.byref(_prompt(**kw)), None) == status


@pytest.mark.parametrize("kw", [dict(q=0), dict(q=17), dict(o=0), dict(kn=0), dict(kr=0), dict(v=0), dict(lse=18), dict(batch=1, cu_seqlens=16, num_seqs=2), dict(batch=1, cu_seqlens_k=16), dict(batch=1, num_seqs=2)])
def test_prompts_with_pointers_that_do_not_fit(lib, kw):
    assert lib.ha_la_latent_prefill(ctypes.byref(_prompt(**kw)), None) == 1


def test_which_path_a_prompt_takes(lib):
    assert ha.ha_la_latent_prefill_path(_prompt()) == "tc"
    for kw in (dict(dtype=1), dict(d_rope=32), dict(scale=-1.0), dict(scale=0.0), dict(kr_stride=68), dict(q=8), dict(v=24), dict(kn_head_stride=132)):
        assert ha.ha_la_latent_prefill_path(_prompt(**kw)) == "simt"
    assert lib.ha_la_latent_prefill(ctypes.byref(_prompt(seqlen=0)), None) == 0


def _token(**kw):
    return mixer.ha_la_latent_decode_args(**{**dict(dtype=0, num_seqs=3, new_tokens=1, num_heads=16, d_latent=512, d_rope=64, page_size=64, num_pages=9, max_pages=4, scale=1.0, q=16, cache=16,
                                                    page_table=16, lengths=16, o=16), **kw})


@pytest.mark.parametrize("kw,status", [(dict(dtype=2), 1), (dict(num_seqs=-1), 1), (dict(new_tokens=0), 1), (dict(num_heads=0), 1), (dict(d_latent=0), 1), (dict(d_latent=513), 2), (dict(d_rope=-1), 1),
                                       (dict(d_rope=129), 2), (dict(page_size=0), 1), (dict(page_size=48), 1), (dict(num_pages=-1), 1), (dict(max_pages=-1), 1), (dict(scale=float("nan")), 1),
                                       (dict(new_tokens=1 << 20, num_heads=2), 2), (dict(num_pages=1 << 30, page_size=64), 2), (dict(num_seqs=1 << 30, num_heads=16), 2)])
def test_tokens_that_the_library_refuses(lib, kw, status):
    n = ctypes.c_size_t(0)
    assert ha.ha_la_latent_decode_path(_token(**kw)) is None
    assert lib.ha_la_latent_decode_workspace_bytes(ctypes.byref(_token(**kw)), ctypes.byref(n)) == status == lib.ha_la_latent_decode(ctypes.byref(_token(**kw)), None)


@pytest.mark.parametrize("kw,status", [(dict(), 3), (dict(q=0), 1), (dict(q=17), 1), (dict(cache=0), 1), (dict(page_table=0), 1), (dict(page_table=18), 1), (dict(lengths=0), 1), (dict(o=0), 1), (dict(lse=18), 1),
                                       (dict(workspace=128, workspace_bytes=1 << 40), 3), (dict(workspace=256, workspace_bytes=100), 3)])
def test_tokens_with_pointers_that_do_not_fit(lib, kw, status):
    assert lib.ha_la_latent_decode(ctypes.byref(_token(**kw)), None) == status


def test_which_path_tokens_take(lib):
    assert ha.ha_la_latent_decode_path(_token()) == "tc" and ha.ha_la_latent_decode_workspace_bytes(_token()) > 1 << 20
    for kw in (dict(dtype=1), dict(d_rope=32), dict(page_size=8), dict(scale=0.0), dict(cache=8)):
        assert ha.ha_la_latent_decode_path(_token(**kw)) == "simt"
    assert lib.ha_la_latent_decode(ctypes.byref(_token(num_seqs=0)), None) == 0
