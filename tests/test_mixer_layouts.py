"""States, outputs and gradients of another layout with as many elements: refused, in both halves of the marshalling.  No GPU: tensors with nothing behind them."""
import subprocess
import sys

import pytest

from tests.test_mixer_arguments import CODE, ROOT

REFUSED = {
    "conv.h0": "conv(h0=e(2, 64, 3))", "conv.hT": "conv(hT=e(2, 64, 3))", "conv.y": "conv(y=e(70, 2, 64))",
    "conv.h0_wide": "conv(h0=e(2, 4, 64))", "conv.hT_flat_short": "conv(hT=e(383))", "conv.hT_none": "conv(hT=e(0, 2, 3, 64))", "conv_back.dhT": "conv_back(dhT=e(2, 64, 3))", "conv_back.dh0": "conv_back(dh0=e(2, 64, 3))", "conv_back.h0": "conv_back(h0=e(2, 64, 3))",
    "conv_back.dw": "conv_back(dw=f(4, 64))", "conv_back.dx": "conv_back(dx=e(2, 64, 70))", "conv_step.state": "conv_step(state=e(5, 64, 3))", "conv_step.state_out": "conv_step(state_out=e(5, 64, 3))",
    "conv_step.y": "conv_step(y=e(64, 5))",
    "scan.h0": "scan(h0=f(2, 16, 64))", "scan.hT": "scan(hT=f(2, 16, 64))", "scan.y": "scan(y=e(2, 64, 70))", "scan_back.dhT": "scan_back(dhT=f(2, 16, 64))", "scan_back.dh0": "scan_back(dh0=f(2, 16, 64))",
    "scan_back.dA": "scan_back(dA=f(16, 64))", "scan_back.dB": "scan_back(dB=e(2, 70, 16, 1))", "scan_back.dC": "scan_back(dC=e(2, 1, 70, 16))", "scan_back.ddt": "scan_back(ddt=e(2, 64, 70))",
    "scan_back.dz": "scan_back(dz=e(70, 128))", "scan_step.state": "scan_step(state=f(5, 16, 64))", "scan_step.state_out": "scan_step(state_out=f(5, 16, 64))",
    "prompt.o": "prompt(o=e(2, 4, 70, 128))", "prompt.lse": "prompt(lse=f(2, 4, 70))", "token.o": "token(o=e(3, 16, 1, 512))", "token.lse": "token(lse=f(3, 16, 1))", "conv.y_scalar": "conv(y=torch.empty((), dtype=torch.bfloat16, device='cuda'))",
}
TAKEN = {
    "conv.more_states": "conv(h0=e(7, 3, 64), hT=e(3, 3, 64))", "conv.more_rows": "conv(x=e(1, 70, 64), y=e(1, 90, 64))", "conv.more_batch": "conv(y=e(4, 70, 64))",
    "conv.rows": "conv(y=e(140, 64), h0=e(6, 64), hT=e(1, 2, 3, 64))", "prompt.one": "prompt(B=1, o=e(70, 4, 128), lse=f(80, 4))", "conv.flat": "conv(h0=e(384), y=e(10000), hT=e(384))", "scan_step.flat": "scan_step(state=f(5 * 64 * 16))",
    "conv_back.more": "conv_back(dw=f(80, 4), db=f(100), dx=e(3, 70, 64))", "conv_step.more": "conv_step(state=e(9, 3, 64), y=e(6, 64))", "scan.more": "scan(h0=f(3, 64, 16), y=e(2, 70, 64))",
    "scan_back.more": "scan_back(dA=f(65, 16), dB=e(3, 70, 1, 16))", "scan_step.more": "scan_step(state=f(6, 64, 16))", "prompt.more": "prompt(o=e(3, 70, 4, 128), lse=f(2, 70, 4))",
    "token.more": "token(o=e(4, 1, 16, 512), lse=f(5, 1, 16))", "token.one_sequence": "token(q=e(1, 2, 16, 576), page_table=i(1, 4), lengths=i(1), o=e(1, 3, 16, 512))",
}


@pytest.fixture(scope="module", params=["native", "python"])
def outcomes(request):
    code = CODE
    if request.param == "python":                            # as if no call were ordinary
        code = code.replace("with FakeTensorMode():", "class Nothing:\n    def __getattr__(self, name): return lambda *a: None\nha.binding._native = lambda: Nothing()\nwith FakeTensorMode():")
        assert code != CODE
    r = subprocess.run([sys.executable, "-c", code], input="\n".join(f"{n}|{c}" for n, c in {**REFUSED, **TAKEN}.items()), cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return dict(line.split(" ", 1) for line in r.stdout.splitlines())


@pytest.mark.parametrize("name", list(REFUSED))
def test_another_layout_is_refused(outcomes, name):
    what = name.split(".")[1]
    what = what if what == "state_out" else what.split("_")[0]
    assert outcomes[name].startswith(f"ValueError {what}:"), outcomes[name]


@pytest.mark.parametrize("name", list(TAKEN))
def test_more_behind_is_taken(outcomes, name):
    assert "ValueError" not in outcomes[name], outcomes[name]
