"""Sizes and bounds that 32 bits do not hold, where the entry points next to the delta rule's marshal calls themselves: the C structs have 32 bits
for them, and a number cut down to its low bits would be another call.  No GPU: tensors with nothing behind them, in a process of its own."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST = 2 ** 31 - 1

# bounds on lengths: (asked, what the library gets).  No sequence is longer than 32 bits count, so a larger bound is that one.
BOUNDS = [(0, 0), (70, 70), (MOST, MOST), (2 ** 31, MOST), (2 ** 32 + 5, MOST), (2 ** 40, MOST), (-3, -3), (-2 ** 32 + 5, -2 ** 31)]
REFUSED = {
    "cols": ("layer._rows_of('x', e(2, 2 ** 32 + 8), f(2 ** 32 + 8))", "x"), "cols_one_more": ("layer._rows_of('x', e(1, 2 ** 31), f(2 ** 31))", "x"),
    "d": ("layer._gla_args('x', e(1, 1, 2 ** 32 + 64), e(1, 1, 2 ** 32 + 64), e(1, 1, 2 ** 32 + 64), f(1, 1), None, None, 0, 1.0)", "q"),
    "heads": ("layer._gla_args('x', e(1, 2 ** 32 + 2, 64), e(1, 2 ** 32 + 2, 64), e(1, 2, 64), f(1, 2), None, None, 0, 1.0)", "q"),
    "v_heads": ("layer._gla_args('x', e(1, 2, 64), e(1, 2, 64), e(1, 2 ** 32 + 2, 64), f(1, 2 ** 32 + 2), None, None, 0, 1.0)", "v"),
    "tokens": ("layer._gla_args('x', e(2 ** 32 + 2, 2, 64), e(2 ** 32 + 2, 2, 64), e(2 ** 32 + 2, 2, 64), f(2 ** 32 + 2, 2), None, None, 0, 1.0)", "q"),
    "step_sequences": ("ha.ha_la_gla_decode(e(2 ** 32 + 1, 1, 64), e(2 ** 32 + 1, 1, 64), e(2 ** 32 + 1, 1, 64), f(2 ** 32 + 1, 1), None)", "q"),
    "step_d": ("ha.ha_la_gla_decode(e(1, 1, 2 ** 32 + 64), e(1, 1, 2 ** 32 + 64), e(1, 1, 2 ** 32 + 64), f(1, 1), None)", "q"),
}
CODE = """
import sys, torch
import paper_2609_32114_b200 as ha
from paper_2609_32114_b200 import layer
from torch._subclasses.fake_tensor import FakeTensorMode
ha.binding._native()
layer._ptr = lambda t: None if t is None else 16
def e(*s): return torch.empty(*s, dtype=torch.bfloat16, device="cuda")
def f(*s): return torch.empty(*s, dtype=torch.float32, device="cuda")
def bound(n):
    return layer._gla_args("x", e(1, 70, 2, 128), e(1, 70, 2, 128), e(1, 70, 4, 128), f(1, 70, 4), None, torch.zeros(3, dtype=torch.int32, device="cuda"), n, 1.0)[0].max_seqlen
with FakeTensorMode():
    for line in sys.stdin.read().splitlines():
        name, call = line.split("|")
        try:
            print(name, "returned", eval(call))
        except Exception as x:
            print(name, type(x).__name__, str(x).splitlines()[0][:200])
"""


@pytest.fixture(scope="module")
def outcomes():
    calls = [f"bound{n}|bound({n})" for n, _ in BOUNDS] + [f"{n}|{c}" for n, (c, _) in REFUSED.items()]
    r = subprocess.run([sys.executable, "-c", CODE], input="\n".join(calls), cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return dict(line.split(" ", 1) for line in r.stdout.splitlines())


@pytest.mark.parametrize("asked,given", BOUNDS)
def test_bound_on_lengths(outcomes, asked, given):
    assert outcomes[f"bound{asked}"] == f"returned {given}"


@pytest.mark.parametrize("name", list(REFUSED))
def test_sizes_are_refused(outcomes, name):
    assert outcomes[name].startswith(f"ValueError {REFUSED[name][1]}:"), outcomes[name]
