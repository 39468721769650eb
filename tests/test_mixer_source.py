"""The mixers' kernels keep to what every kernel here owes the ones around it: nothing is read before the wait for the kernel ahead, a wait that ran out is
reported and its copies land, every wait has a limit, warps come together behind elected blocks and waits, registers that roles share out are there.  Checked on the sources, with the
checks of the older kernels, without a GPU."""
import glob
import os
import re

import pytest
from tests import test_converged_warps_cpu as warps
from tests import test_gla_source as gla
from tests import test_launch_order_cpu as order

FILES = sorted(glob.glob(os.path.join(order.CSRC, "mix", "*.cu")))
TENSOR_CORES = ["latent_prompt.cu", "latent_decode.cu"]


def _source(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


def _kernels():
    for f in FILES:
        for part in _source(f).split("__global__")[1:]:
            name = re.search(r"(\w+_kernel)\s*\(", part)
            yield os.path.basename(f), name.group(1), part[part.index("{"):part.index("\n}")]


KERNELS = list(_kernels())


def test_the_kernels_are_found():
    assert {k for _, k, _ in KERNELS} == {
        "conv_kernel", "conv_back_kernel", "conv_sum_kernel", "conv_decode_kernel", "scan_kernel", "scan_decode_kernel", "scan_back_kernel", "scan_sum_kernel", "scan_bc_kernel",
        "latent_prompt_kernel", "latent_token_kernel", "latent_prompt_tc_kernel", "latent_token_tc_kernel", "latent_join_kernel"}


# (p.x and the like are pointers: an access is one that is followed, by an index, a load or a helper that does it)
ACCESS = (order.ACCESS + r"|\b(?:seq_of|span_of|rows_of|units_of|check_\w+|find_seq|seq_of_token|cache_row|count_units|input_at|last_inputs|front_back|load_taps|load_row|load_v|stage_row|fetch\w*)"
          r"(?:<[^>]*>)?\s*\(|\bp\.(?:A|D|dt_bias|w|bias|part\w*|ckpt|seg_\w+|first|table|lengths)\s*\[|(?<![\w.])part\s*\[")


@pytest.mark.parametrize("file,kernel,body", KERNELS, ids=[k for _, k, _ in KERNELS])
def test_nothing_is_read_before_the_wait(file, kernel, body):
    assert body.count("griddepcontrol.wait;") == 1 and body.index("griddepcontrol.wait;") < body.index("griddepcontrol.launch_dependents;")
    before = body[:body.index("griddepcontrol.wait")]
    assert re.findall(order.TABLES, before) == [] and re.findall(order.INPUTS, before) == [] and re.findall(ACCESS, before) == []


@pytest.mark.parametrize("early", ["const Seq q = seq_of(p.seqs, n);", "check_spans(p);", "x = load_v<4>(x0);", "s += part[i];", "const int n = find_seq(p.seqs, t);", "a = p.A[c];", "int page = p.table[n];"])
def test_planted_access(early):
    assert re.findall(ACCESS, early)


def test_a_wait_that_ran_out_is_reported():
    copying = [(k, body) for _, k, body in KERNELS if "tma_load_4d(" in body]
    assert [k for k, _ in copying] == ["latent_token_tc_kernel", "latent_prompt_tc_kernel"]
    header = open(os.path.join(order.CSRC, "fp32_common.cuh")).read()
    assert order.unreported(copying, header) == []
    for _, body in copying:                                # ... ahead of giving tensor memory and the CTA's shared memory back
        assert body.index("report_timeout(p.status)") < body.index("tmem_dealloc(")


def test_every_wait_has_a_limit():
    for f in FILES:
        assert not re.search(r"\bmbar_wait\(|mbarrier\.(?:try|test)_wait|while \(true\)|for \(;;\)", _source(f)), f


@pytest.mark.parametrize("name", [os.path.basename(f) for f in FILES])
def test_elected_blocks(name):
    src = open(os.path.join(order.CSRC, "mix", name)).read()
    assert warps.loose_ends(src) == [] and (name not in TENSOR_CORES or "elect_one()" in src)


@pytest.mark.parametrize("name", TENSOR_CORES)
def test_warps_come_together_behind_waits(name):
    src = open(os.path.join(order.CSRC, "mix", name)).read()
    # (what an elected thread's own lambdas wait for is that thread's)
    src = re.sub(r"auto (?:keys|make_scores|add_values) = \[&\]\([^)]*\) \{(?:[^{}]|\{(?:[^{}]|\{[^{}]*\})*\})*\};", "", src)
    assert src.count("wait_for(") >= 5
    assert [x for x in gla.loose_waits(src)] == []


def test_registers_that_roles_share_out_are_asked_for():
    src = _source(os.path.join(order.CSRC, "mix", "scan.cu"))
    assert src.count("setmaxnreg.") == 2 and len(re.findall(r"allow_smem<scan_kernel<In, SP, LS, k\w+>>\(smem, kRegs\)", src)) == 3
    regs, up, down = (int(x) for x in re.search(r"kRegs = (\d+), kScanRegs = (\d+), kHelpRegs = (\d+)", src).groups())
    assert 128 * up + 256 * down <= 384 * regs and up % 8 == 0 == down % 8
    assert "has.numRegs < regs" in open(os.path.join(order.CSRC, "mix", "mix.cuh")).read()


def test_no_load_is_sent_to_several_ctas():
    for f in FILES:
        assert ".multicast" not in _source(f)
