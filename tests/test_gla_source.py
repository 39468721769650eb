"""The kernels of gated linear attention and of the norms keep to what every kernel here owes the ones around it: nothing is read before
the wait for the kernel ahead, a wait that ran out is reported and its copies land, warps come together behind elected blocks.  Checked on
the sources, with the checks of the older kernels, without a GPU."""
import glob
import os
import re

import pytest
from tests import test_converged_warps_cpu as warps
from tests import test_launch_order_cpu as order

CSRC = order.CSRC
FILES = sorted(glob.glob(os.path.join(CSRC, "gla", "*.cu"))) + [os.path.join(CSRC, "norm.cu")]
TENSOR_CORES = ["tc_back.cu", "tc_walk.cu", "tc_state.cu"]


def _source(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


def _kernels():
    for f in FILES:
        for part in _source(f).split("__global__")[1:]:
            name = re.search(r"(\w+_kernel)\s*\(", part)
            body = part[part.index("{"):part.index("\n}")]
            yield os.path.basename(f), name.group(1), body


KERNELS = list(_kernels())


def test_the_kernels_are_found():
    assert {k for _, k, _ in KERNELS} == {
        "gla_decode_kernel", "gla_state_kernel", "gla_combine_kernel", "gla_out_kernel", "gla_back_kernel", "gla_sum_kernel", "gla_tc_state_kernel", "gla_tc_walk_kernel",
        "gla_tc_back_kernel", "gated_norm_kernel", "gated_norm_back_kernel", "add_norm_kernel", "add_norm_back_kernel", "norm_reduce_kernel"}


ACCESS = order.ACCESS + r"|\b(?:fetch_gates|tma_load|cp_async\w*)\s*\(|p\.(?:g|part|chunks|seqs)\b[^;]*\["


@pytest.mark.parametrize("file,kernel,body", KERNELS, ids=[k for _, k, _ in KERNELS])
def test_nothing_is_read_before_the_wait(file, kernel, body):
    assert body.count("griddepcontrol.wait;") == 1 and body.index("griddepcontrol.wait;") < body.index("griddepcontrol.launch_dependents;")
    before = body[:body.index("griddepcontrol.wait")]
    before = re.sub(r"auto \w+ = \[&\]\([^)]*\) \{(?:[^{}]|\{[^{}]*\})*\};", "", before)
    assert re.findall(order.TABLES, before) == [] and re.findall(order.INPUTS, before) == [] and re.findall(ACCESS, before) == []


@pytest.mark.parametrize("early", ["tma_load_4d(sm, &map_k, &full[0], 0, jq, t0, 0);", "float4 raw = fetch_gates(p.g, p.HV, j, geom(0), lane);", "tok0 = p.seqs.tok0[n];",
                                   "const float x = p.part[rev][part];", "const int n = p.chunks.seq[0];"])
def test_planted_access(early):
    assert re.findall(ACCESS + "|" + order.TABLES, early)


def test_a_wait_that_ran_out_is_reported():
    header = open(os.path.join(CSRC, "fp32_common.cuh")).read()
    copying = [(k, body) for _, k, body in KERNELS if re.search(r"\b(?:bulk_load|tma_load_4d)\(", body)]
    assert [k for k, _ in copying] == ["gla_tc_back_kernel", "gla_tc_state_kernel", "gla_tc_walk_kernel"]
    assert order.unreported(copying, header) == []
    for k, body in copying:                                # ... ahead of giving tensor memory and the CTA's shared memory back
        assert body.index("report_timeout(p.status)") < body.index("tmem_dealloc(")


def test_every_wait_has_a_limit():
    """wait_for gives up after a limit of its own, and at once when another wait of the CTA has; no kernel polls in another way."""
    header = _source(os.path.join(CSRC, "gla", "tc.cuh"))
    body = header[header.index("wait_for("):].split("\n}")[0]
    assert "abort_flag" in body and re.search(r"for \([^;]*;[^;]*<[^;]*;", body)
    for f in FILES:
        src = _source(f)
        assert not re.search(r"\bmbar_wait\(|mbarrier\.(?:try|test)_wait|while \(true\)|for \(;;\)", src), f


@pytest.mark.parametrize("name", [os.path.basename(f) for f in FILES])
def test_elected_blocks(name):
    path = next(f for f in FILES if os.path.basename(f) == name)
    assert warps.loose_ends(open(path).read()) == []
    if name in TENSOR_CORES:
        assert "elect_one()" in open(path).read()


# Warps' threads may also part at a polling wait; the next aligned instruction has to come behind a __syncwarp or a barrier of the CTA.
ALIGNED = re.compile(r"__syncwarp|__syncthreads|\"bar\.|\b(?:ldsm4t?|tmem_(?:ld|st)\w*|\w*shfl\w*|exchange\d)\(|elect_one\(\)|named_sync|(?<![\w=] )\b(?:arrive|wait|seen)\(")
TOGETHER = ("__syncwarp", "__syncthreads", "arrive(", "wait(", "seen(")   # (the last three: the gradient kernel's lambdas, which hold one)


def loose_waits(src):
    src = re.sub(r"//[^\n]*", "", src)
    bad = []
    for m in re.finditer(r"\bwait_for\(", src):
        block = src.rfind("elect_one()", 0, m.start())
        if block >= 0 and warps._statement_end(src, block + len("elect_one())")) > m.start():
            continue                                       # one thread's own
        nxt = ALIGNED.search(src, src.index(";", m.end()) + 1)
        if nxt and nxt.group() not in TOGETHER:
            bad.append((src.count("\n", 0, m.start()) + 1, nxt.group()))
    return bad


@pytest.mark.parametrize("name", TENSOR_CORES)
def test_warps_come_together_behind_waits(name):
    src = open(os.path.join(CSRC, "gla", name)).read()
    assert src.count("wait_for(") >= 5 and loose_waits(src) == []


def test_the_lambdas_bring_warps_together():
    src = _source(os.path.join(CSRC, "gla", "tc_back.cu"))
    src = src[src.index("} else {", src.index("p.dg[")):]
    for name in ("arrive", "wait", "seen"):
        assert "__syncwarp();" in re.search(r"auto %s = \[&\]\([^)]*\) \{([^}]*)\};" % name, src).group(1), name


def test_planted_wait():
    src = _source(os.path.join(CSRC, "gla", "tc_state.cu"))
    at = src.index("wait_for(&product[b]")
    assert len(loose_waits(src[:at] + src[at:].replace("__syncwarp();", "", 1))) == 1
