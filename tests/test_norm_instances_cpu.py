"""Every instance of the norms' kernels that is built is one that some row length takes.  The rule (shape_of and by_length in csrc/norm.cu) is stated
once more here; the instances are the names in the library.  No GPU."""
import re
import shutil
import subprocess

import pytest

from paper_2609_32114_b200 import build


def taken(vec, cols, back):
    """(vectors of 16 bytes or elements, of a thread, threads a kernel is built for, whole vectors?) of rows of `cols` values."""
    full = cols % vec == 0
    vectors = cols // vec if full else -(-cols // vec) + 1
    if vectors <= 32:
        return vec, 1, 256, full
    nv = 1
    while nv * (256 if back and nv == 1 else 1024) < vectors:
        nv *= 2
    threads = -(-(-(-vectors // nv)) // 32) * 32
    if threads <= 256 and (nv == 1 or (back and nv == 2)):
        return vec, nv, 257, full                          # (257: up to 256 threads to a row, told apart from several rows to 256 threads)
    return vec, nv, 512 if threads <= 512 and (nv == 1 or (back and nv == 2)) else 1024, full


@pytest.mark.parametrize("kernel,back,flags", [("gated_norm_kernel", False, [()]), ("gated_norm_back_kernel", True, [()]),
                                               ("add_norm_kernel", False, [(False,), (True,)]), ("add_norm_back_kernel", True, [(False,), (True,)])])
def test_instances(kernel, back, flags):
    if shutil.which("nm") is None:
        pytest.skip("needs nm")
    names = subprocess.run(["nm", "-C", build.build()], capture_output=True, text=True, check=True).stdout
    built = set(re.findall(r"::%s<(\w+), (\d+), (\d+), (\d+), (\w+)(?:, (\w+))?>\(" % kernel, names))
    want = {(t, *(str(x).lower() for x in (*taken(vec, cols, back), *(f or ("",)))))
            for t, vecs in (("__nv_bfloat16", (8, 1)), ("float", (4, 1))) for vec in vecs for cols in range(1, 16385) for f in flags}
    assert built == want
