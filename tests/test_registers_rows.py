"""What the compiler reports of the operators on the rows of many parts: which kernels spill, and how much at most.  The figures stand
in the comments of the kernels; a kernel that is not named here keeps its values in registers."""
import os
import re
import subprocess

import pytest

from paper_2305_09887_b200 import build

# bytes of spill stores a thread, by part of the mangled name
MOST = {
    "grouped_linear.cu": {"linear_kernelI6__halfLi2ELi0E": 256, "linear_kernelI13__nv_bfloat16Li2ELi0E": 256},
    "grouped_split.cu": {"split_kernelILi1E": 16},
    "group_norm.cu": {"norm_warp_rows_grad_kernelIfLb1ELb0E": 56, "norm_warp_rows_grad_kernelIfLb1ELb1E": 64, "norm_warp_rows_grad_kernelIfLb0ELb0E": 104,
                      "norm_warp_rows_grad_kernelIfLb0ELb1E": 152, "norm_unit_rows_grad_kernelIfLi1ELb0E": 32, "norm_grad_sums_kernelIfLb1E": 16,
                      "norm_grad_sums_kernelIfLb0E": 44, "norm_grad_sums_kernelI": 52, "norm_grad_apply_kernelIfLb1E": 8, "norm_grad_apply_kernelIfLb0E": 36,
                      "norm_grad_apply_kernelI": 28, "norm_apply_kernelI": 4},
    "dropout.cu": {},
}


@pytest.fixture(scope="module")
def spills(tmp_path_factory):
    where = tmp_path_factory.mktemp("registers")
    running = {s: subprocess.Popen([build._nvcc()] + build.NVCC_FLAGS + ["-Xptxas", "-v", "-c", os.path.join(build.CSRC, s), "-o", os.path.join(where, s + ".o")],
                                   stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for s in MOST}
    pattern = r"Compiling entry function '(\w+)'[^\n]*\n[^\n]*Function properties[^\n]*\n[^\n]*?(\d+) bytes spill stores"
    found = {}
    for s, p in running.items():
        out, _ = p.communicate()
        assert p.returncode == 0, out
        found[s] = {m.group(1): int(m.group(2)) for m in re.finditer(pattern, out)}
    return found


@pytest.mark.parametrize("source", MOST)
def test_kernels_spill_no_more_than_is_said_of_them(spills, source):
    got = spills[source]
    assert got
    for kernel, bytes_spilled in got.items():
        most = next((v for k, v in MOST[source].items() if k in kernel), 0)
        assert bytes_spilled <= most, (kernel, bytes_spilled, most)
