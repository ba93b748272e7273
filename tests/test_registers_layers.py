"""What the compiler reports of the layers' kernels and of clipping: which spill, and how much at most.  The figures stand in the comments
of the kernels; a kernel that is not named here keeps its values in registers."""
import os
import re
import subprocess

import pytest

from paper_2305_09887_b200 import build

# bytes of spill stores a thread, by part of the mangled name
MOST = {
    "layer.cu": {},
    "layer_bf16.cu": {},
    "layer_f16.cu": {},
    "layer_f32.cu": {"layer_f32_kernelILb0ELb0E": 224, "layer_f32_kernelILb0ELb1E": 120, "layer_f32_kernelILb1ELb0E": 132, "layer_f32_kernelILb1ELb1E": 304},
    "layer_wgrad.cu": {"layer_wgrad_f32_kernel": 40},
    "clip.cu": {},
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
    for kernel, spilled in got.items():
        most = max([m for part, m in MOST[source].items() if part in kernel], default=0)
        assert spilled <= most, (kernel, spilled, most)
