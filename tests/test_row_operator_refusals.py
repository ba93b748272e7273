"""What the operators on the rows of many parts refuse before they touch a device.

The C calls are made on a context that has no device: what passes the checks of its arguments ends in RTMA_ERR_CUDA or behind them,
without a launch.
"""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2305_09887_b200 import binding, build

INVALID_ARG = -1


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("for machines without a GPU")
    build.build_library()
    return binding.load_library()


@pytest.fixture(scope="module")
def handle(tmp_path_factory):
    """A context as rtma_create has it before it looks for its device."""
    where = tmp_path_factory.mktemp("context")
    source, shared = os.path.join(where, "context.cpp"), os.path.join(where, "context.so")
    with open(source, "w") as f:
        f.write('#include "common.cuh"\nextern "C" rtma_ctx* plain_context() { return new rtma_ctx; }\n')
    subprocess.run([build._nvcc(), "-shared", "-Xcompiler", "-fPIC", "-std=c++17", "-I", build.INCLUDE, "-I", build.CSRC, source, "-o", shared], check=True)
    make = ctypes.CDLL(shared).plain_context
    make.restype = ctypes.c_void_p
    return ctypes.c_void_p(make())


def error_of(lib, handle):
    lib.rtma_last_error.restype = ctypes.c_char_p
    return lib.rtma_last_error(handle).decode()


@pytest.mark.parametrize("scope", [0, 1])
@pytest.mark.parametrize("off", [0, 4, 8, 12])
def test_statistics_off_8_byte_boundaries(lib, handle, scope, off):
    """(mean, 1 / std) are one access of 8 bytes."""
    n, C, groups = 6, 16, 4
    rows = torch.zeros(n, C)
    stats = torch.zeros(2 * n * groups + 4)
    assert stats.data_ptr() % 16 == 0 and rows.data_ptr() % 16 == 0
    desc = binding.NormDesc(0, C, groups, scope, 0, 1e-5, 0.0, 0, 0, 0, 0)
    x, st = rows.data_ptr(), stats.data_ptr() + off
    for status in (lib.rtma_group_norm(handle, desc, n, 1, None, x, C, None, None, None, None, x, C, st, None),
                   lib.rtma_group_norm_grad(handle, desc, n, 1, None, x, C, x, C, st, None, None, None, None, x, C, None, 0, None, 0, None, 0, None)):
        assert (status == INVALID_ARG) == (off % 8 != 0)
        assert ("8-byte boundary" in error_of(lib, handle)) == (off % 8 != 0)
