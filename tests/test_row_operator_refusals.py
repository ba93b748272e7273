"""What the operators on the rows of many parts refuse before they touch a device.

The C calls are made on a context that has no device: what passes the checks of its arguments ends in RTMA_ERR_CUDA or behind them,
without a launch.
"""
import contextlib
import ctypes
import math
import os
import subprocess
import types

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


class Recorder:
    """Stands in for the library: takes every call, remembers its name and arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def ctx():
    """A binding context whose tensors live on the CPU and whose library does nothing."""
    c = binding.Context.__new__(binding.Context)
    c._lib, c._h = Recorder(), None
    c.device = torch.device("cpu")
    c._index = -1
    c._stream = lambda stream: 0
    return c


G, D_IN, D_OUT, N = 3, 8, 4, 10
OFF = torch.tensor([0, 2, 5, 10])


def grads(ctx, **results):
    x, dy = torch.ones(N, D_IN), torch.ones(N, D_OUT)
    return ctx.grouped_linear_dw(x, dy, OFF, **results)


def norm_grads(ctx, **results):
    x, st = torch.ones(N, D_IN), torch.ones(N, 2, 2)
    p = torch.ones(G, D_IN)
    return ctx.group_norm_grad(x, x, st, OFF, 2, p, p, act="prelu", slope=torch.ones(G), **results)


@pytest.mark.parametrize("call,name,part,distance", [(grads, "dw", (D_IN, D_OUT), 12), (grads, "db", (D_OUT,), 14), (norm_grads, "dgamma", (D_IN,), 17),
                                                     (norm_grads, "dbeta", (D_IN,), 19), (norm_grads, "dslope", (), 21)])
def test_results_that_are_expanded_views(ctx, call, name, part, distance):
    """Every part's result would go to one place (the C call sums over the parts where their distance is 0)."""
    alone = dict(bias=False) if name == "dw" else {}
    with pytest.raises(binding.RtmaError, match=f"{name} must have memory of its own"):
        call(ctx, **alone, **{name: torch.ones(part).expand(G, *part)})
    assert not ctx._lib.calls
    call(ctx, **alone, **{name: torch.ones(G, *part)})
    (_, args), = ctx._lib.calls
    assert args[distance] == math.prod(part)


def test_one_result_for_all_parts_and_of_one_part(ctx):
    """Neither is an expanded view: a result without a leading dimension is the sum, a single part's distance is not used."""
    ctx.grouped_linear_dw(torch.ones(N, D_IN), torch.ones(N, D_OUT), OFF, shared=True, dw=torch.ones(D_IN, D_OUT), db=torch.ones(D_OUT))
    ctx.grouped_linear_dw(torch.ones(N, D_IN), torch.ones(N, D_OUT), None, dw=torch.ones(D_IN, D_OUT).expand(1, D_IN, D_OUT), bias=False)
    norm_grads(ctx, dgamma=torch.ones(D_IN), dbeta=torch.ones(D_IN), dslope=torch.ones(1))
    assert len(ctx._lib.calls) == 3


def test_prelu_without_a_slope(lib, handle, ctx):
    """Forward and gradient say what is missing."""
    ctx._lib, ctx._h = lib, handle
    lib.rtma_last_error.restype = ctypes.c_char_p
    x, st = torch.ones(N, D_IN), torch.ones(N, 2, 2)
    for call in (lambda: ctx.group_norm(x, OFF, 2, act="prelu"), lambda: ctx.group_norm_grad(x, x, st, OFF, 2, act="prelu")):
        with pytest.raises(binding.RtmaError, match="PReLU without a slope"):
            call()
    ctx._h = None  # it is not this binding's to destroy


def every_call(ctx, **k):
    x, dy, W, st = torch.ones(N, D_IN), torch.ones(N, D_OUT), torch.ones(G, D_IN, D_OUT), torch.ones(N, 2, 2)
    p = torch.ones(G, D_IN)
    yield ctx.grouped_linear(x, OFF, W, **k)
    yield ctx.grouped_linear_dx(dy, OFF, W, **k)
    yield ctx.grouped_linear_dw(x, dy, OFF, **k)
    yield ctx.group_norm(x, OFF, 2, p, p, **k)
    yield ctx.group_norm_grad(x, x, st, OFF, 2, p, p, act="prelu", slope=torch.ones(G), **k)
    yield ctx.dropout(x, 0.5, 1, **k)


@pytest.mark.parametrize("stream", [None, 77, types.SimpleNamespace(cuda_stream=77)])
def test_results_are_allocated_on_the_stream_that_writes_them(ctx, monkeypatch, stream):
    """Memory of the current stream's might still be in use there, for something that has been freed."""
    on, made = [], []

    @contextlib.contextmanager
    def current(s):
        on.append(s)
        yield
        on.pop()

    real = torch.empty
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
    monkeypatch.setattr(torch.cuda, "stream", current)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (made.append(on[-1] if on else None), real(*a, **k))[1])
    monkeypatch.setattr(torch, "empty_like", lambda t, **k: torch.empty(t.shape, dtype=t.dtype))
    results = list(every_call(ctx, stream=stream))
    assert len(results) == 6 and not on
    assert made == [None if stream is None else 77] * 11  # Y; dX; dW, db; Y, stats; dX and three gradients; Y


WIDE = 2 ** 32 + 8  # 8 in 32 bits


def meta(*shape, dtype=torch.float16):
    return torch.empty(shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("call", [
    lambda c: c.dropout(meta(1, WIDE), 0.5, 1),
    lambda c: c.dropout(meta(1, 2 ** 31), 0.5, 1),
    lambda c: c.grouped_linear(meta(1, WIDE), None, meta(WIDE, 4)),
    lambda c: c.grouped_linear(meta(1, 4), None, meta(4, WIDE), out=meta(1, WIDE)),
    lambda c: c.grouped_linear_dx(meta(1, WIDE), None, meta(4, WIDE)),
    lambda c: c.grouped_linear_dx(meta(1, 4), None, meta(WIDE, 4), out=meta(1, WIDE)),
    lambda c: c.grouped_linear_dw(meta(1, WIDE), meta(1, 4), None, dw=meta(1, WIDE, 4, dtype=torch.float32)),
    lambda c: c.grouped_linear_dw(meta(1, 4), meta(1, WIDE), None, dw=meta(1, 4, WIDE, dtype=torch.float32)),
    lambda c: c.group_norm(meta(1, WIDE), None, 8, out=meta(1, WIDE), stats=meta(1, 8, 2, dtype=torch.float32)),
    lambda c: c.group_norm(meta(1, 8), None, 2 ** 32 + 8, stats=meta(1, 2 ** 32 + 8, 2, dtype=torch.float32)),
    lambda c: c.group_norm(meta(1, 8), meta(2 ** 32 + 2, dtype=torch.int64), 8),
])
def test_sizes_of_more_than_31_bits(ctx, call):
    """The C calls take them as int32; ctypes would cut them down without a word."""
    with pytest.raises((ValueError, binding.RtmaError)):
        call(ctx)
    assert not ctx._lib.calls
