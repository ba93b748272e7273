"""What whole layers and the clipping of gradients refuse before they touch a device (see test_row_operator_refusals for the way)."""
import contextlib
import ctypes
import math
import os
import struct
import subprocess

import pytest
import torch

from paper_2305_09887_b200 import binding, build



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


BASE = dict(dtype=1, d_in=8, d_out=16, act=3, gated=0, grad_dtype=1, n=6, G=1, ldx=8, ldy=16, ldr=16, ldz=16, lddx=8)


def calls(lib, handle, **more):
    """The statuses and messages of the forward call and of the gradient with these arguments."""
    a = {**BASE, **more}
    memory = torch.zeros(4096)
    x, w, y, z = (memory.data_ptr() + 2048 * i for i in range(4))
    desc = binding.LayerDesc(a["dtype"], a["d_in"], a["d_out"], a["act"], a["gated"], a["grad_dtype"], 0, 0, 0)
    got = []
    for call in (lambda: lib.rtma_grouped_layer(handle, desc, a["n"], a["G"], None, a.get("x", x), a["ldx"], a.get("w", w), None, a.get("slope"), a.get("r"), a["ldr"],
                                                a.get("y", y), a["ldy"], None),
                 lambda: lib.rtma_grouped_layer_grad(handle, desc, a["n"], a["G"], None, a.get("x", x), a["ldx"], a.get("w", w), None, a.get("slope"), a.get("dy", y),
                                                     a["ldy"], a.get("z", z), a["ldz"], a.get("dx"), a["lddx"], a.get("dw"), 0, a.get("db"), 0, a.get("dslope"), 0, None)):
        status = call()
        got.append((status, error_of(lib, handle)))
    return got


@pytest.mark.parametrize("change,words,which", [
    (dict(dtype=3), "dtype=3", 3), (dict(act=4), "act=4", 3), (dict(act=-1), "act=-1", 3), (dict(act=2), "PReLU without a slope", 3),
    (dict(d_in=0), "outside", 3), (dict(d_out=16385, ldy=20000, ldz=20000), "outside", 3), (dict(gated=1, d_out=8193, ldy=9000, ldz=20000), "outside", 3),
    (dict(n=-1), "outside", 3), (dict(n=2**31), "outside", 3), (dict(G=0), "outside", 3), (dict(G=513), "outside", 3), (dict(G=2), "without offsets", 3),
    (dict(ldx=7), "closer", 3), (dict(ldy=15), "closer", 3), (dict(r=64, ldr=15), "closer", 1), (dict(ldz=15), "closer", 2), (dict(ldz=20), "16-byte", 2), (dict(z=66), "16-byte", 2), (dict(d_out=15, dy=64, z=64, ldy=16, ldz=16), "overlap", 2), (dict(gated=1, ldz=31), "closer", 2),
    (dict(dx=64, lddx=7), "closer", 2), (dict(x=None), "null", 3), (dict(w=None), "null", 3), (dict(z=None), "null", 2), (dict(dslope=64), "without PReLU", 2),
    (dict(db=64), "comes with", 2), (dict(grad_dtype=2), "type 2", 2), (dict(x=64, y=64), "overlap", 1), (dict(x=64, z=64), "overlap", 2), (dict(x=64, dx=64), "overlap", 2),
    (dict(gated=1, ldz=32, dy=64, z=64), "overlap", 2), (dict(dy=64, z=64, ldz=17), "overlap", 2), (dict(z=64, dx=64), "overlap", 2), (dict(act=0, dy=64, dx=64), "overlap", 2),
])
def test_layers(lib, handle, change, words, which):
    for k, (status, message) in enumerate(calls(lib, handle, **change)):
        if which >> k & 1:
            assert status < 0 and words in message, (k, status, message)


def test_a_call_that_is_right_reaches_the_device(lib, handle):
    for status, message in calls(lib, handle, dx=64, dw=128):
        assert status != 0 and "cuda" in message.lower(), (status, message)


@pytest.mark.parametrize("change,words", [
    (dict(count=-1), "-1 gradients"), (dict(G=0), "G=0"), (dict(G=513), "G=513"), (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=math.nan), "max_norm"),
    (dict(dtype=3), "type 3"), (dict(out=64, out_dtype=2), "its result 2"), (dict(size=-1), "-1 values"), (dict(grad=0), "of 10 values"),
    (dict(G=2, out=4096, out_stride=9), "overlap"), (dict(out=1024, out_dtype=0), "another form"), (dict(G=2, out=1024, grad_stride=12, out_stride=10), "another form"),
])
def test_clipping(lib, handle, change, words):
    a = {**dict(count=1, G=1, max_norm=1.0, dtype=1, out_dtype=1, size=10, grad=1024, out=0, grad_stride=10, out_stride=10), **change}
    table = struct.pack("<QQqqqii", a["grad"], a["out"], a["size"], a["grad_stride"], a["out_stride"], a["dtype"], a["out_dtype"])
    assert lib.rtma_clip_gradients(handle, a["count"], table, a["G"], 0, a["max_norm"], 0, None, None) < 0
    assert words in error_of(lib, handle)


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
    c.device, c._index = torch.device("cpu"), -1
    c._stream = lambda stream: 0
    c.close = lambda: None
    return c


def test_layer_sizes_go_through(ctx):
    X, W, b, dY = torch.zeros(5, 6), torch.zeros(2, 6, 8), torch.zeros(2, 8), torch.zeros(5, 4)
    o = torch.tensor([0, 2, 5])
    assert ctx.grouped_linear_act(X, o, W, b).shape == (5, 8)
    assert ctx.grouped_gated_linear(X, o, W, b).shape == (5, 4)
    dx, dw, db, ds = ctx.grouped_gated_linear_grad(X, dY, o, W, b, act="prelu", slope=torch.zeros(2))
    assert dx.shape == X.shape and dw.shape == W.shape and db.shape == b.shape and ds.shape == (2,)
    half = X.bfloat16(), dY.bfloat16(), W.bfloat16()
    assert ctx.grouped_gated_linear_grad(half[0], half[1], o, half[2])[1].dtype == torch.bfloat16
    assert ctx.grouped_gated_linear_grad(half[0], half[1], o, half[2], grad_dtype=torch.float32)[1].dtype == torch.float32


@pytest.mark.parametrize("change,error", [
    (dict(W=torch.zeros(2, 6, 7)), ValueError), (dict(W=torch.zeros(2, 5, 8)), ValueError), (dict(W=torch.zeros(2, 6, 8).half()), TypeError),
    (dict(bias=torch.zeros(3, 8)), ValueError), (dict(act="gelu"), ValueError), (dict(X=torch.zeros(5, 6).double()), TypeError),
    (dict(X=torch.zeros(5, 12)[:, ::2]), ValueError), (dict(slope=torch.zeros(3), act="prelu"), ValueError), (dict(W=torch.zeros(2, 8, 6).transpose(1, 2)), ValueError),
])
def test_layer_tensors(ctx, change, error):
    a = {**dict(X=torch.zeros(5, 6), offsets=torch.tensor([0, 2, 5]), W=torch.zeros(2, 6, 8), bias=None, act="silu", slope=None), **change}
    with pytest.raises(error):
        ctx.grouped_gated_linear(**a)
    assert not ctx._lib.calls


@pytest.mark.parametrize("change,error", [
    (dict(dH=torch.zeros(5, 8)), ValueError), (dict(dH=torch.zeros(4, 4)), ValueError), (dict(dH=torch.zeros(5, 4).half()), TypeError), (dict(dz=torch.zeros(5, 4)), ValueError),
    (dict(out=torch.zeros(5, 5)), ValueError), (dict(dw=torch.zeros(6, 8)), ValueError), (dict(dw=torch.zeros(2, 6, 8).half()), TypeError),
    (dict(dw=torch.zeros(1, 6, 8).expand(2, 6, 8)), binding.RtmaError), (dict(grad_dtype=torch.float16), TypeError), (dict(db=torch.zeros(8)), ValueError),
])
def test_gradient_tensors(ctx, change, error):
    a = {**dict(X=torch.zeros(5, 6), dH=torch.zeros(5, 4), offsets=torch.tensor([0, 2, 5]), W=torch.zeros(2, 6, 8), bias=torch.zeros(2, 8)), **change}
    with pytest.raises(error):
        ctx.grouped_gated_linear_grad(**a)
    assert not ctx._lib.calls


@pytest.mark.parametrize("grads,more,error", [
    ([torch.zeros(3)], dict(parts=0), ValueError), ([torch.zeros(3)], dict(parts=2), ValueError), ([torch.zeros(2, 3).double()], {}, TypeError),
    ([torch.zeros(4, 4).t()[1:]], dict(parts=3), ValueError), ([torch.zeros(6)[::2]], {}, None), ([torch.zeros(600, 2)[:, :1], torch.zeros(3)], {}, ValueError),
    ([torch.zeros(3)], dict(out=[]), ValueError), ([torch.zeros(3)], dict(out=[torch.zeros(4)]), ValueError), ([torch.zeros(3)], dict(out=[torch.zeros(3).half()]), ValueError),
    ([torch.zeros(2, 3)], dict(parts=2, out=[torch.zeros(1, 3).expand(2, 3)]), binding.RtmaError),
])
def test_clipped_tensors(ctx, grads, more, error):
    with pytest.raises(error) if error else contextlib.nullcontext():
        ctx.clip_gradients(grads, 1.0, **more)
    assert bool(ctx._lib.calls) == (error is None)


def test_the_table_of_gradients(ctx):
    flat = torch.zeros(2, 50)
    grads = [torch.zeros(2, 3, 4).bfloat16(), flat[:, 30:37]]
    out = [flat[:, 3:15].unflatten(1, (3, 4)), None]
    ctx.clip_gradients(grads, 2.5, parts=2, out=out, zero_nonfinite=True)
    (name, args), = ctx._lib.calls
    assert name == "rtma_clip_gradients" and args[1] == 2 and args[3:7] == (2, 0, 2.5, 1)
    first, second = (binding.GRADIENT.unpack_from(args[2], binding.GRADIENT.size * i) for i in range(2))
    assert first == (grads[0].data_ptr(), flat.data_ptr() + 12, 12, 12, 50, 1, 0)
    assert second == (grads[1].data_ptr(), 0, 7, 50, 0, 0, 0)
    assert binding.GRADIENT.size == 48


@pytest.mark.parametrize("count", [2, 30])
@pytest.mark.parametrize("grads,outs", [((1024, 1024), (1024, 1024)), ((1024, 2048), (4096, 4096)), ((1024, 2048), (2048, 4096)), ((1024, 2048), (4096, 1024))])
def test_a_tensor_listed_twice(lib, handle, grads, outs, count):
    """Two results at one place, or one where another's gradient still has to be read."""
    rows = [(1 << 20, 0, 10)] * (count - 2) + [(g, o, 10) for g, o in zip(grads, outs)]
    table = b"".join(struct.pack("<QQqqqii", g, o, size, 10, 10, 1, 1) for g, o, size in rows)
    assert lib.rtma_clip_gradients(handle, count, table, 1, 0, 1.0, 0, None, None) == -1
    assert f"the result of gradient {count - 1}" in error_of(lib, handle) or f"the result of gradient {count - 2}" in error_of(lib, handle)


def test_a_gradient_twice_where_nothing_is_written_to_it(lib, handle):
    """One gradient with two results, or one that is only part of the norm besides, passes the checks (and then finds no device)."""
    for rows in ([(1024, 2048), (1024, 4096)], [(1024, 1024), (1024, 0)]):
        table = b"".join(struct.pack("<QQqqqii", g, o, 10, 10, 10, 1, 1) for g, o in rows)
        assert lib.rtma_clip_gradients(handle, 2, table, 1, 0, 1.0, 0, None, None) < 0
        assert "result" not in error_of(lib, handle)
