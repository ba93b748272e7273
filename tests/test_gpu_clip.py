"""Norms of gradients over many tensors, and clipping, against their definition in 64 bits.  A norm is a sum in 64 bits of squares, eight
of them at a time in fp32 (8 roundings, half of which pass to the root), rounded once: 8 2^-24.  A clipped value has two roundings
in fp32 (the factor's and its own) and one of its type."""
import math

import pytest
import torch

from layer_reference import F64, rounding
from paper_2305_09887_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
NORM = 8 * 2.0**-24


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def tensors(shapes, dtypes, parts, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    lead = (parts,) if parts > 1 else ()
    sizes = 0.2 + 2 * torch.rand(parts, generator=g)
    out = []
    for i, s in enumerate(shapes):
        t = torch.randn(*lead, *s, generator=g) * scale
        if parts > 1:
            t = t * sizes.view(parts, *[1] * len(s))
        out.append(t.to(dtypes[i % len(dtypes)]).cuda())
    return out


def norms_of(grads, parts):
    if parts == 1:
        return torch.stack([t.to(F64).pow(2).sum() for t in grads]).sum().sqrt().view(1)
    return torch.stack([t.to(F64).reshape(parts, -1).pow(2).sum(1) for t in grads]).sum(0).sqrt()


def check(ctx, grads, parts, max_norm, out=None, **more):
    before = [t.clone() for t in grads]
    norms = ctx.clip_gradients(grads, max_norm, parts=parts, out=out, **more)
    want = norms_of(before, parts)
    assert norms.shape == (parts,) and norms.dtype == torch.float32
    assert ((norms.to(F64) - want).abs() <= NORM * want).all(), (norms, want)
    scale = torch.where(want > max_norm, max_norm / want, torch.ones_like(want))
    for i, (t, b) in enumerate(zip(grads if out is None else out, before)):
        if t is None:
            continue
        y = b.to(F64) * scale.view(parts, *[1] * (b.dim() - 1)) if parts > 1 else b.to(F64) * scale
        off = (t.to(F64) - y).abs()
        tol = (NORM + 3 * 2.0**-24) * y.abs() + rounding(y, t.dtype)
        # a scale within the norm's error of one may be one
        assert (off <= tol).all(), (i, (off / tol).max())
    if out is not None:
        for t, b in zip(grads, before):
            assert torch.equal(t, b)


SHAPES = [(1,), (7,), (64, 128), (128,), (33, 47), (0,), (3, 5, 7), (2047,), (2048,), (2049,), (100, 266)]


@pytest.mark.parametrize("parts", [1, 2, 5])
@pytest.mark.parametrize("dtypes", [[t] for t in TYPES] + [TYPES])
@pytest.mark.parametrize("max_norm", [1e-3, 150.0, 1e9, math.inf, 0.0])
def test_in_place(ctx, dtypes, parts, max_norm):
    check(ctx, tensors(SHAPES, dtypes, parts, 3), parts, max_norm)


@pytest.mark.parametrize("parts", [1, 3])
@pytest.mark.parametrize("dtype", TYPES)
def test_into_other_tensors(ctx, dtype, parts):
    grads = tensors(SHAPES, [dtype], parts, 5)
    check(ctx, grads, parts, 100.0, out=[torch.empty_like(t) for t in grads])
    check(ctx, grads, parts, 100.0, out=[torch.empty_like(t, dtype=torch.float32) if i % 2 else None for i, t in enumerate(grads)])


@pytest.mark.parametrize("parts", [1, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_into_the_rows_of_replicas(ctx, dtype, parts):
    """Results (and gradients) that are contiguous within a part only, at odd places; one norm over them, too."""
    M = 4
    shapes = [(30, 42), (42,), (21, 30), (5,)]
    grads = tensors(shapes, [dtype], M, 7)
    flat = torch.full((M, 3001), 9.0, device="cuda")
    ends = [3]
    for t in grads:
        ends.append(ends[-1] + t[0].numel())
    out = [flat[:, a:b].unflatten(1, s) for a, b, s in zip(ends, ends[1:], shapes)]
    check(ctx, grads, parts, 20.0, out=out)
    assert (flat[:, :3] == 9).all() and (flat[:, ends[-1]:] == 9).all()
    check(ctx, out, parts, 5.0)
    assert (flat[:, :3] == 9).all() and (flat[:, ends[-1]:] == 9).all()


@pytest.mark.parametrize("count", [23, 24, 25, 159, 161, 400])
def test_many_tensors(ctx, count):
    grads = tensors([(1 + i % 5, 3 + i % 11) for i in range(count)], TYPES, 2, 11)
    check(ctx, grads, 2, 3.0)


def test_large_tensors_and_the_norm_alone(ctx):
    grads = tensors([(3000, 1001), (5_000_000,), (17,)], [torch.bfloat16, torch.float32], 1, 13)
    want = norms_of(grads, 1)
    assert abs(ctx.gradient_norms(grads).item() - want.item()) <= NORM * want.item()
    check(ctx, grads, 1, 10.0)


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e25, 1e36])
def test_squares_beyond_fp32(ctx, scale):
    for dtype in (torch.float32, torch.bfloat16):
        grads = tensors([(50, 40), (7,)], [dtype], 1, 17, scale)
        check(ctx, grads, 1, 0.5 * scale, out=[torch.empty_like(t, dtype=torch.float32) for t in grads])
        check(ctx, grads, 1, 1e-3 * scale)


def test_a_scale_below_fp32(ctx):
    """Values of 1e30 down to a norm of 1e-10: the factor has no bits left in fp32."""
    grads = tensors([(50, 40)], [torch.float32], 1, 19, 1e30)
    check(ctx, grads, 1, 1e-10)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("zero", [False, True])
def test_what_is_not_finite(ctx, bad, zero):
    grads = tensors([(40, 30), (9,)], TYPES, 3, 23)
    grads[0][1, 5, 6] = bad
    before = [t.clone() for t in grads]
    norms = ctx.clip_gradients(grads, 1.0, parts=3, zero_nonfinite=zero)
    assert math.isfinite(norms[0]) and math.isfinite(norms[2]) and not math.isfinite(norms[1])
    for t, b in zip(grads, before):
        assert (not t[1].any()) if zero else torch.equal(t[1].nan_to_num(77), b[1].nan_to_num(77))
        assert not torch.equal(t[0], b[0]) and t[0].isfinite().all()


def test_nothing_and_zeros(ctx):
    assert ctx.clip_gradients([], 1.0).tolist() == [0.0]
    assert ctx.clip_gradients([torch.empty(3, 0, device="cuda")], 1.0, parts=3).tolist() == [0.0] * 3
    z = torch.zeros(2, 300, device="cuda")
    assert ctx.clip_gradients([z], 0.0, parts=2).tolist() == [0.0, 0.0] and not z.any()
    assert ctx.clip_gradients([torch.tensor(-3.0, device="cuda")], 1.0).tolist() == [3.0]


def test_a_captured_clip_follows_its_gradients():
    ctx = binding.Context(0)
    grads = tensors([(300, 20), (300,)], [torch.bfloat16, torch.float32], 1, 29)
    out = [torch.empty_like(t, dtype=torch.float32) for t in grads]
    with pytest.raises(binding.RtmaError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            ctx.clip_gradients(grads, 2.0, out=out)
    ctx.clip_gradients(grads, 2.0, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norms = ctx.clip_gradients(grads, 2.0, out=out)
    for t in grads:
        t.mul_(3)
    graph.replay()
    want = [torch.empty_like(t) for t in out]
    assert torch.equal(norms, ctx.clip_gradients(grads, 2.0, out=want))
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_same_bits_every_time_on_any_stream(ctx):
    grads = tensors([(700, 900), (33,), (9, 1001)], TYPES, 2, 31)
    out = [torch.empty_like(t) for t in grads]
    norms = ctx.clip_gradients(grads, 2.0, parts=2, out=out)
    first = [t.clone() for t in out]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    again = ctx.clip_gradients(grads, 2.0, parts=2, out=out, stream=stream)
    stream.synchronize()
    assert torch.equal(norms, again) and all(torch.equal(a, b) for a, b in zip(first, out))
