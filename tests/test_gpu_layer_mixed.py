"""Gradients of layers of which either the matrix or the bias alone is one for all parts, against the definition in 64 bits (tolerances: layer_reference)."""
import pytest
import torch

from layer_reference import Layer, rounding
from paper_2305_09887_b200 import binding
from test_gpu_layers import TYPES, Case, assert_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def check(ctx, case, one, kind):
    """one: "W" or "bias", the one that the parts share."""
    G = len(case.sizes)
    W, b = (case.W[1], case.b) if one == "W" else (case.W, case.b[1])
    case.W, case.b = W, b
    dx, dw, db, dslope = case.gradient(ctx, grad_dtype=kind)
    ctx.check()
    assert dw.shape == W.shape and db.shape == b.shape and dw.dtype == db.dtype == kind
    parts = [Layer(case.X[p:q], W if one == "W" else W[g], b[g] if one == "W" else b, case.act, 0.0 if case.slope is None else case.slope[g].item(), case.gated, case.dtype,
                   None, case.dY[p:q]) for g, (p, q) in enumerate(zip(case.o, case.o[1:]))]
    for g, (p, q) in enumerate(zip(case.o, case.o[1:])):
        assert_close(dx[p:q], parts[g].dx, parts[g].dx_off, f"dX of part {g}")
        if dslope is not None:
            assert_close(dslope[g], parts[g].dslope, parts[g].dslope_off + rounding(parts[g].dslope, torch.float32), f"dslope of part {g}")
    for name, got, per_part in (("dw", dw, one == "bias"), ("db", db, one == "W")):
        want, off = [getattr(p, name) for p in parts], [getattr(p, name + "_off") for p in parts]
        if not per_part:
            got, want, off = [got], [sum(want)], [sum(off)]
        for g in range(G if per_part else 1):
            assert_close(got[g], want[g], off[g] + rounding(want[g].abs() + off[g], kind), f"{name} {g}")


@pytest.mark.parametrize("one", ["W", "bias"])
@pytest.mark.parametrize("act", ["none", "prelu", "silu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_of_the_two(ctx, dtype, gated, act, one):
    for kind in {dtype, torch.float32}:
        check(ctx, Case(dtype, [70, 0, 200, 1], 40, 56, act, gated, seed=103), one, kind)


@pytest.mark.parametrize("one", ["W", "bias"])
@pytest.mark.parametrize("sizes,d_in,d_out", [([3000, 0, 1700], 100, 47), ([400] * 12, 13, 7), ([1, 5000], 47, 130), ([900, 900], 256, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_odd_widths_and_many_chunks(ctx, dtype, sizes, d_in, d_out, one):
    for act, gated in (("none", False), ("silu", True)):
        check(ctx, Case(dtype, sizes, d_in, d_out, act, gated, seed=107), one, torch.float32)


@pytest.mark.parametrize("one", ["W", "bias"])
@pytest.mark.parametrize("dtype", TYPES)
def test_most_parts(ctx, dtype, one):
    sizes = [(7 * g) % 11 for g in range(binding.MAX_GROUPS)]
    sizes[3], sizes[-1] = 700, 0
    check(ctx, Case(dtype, sizes, 24, 10, "none", False, seed=109), one, torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(ctx, dtype):
    X, W, dY = torch.empty(0, 12, dtype=dtype, device="cuda"), torch.ones(12, 16, dtype=dtype, device="cuda"), torch.empty(0, 16, dtype=dtype, device="cuda")
    _, dw, db, _ = ctx.grouped_linear_act_grad(X, dY, torch.zeros(3, dtype=torch.int64, device="cuda"), W, torch.ones(2, 16, dtype=dtype, device="cuda"), act="none")
    assert dw.shape == (12, 16) and db.shape == (2, 16) and not dw.any() and not db.any()
