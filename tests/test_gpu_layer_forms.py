"""Forms of whole layers that the other tests' shapes do not meet: gradients without an activation (dZ is dY) and SiLU in every shape, on any boundary, of shared
matrices and at the largest widths; odd widths whose rows lie on 16-byte boundaries with something else behind them."""
import pytest
import torch

from paper_2305_09887_b200 import binding
from test_gpu_layers import SHAPES, TYPES, Case, normal, rows_of

pytestmark = pytest.mark.gpu
WIDEST = 16384


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


class Apart(Case):
    """Rows at the next multiple of 16 bytes, `more` of them further; NaN between them."""

    def __init__(self, *args, more=0, **how):
        super().__init__(*args, **how)
        lift = lambda t: rows_of(t[:-2].float(), self.dtype, -t.shape[1] % 8 + 8 * more)  # noqa: E731
        self.X, self.dY = lift(self.X), lift(self.dY)
        self.residual = None if self.residual is None else lift(self.residual)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_gradient_without_activation(ctx, dtype, sizes, d_in, d_out, bias, wide):
    Case(dtype, sizes, d_in, d_out, "none", False, bias=bias, seed=131).check_gradient(ctx, torch.float32 if wide else None)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_silu(ctx, dtype, sizes, d_in, d_out, gated):
    case = Case(dtype, sizes, d_in, d_out, "silu", gated, residual=d_out % 2 == 1, seed=137)
    case.check_forward(ctx)
    case.check_gradient(ctx)


@pytest.mark.parametrize("gated,act", [(True, "none"), (True, "relu"), (False, "relu")])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_other_activations(ctx, dtype, sizes, d_in, d_out, gated, act):
    case = Case(dtype, sizes, d_in, d_out, act, gated, residual=True, seed=139)
    case.check_forward(ctx)
    case.check_gradient(ctx)


@pytest.mark.parametrize("act,gated", [("none", False), ("none", True), ("relu", False), ("prelu", False), ("silu", True)])
@pytest.mark.parametrize("more", [0, 1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_something_else_behind_the_rows(ctx, dtype, sizes, d_in, d_out, more, act, gated):
    case = Apart(dtype, sizes, d_in, d_out, act, gated, residual=True, seed=149, more=more)
    case.check_forward(ctx)
    case.check_gradient(ctx)


@pytest.mark.parametrize("d_in,d_out", [(64, 96), (47, 13), (33, 130), (100, 47)])
@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (4, 4), (8, 0), (3, 2)])
@pytest.mark.parametrize("dtype", TYPES)
def test_without_activation_on_any_boundary(ctx, dtype, pad, shift, d_in, d_out):
    case = Case(dtype, [150, 61], d_in, d_out, "none", False, residual=True, pad=pad, shift=shift, seed=151)
    case.check_forward(ctx)
    case.check_gradient(ctx)


@pytest.mark.parametrize("d_in,d_out", [(40, 56), (47, 13), (256, 47), (13, 300)])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_matrix_without_activation(ctx, dtype, d_in, d_out):
    Case(dtype, [70, 0, 2000, 33], d_in, d_out, "none", False, seed=157, shared=True).check_gradient(ctx, torch.float32)


@pytest.mark.parametrize("d_in,d_out", [(WIDEST, 40), (40, WIDEST), (WIDEST - 1, 9), (9, WIDEST - 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_widest_without_activation(ctx, dtype, d_in, d_out):
    case = Case(dtype, [150, 3], d_in, d_out, "none", False, residual=True, seed=163)
    case.check_forward(ctx)
    case.check_gradient(ctx)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_activation_many_tiles(ctx, dtype):
    """Enough rows for every pair of blocks to have several tiles, in parts that end anywhere."""
    for d_in, d_out in ((100, 47), (256, 130), (24, 8)):
        Case(dtype, [20011, 0, 17, 9000, 255], d_in, d_out, "none", False, seed=167).check_gradient(ctx)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_in_columns_of_one_buffer(ctx, dtype, gated):
    """Rows, residual branch, result and dZ as columns of the same rows, odd widths; what lies between them keeps its bits."""
    n, d_in, d_out = 700, 13, 21
    up = 24 * (2 if gated else 1)
    buffer = torch.full((n, 200), 5.0, dtype=dtype, device="cuda")
    X, side, out, dz, dx = buffer[:, 8:8 + d_in], buffer[:, 24:24 + d_out], buffer[:, 48:48 + d_out], buffer[:, 72:72 + up], buffer[:, 121:121 + d_in]
    X.copy_(normal(171, n, d_in))
    side.copy_(normal(172, n, d_out))
    W = normal(173, d_in, 2 * d_out if gated else d_out).to(dtype)
    forward, back = (ctx.grouped_gated_linear, ctx.grouped_gated_linear_grad) if gated else (ctx.grouped_linear_act, ctx.grouped_linear_act_grad)
    near_X, near_side = X.contiguous(), side.contiguous()
    forward(X, None, W, act="silu", residual=side, out=out)
    got = back(X, side, None, W, act="silu", out=dx, dz=dz)
    want, grads = forward(near_X, None, W, act="silu", residual=near_side), back(near_X, near_side, None, W, act="silu")
    ctx.check()
    assert torch.equal(out, want) and torch.equal(got[0], grads[0]) and torch.equal(got[1], grads[1])
    for view in (X, side, out, dz, dx):
        view.fill_(5.0)
    assert (buffer == 5).all()
