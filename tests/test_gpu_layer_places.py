"""Results of layers in the place of what has been read by then: the same bits as results of their own."""
import pytest
import torch

from paper_2305_09887_b200 import binding
from test_gpu_layers import TYPES, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("width", [47, 64, 300])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(ctx, dtype, gated, width, pad, shift):
    case = Case(dtype, [1500, 0, 800], width, width, "prelu", gated, residual=True, pad=pad, shift=shift, seed=113)
    a, b = case.o[0], case.o[-1]
    want = case.forward(ctx)
    dx, dw, db, dslope = case.gradient(ctx)
    assert torch.equal(case.forward(ctx, out=case.residual)[a:b], want[a:b])
    got = case.gradient(ctx, out=case.dY, dw=case.W, db=case.b, dslope=case.slope)
    ctx.check()
    assert got[0] is case.dY and torch.equal(case.dY[a:b], dx[a:b])
    assert torch.equal(case.W, dw) and torch.equal(case.b, db) and torch.equal(case.slope, dslope)


@pytest.mark.parametrize("dtype", TYPES)
def test_refused_with_nothing_written(ctx, dtype):
    case = Case(dtype, [300], 40, 40, "silu", False, residual=True, seed=127)
    wide = torch.full((case.X.shape[0], 80), 5.0, dtype=dtype, device="cuda")
    out = wide.view(-1)[:case.X.shape[0] * 40].view(-1, 40)  # the rows of `wide` half as far apart
    case.residual = wide[:, :40]
    with pytest.raises(binding.RtmaError, match="other rows"):
        case.forward(ctx, out=out)
    torch.cuda.synchronize()
    assert (wide == 5).all()
