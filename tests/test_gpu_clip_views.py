"""Clipping views of something larger: what lies around a view keeps its bits, whether the view is taken or refused."""
import pytest
import torch

from paper_2305_09887_b200 import binding
from layer_reference import rounding
from test_gpu_clip import NORM, TYPES
from test_gpu_layers import normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [5, binding.MAX_GROUPS, binding.MAX_GROUPS + 1, 3000])
@pytest.mark.parametrize("beside", [False, True])
def test_a_column(ctx, dtype, rows, beside):
    whole = normal(1, rows, 3).to(dtype)
    before, column = whole.clone(), whole[:, 1]
    other = normal(2, 7).to(dtype)
    grads = [column, other] if beside else [column]
    if beside or rows > binding.MAX_GROUPS:
        for call in (lambda: ctx.clip_gradients(grads, 0.5), lambda: ctx.gradient_norms(grads), lambda: ctx.clip_gradients([before[:, 1].contiguous(), other][:len(grads)], 0.5, out=grads)):
            with pytest.raises(ValueError, match="contiguous"):
                call()
        torch.cuda.synchronize()
        assert torch.equal(whole, before)
        return
    want = before[:, 1].double().norm()
    norm = ctx.clip_gradients(grads, 0.5)
    assert abs(norm.item() - want.item()) <= NORM * want.item()
    assert torch.equal(whole[:, ::2], before[:, ::2])
    near = before[:, 1].contiguous()
    ctx.clip_gradients([near], 0.5)
    # (the sums of squares are put together in another order: two factors in fp32 that are a step apart, and a rounding to the type each)
    most = (2 * NORM + 2.0**-22) * near.double().abs() + 2 * rounding(near.double(), dtype)
    assert ((column.double() - near.double()).abs() <= most).all()
