"""In which type a layer's parameter gradients come, where both a type and a place are given."""
import pytest
import torch

from test_layer_refusals import ctx  # noqa: F401


@pytest.mark.parametrize("wanted,given", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_a_place_of_another_type(ctx, wanted, given):  # noqa: F811
    X, W, dY = torch.zeros(5, 6).bfloat16(), torch.zeros(6, 8).bfloat16(), torch.zeros(5, 8).bfloat16()
    with pytest.raises(TypeError, match="dw"):
        ctx.grouped_linear_act_grad(X, dY, None, W, act="silu", grad_dtype=wanted, dw=torch.zeros(6, 8, dtype=given))
    assert not ctx._lib.calls


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_place_of_the_same_type(ctx, dtype):  # noqa: F811
    X, W, dY = torch.zeros(5, 6).bfloat16(), torch.zeros(6, 8).bfloat16(), torch.zeros(5, 8).bfloat16()
    for kind in (None, dtype):
        dw = torch.zeros(6, 8, dtype=dtype)
        assert ctx.grouped_linear_act_grad(X, dY, None, W, act="silu", grad_dtype=kind, dw=dw)[1] is dw
