"""Tensors that clipping takes only where their values lie as it says: what the binding hands on of views, and what it refuses."""
import pytest
import torch

from paper_2305_09887_b200 import binding
from test_layer_refusals import ctx  # noqa: F401

LONG = binding.MAX_GROUPS + 1


def column(n):
    return torch.zeros(n, 3)[:, 0]


# gradients of which one is no run of adjacent values, and of which no first dimension is as long as the others'
SCATTERED = {
    "a column beside another length": lambda: [torch.zeros(7), column(5)],
    "a column first": lambda: [column(5), torch.zeros(7)],
    "every second of many": lambda: [torch.zeros(2 * LONG)[::2]],
    "a long column": lambda: [column(5000)],
    "one value for many": lambda: [torch.zeros(1).expand(5000)],
    "one value for a few, beside another length": lambda: [torch.zeros(1).expand(5), torch.zeros(7)],
    "a column beside a single value": lambda: [column(5), torch.zeros(())],
}


@pytest.mark.parametrize("which", SCATTERED)
def test_scattered_gradients_of_one_part(ctx, which):  # noqa: F811
    for call in (lambda g: ctx.clip_gradients(g, 1.0), ctx.gradient_norms, lambda g: ctx.clip_gradients(g, 1.0, out=[torch.zeros(t.shape) for t in g])):
        with pytest.raises(ValueError, match="contiguous"):
            call(SCATTERED[which]())
    assert not ctx._lib.calls


@pytest.mark.parametrize("which", SCATTERED)
def test_scattered_results_of_one_part(ctx, which):  # noqa: F811
    out = SCATTERED[which]()
    with pytest.raises(ValueError, match="contiguous"):
        ctx.clip_gradients([torch.zeros(t.shape) for t in out], 1.0, out=out)
    assert not ctx._lib.calls


@pytest.mark.parametrize("grads,out", [
    ([torch.zeros(1).expand(6)], None), ([torch.zeros(6)], [torch.zeros(1).expand(6)]), ([torch.zeros(6, 2)], [torch.zeros(1, 2).expand(6, 2)]),
])
@pytest.mark.parametrize("parts", [1, 6])
def test_results_without_memory_of_their_own(ctx, grads, out, parts):  # noqa: F811
    with pytest.raises((ValueError, binding.RtmaError)):
        ctx.clip_gradients(grads, 1.0, parts=parts, out=out)
    assert not ctx._lib.calls


def test_views_that_are_taken(ctx):  # noqa: F811
    """A first dimension as long as the others' (a row for each of something's replicas) makes single values that lie apart shares of their own."""
    t = torch.zeros(12)[::2]
    ctx.clip_gradients([t, torch.zeros(6, 3)], 1.0)
    (name, args), = ctx._lib.calls
    first, second = (binding.GRADIENT.unpack_from(args[2], binding.GRADIENT.size * i) for i in range(2))
    assert name == "rtma_clip_gradients" and args[3:5] == (6, 1)
    assert first[0] == first[1] == t.data_ptr() and first[2:5] == (1, 2, 2)
    assert second[2:5] == (3, 3, 3)
