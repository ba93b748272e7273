"""fp32 layers over many stages of many tiles: what one block of a pair splits and the other one's MMAs read has come every time."""
import pytest
import torch

from paper_2305_09887_b200 import binding
from test_gpu_layers import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_in,d_out,gated", [(64, 2, False), (256, 256, False), (130, 47, True), (33, 64, False), (1000, 24, False)])
def test_the_same_bits_in_twenty_runs(d_in, d_out, gated):
    ctx = binding.Context(0)
    case = Case(torch.float32, [30011, 0, 9000], d_in, d_out, "silu", gated, seed=101)
    case.check_forward(ctx)
    case.check_gradient(ctx)
    first = [t.clone() for t in (case.forward(ctx), *case.gradient(ctx)[:3])]
    a, b = case.o[0], case.o[-1]
    for _ in range(20):
        for got, want in zip((case.forward(ctx), *case.gradient(ctx)[:3]), first):
            assert torch.equal(got[a:b], want[a:b]) if got.shape[0] == case.X.shape[0] else torch.equal(got, want)
    ctx.check()
