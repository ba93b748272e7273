"""The operators on the rows of many parts where their arguments are at an end: the most rows, expanded and overlapping tensors,
runs of rows of every length, values whose squares do not fit.  Tolerances as in test_gpu_row_operators.py."""
import pytest
import torch

from paper_2305_09887_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F64 = torch.float64


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def test_weight_gradient_of_nearly_two_to_the_31_rows(ctx):
    """Every row counts: sums of ones.  A chunk's sum, below 2^24, is exact in fp32; its slots are added up with a rounding each."""
    n = 2_140_000_000
    one = torch.ones(n, 1, dtype=torch.bfloat16, device="cuda")
    dw, db = ctx.grouped_linear_dw(one, one, None)
    for got in (dw, db):
        assert abs(got.item() - n) <= 600 * 2 * U * n
    ctx.check()
