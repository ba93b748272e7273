"""Gradients that are sums over many rows, of one sign and of very different sizes: db, the slope's and dW against sums in 64 bits."""
import pytest
import torch

from paper_2305_09887_b200 import binding

pytestmark = pytest.mark.gpu
HALF = 2.0**-24  # half a step of fp32
N, D = 6_000_000, 8


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def positive(n, d, dtype, seed):
    """Values above zero, most of them between 2^-6 and 2^6: sums of a few thousand need more bits than fp32 has."""
    return torch.exp(1.4 * torch.randn(n, d, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")).clamp(2.0**-8, 2.0**8).to(dtype)


def inputs(dtype, gated, sign=1.0):
    """Z is `sign` everywhere, in both halves."""
    X = torch.zeros(N, D, dtype=dtype, device="cuda")
    X[:, 0] = 1
    W = torch.zeros(D, 2 * D if gated else D, dtype=dtype, device="cuda")
    W[0] = sign
    return X, W, torch.zeros_like(W[0])


def calls(ctx, gated):
    return ctx.grouped_gated_linear_grad if gated else ctx.grouped_linear_act_grad


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_bias_behind_an_activation(ctx, dtype, gated):
    """Sums of 32 rows are truncated twice, by 2^-23 each.  Everything after that is rounded to nearest, without a preferred sign: chains of 64 tiles' sums, whose errors
    have a standard deviation below sqrt(64 / 3) half steps, of which six are taken, and then fewer, longer steps, in 64 bits, and the result's rounding."""
    X, W, b = inputs(dtype, gated)
    dY = positive(N, D, dtype, 1)
    db = calls(ctx, gated)(X, dY, None, W, b, act="relu", need_dx=False, grad_dtype=torch.float32)[2]
    want = dY.sum(0, dtype=torch.float64).repeat(2 if gated else 1)
    tol = 2 * 2.0**-23 + (6 * (64 / 3) ** 0.5 + 2) * HALF
    assert ((db.double() - want).abs() <= tol * want).all(), ((db.double() - want) / want).tolist()


@pytest.mark.parametrize("gated", [False, True])
def test_no_truncation_in_long_chains(ctx, gated):
    """Values between 4 and 8 (multiples of 2^-8) and between 2^-4 and 2^-3 (of 2^-14): 32 of them have an exact sum in fp32, 2,048 have not.  Sums of 64 tiles, eight by
    each of half as many pairs as there are SMs, then eleven of these, all rounded to nearest: independent errors, of which six standard deviations
    are taken, and the result's rounding.  (Accumulators that truncate over 64 tiles were off by 2e-7 and more.)"""
    X, W, b = inputs(torch.float16, gated)
    g = torch.Generator("cuda").manual_seed(7)
    scale = torch.where(torch.rand(N, D, generator=g, device="cuda") < 0.5, 4.0, 2.0**-4)
    dY = (scale * (1 + torch.rand(N, D, generator=g, device="cuda") * 0.999)).half()
    db = calls(ctx, gated)(X, dY, None, W, b, act="relu", need_dx=False, grad_dtype=torch.float32)[2]
    want = dY.sum(0, dtype=torch.float64).repeat(2 if gated else 1)
    pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
    tol = 6 * ((64 / 3) ** 0.5 + (11 / 3) ** 0.5) * HALF / (8 * pairs) ** 0.5 + HALF
    assert ((db.double() - want).abs() <= tol * want).all(), (tol, ((db.double() - want) / want).tolist())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_bias_without_an_activation(ctx, dtype):
    """The rows are cut into 2 x 74 chunks of 40,541 (on 148 SMs; fewer and longer ones on fewer).  16-bit rows: a lane adds up every sixteenth of a chunk one by one, 2,560 roundings to nearest, standard deviation
    below sqrt(2,560 / 3) half steps of the largest partial sum, of which six are taken.  fp32 rows: 32 values a sum, and 80 of those.  The joins of lanes and chunks, 300 at most, likewise."""
    X, W, b = inputs(dtype, False)
    dY = positive(N, D, dtype, 2)
    db = ctx.grouped_linear_act_grad(X, dY, None, W, b, act="none", need_dx=False, grad_dtype=torch.float32)[2]
    want = dY.sum(0, dtype=torch.float64)
    steps = (112 if dtype == torch.float32 else 2560) + 300
    tol = (6 * (steps / 3) ** 0.5 + 2) * HALF
    assert ((db.double() - want).abs() <= tol * want).all(), ((db.double() - want) / want).tolist()


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("gated", [False, True])
def test_fp32_weights_and_bias(ctx, gated, act):
    """dW's first row is the sum of dZ as well, as products with one: 32 rows in the tensor cores' accumulators (twelve additions that truncate, by 2^-23 each), then 1,270 sums of a chunk rounded
    to nearest (six standard deviations of them), then 148 chunks.  X's other columns are zero, and so are the other rows."""
    X, W, b = inputs(torch.float32, gated)
    dY = positive(N, D, torch.float32, 3)
    _, dw, db, _ = calls(ctx, gated)(X, dY, None, W, b, act=act, need_dx=False)
    want = dY.sum(0, dtype=torch.float64).repeat(2 if gated else 1)
    tol = (6 * (412 / 3) ** 0.5 + 2) * HALF
    assert ((db.double() - want).abs() <= tol * want).all(), ((db.double() - want) / want).tolist()
    tol = 2.0**-22 + 12 * 2.0**-23 + (6 * (1420 / 3) ** 0.5 + 2) * HALF
    assert ((dw[0].double() - want).abs() <= tol * want).all(), ((dw[0].double() - want) / want).tolist()
    assert not dw[1:].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_slope(ctx, dtype):
    """Z is -1, the slope's gradient minus the sum of dY.  Of 81,081 rows of a pair of blocks (74 pairs) a lane has one of 256 and eight columns: 317 tiles' sums of eight, 400 roundings with
    the joins' (six standard deviations), then in 64 bits."""
    X, W, b = inputs(dtype, False, -1.0)
    dY = positive(N, D, dtype, 4)
    dslope = ctx.grouped_linear_act_grad(X, dY, None, W, b, act="prelu", slope=torch.tensor(0.3, device="cuda"), need_dx=False)[3]
    want = -dY.sum(dtype=torch.float64)
    assert abs(dslope.double() - want) <= (6 * (400 / 3) ** 0.5 + 8) * HALF * abs(want), ((dslope.double() - want) / want).item()
