"""Group norm against 64 bits where rows and results lie as torch makes them (whole units, whole loads), and where a block's run of
rows is many loads deep.

How deep fp32 sums are, whatever the number of rows: a lane has the rows of one run, some 120 at most here in up to 4 rows a step; a
block's lanes are joined in 8 steps, a part's runs by 32 lanes (statistics) or 8 (gradients) that have 600 / 8 at most each and 8 more
steps.  DEEP = 240 is above the sum of these; a set's channels come on top.
"""
import pytest
import torch

import row_reference as ref
from paper_2305_09887_b200 import binding
from test_gpu_row_operators import F64, NORM_CASES, TYPES, U, half_step

pytestmark = pytest.mark.gpu
DEEP = 240


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rounding(y, dtype):
    return half_step(dtype) * y.abs() * 1.001 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def check(got, want, tol, what):
    off = (got.to(F64) - want).abs() / tol
    assert off.numel() == 0 or off.max() <= 1, f"{what}: {off.max().item():.3g} tolerances, {int((off > 1).sum())} of {off.numel()}"
    assert not off.isnan().any(), what


def by_rows(stats, o, scope, C):
    """[rows, C] of a column of statistics [.., groups]."""
    groups = stats.shape[1]
    each = stats if scope == "row" else stats.repeat_interleave(torch.tensor([b - a for a, b in zip(o, o[1:])], device="cuda"), 0)
    return each.repeat_interleave(C // groups, 1)


def mean_over(t, o, groups, scope):
    n, C = t.shape
    out = []
    for a, b in zip(o, o[1:]):
        v = t[a:b].view(b - a, groups, C // groups)
        out.append(v.mean(dim=(2,) if scope == "row" else (0, 2), keepdim=True).expand_as(v).reshape(b - a, C) if b > a else t[a:b])
    return torch.cat(out)


def most_over(t, o, groups, scope):
    n, C = t.shape
    out = []
    for a, b in zip(o, o[1:]):
        v = t[a:b].view(b - a, groups, C // groups)
        out.append(v.amax(dim=(2,) if scope == "row" else (0, 2), keepdim=True).expand_as(v).reshape(b - a, C) if b > a else t[a:b])
    return torch.cat(out)


def forward_and_back(ctx, dtype, scope, sizes, C, groups, act, back_act, mean=0.7):
    o = [0]
    for s in sizes:
        o.append(o[-1] + s)
    n, G, per = o[-1], len(sizes), C // groups
    off = torch.tensor(o, device="cuda")
    g = gen(C + groups)
    draw = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dy = (1.5 * draw(n, C) + mean).to(dtype), draw(n, C).to(dtype)
    gamma, beta, slope = 1 + 0.3 * draw(G, C), 0.3 * draw(G, C), torch.linspace(0.1, 0.4, G, device="cuda")
    steps = per + 16 + (DEEP if scope == "part" else 0)
    # forward
    y, st = ctx.group_norm(x, off, groups, gamma, beta, scope=scope, act=act, slope=slope)
    want, stats, u, xhat = ref.group_norm(x.to(F64), o, groups, gamma.to(F64), beta.to(F64), scope, act, slope.to(F64), 1e-5)
    size, big = most_over(x.to(F64).abs(), o, groups, scope), max(gamma.abs().max().item(), 1.0)
    rstd = by_rows(stats[..., 1], o, scope, C)
    # each step of a mean or a variance is three roundings at most (a weighted difference added)
    tol_x = 3 * U * ((steps + 2) * size * rstd + (steps + 6) * xhat.abs())
    tol = 1.1 * (big * tol_x + 4 * U * (xhat.abs() * big + 1.5)) + (2 + u.abs()) * 2.0 ** -22 * u.abs() + 2 * U * want.abs()
    check(y, want, tol + rounding(want, dtype), "y")
    check(st[..., 0], stats[..., 0], 3 * U * (steps + 4) * x.to(F64).abs().max().clamp(min=1) if n else torch.ones(()), "mean")
    # A mean that is off by e adds e^2 to the variance: sum (x - m - e)^2 = sum (x - m)^2 + n e^2, as sum (x - m) = 0.  That is
    # e^2 rstd^2 / 2 of 1 / std, with e up to 3 U steps |x|: what a set of two nearly equal values far from zero shows.
    e = 3 * U * (steps + 2) * (x.to(F64).abs().max() if n else 0)
    check(st[..., 1], stats[..., 1], stats[..., 1] * (3 * U * (steps + 8) * 2 + (e * stats[..., 1]) ** 2 / 2), "1 / std")
    del want, u, xhat, tol, tol_x, y
    # gradient, from rounded statistics; nothing flows through values so near to a kink that fp32 may see the other side
    X, ga, be, sl = (t.to(F64).requires_grad_() for t in (x, gamma, beta, slope))
    want, stats, u, xhat = ref.group_norm(X, o, groups, ga, be, scope, back_act, sl, 1e-5)
    if back_act in ("relu", "prelu"):
        dy = torch.where(u.detach().abs() < 1e-3, torch.zeros((), dtype=dtype, device="cuda"), dy)
    want.backward(dy.to(F64))
    stats, u, xhat = stats.detach(), u.detach(), xhat.detach()
    dx, dg, db, ds = ctx.group_norm_grad(x, dy, stats.float(), off, groups, gamma, beta, scope=scope, act=back_act, slope=slope)
    a, xh, big = dy.to(F64).abs(), xhat.abs(), gamma.abs().max().item() + 0.1
    tol_x = U * (2 * size * rstd + 8 * xh)  # of the statistics given and of three operations
    tol_du = a * (1.1 * big * tol_x + 2.0 ** -20 * (2 + u.abs()) + 4 * U)
    for k, (lo, hi) in enumerate(zip(o, o[1:])):
        r = slice(lo, hi)
        check(db[k], be.grad[k], tol_du[r].sum(0) + U * DEEP * (1.1 * a[r]).sum(0) + 1e-30, f"dbeta {k}")
        check(dg[k], ga.grad[k], (tol_du * xh + 1.1 * a * tol_x)[r].sum(0) + U * DEEP * (1.1 * a * xh)[r].sum(0) + 1e-30, f"dgamma {k}")
        if back_act == "prelu":  # a lane adds up its eight channels of every row
            check(ds[k], sl.grad[k], (a * (big * tol_x + 4 * U * (xh * big + 1.5)))[r].sum() + U * 8 * DEEP * (a * u.abs())[r].sum() + 1e-30, f"dslope {k}")
    deep = per + 24 + (DEEP if scope == "part" else 0)
    over = lambda t: mean_over(t, o, groups, scope)  # noqa: E731
    m1, m2 = over(1.1 * big * a), over(1.1 * big * a * xh)
    tol = rstd * (big * tol_du + over(big * tol_du) + xh * over(big * (tol_du * xh + 1.1 * a * tol_x)) + tol_x * m2
                  + U * (deep * m1 + deep * xh * m2 + 8 * big * 1.1 * a))
    check(dx, X.grad, tol + rounding(X.grad, dtype), "dx")


ACTS = ["none", "relu", "prelu", "silu"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("sizes,C,groups", NORM_CASES)
def test_rows_as_they_come(ctx, dtype, scope, sizes, C, groups):
    k = (C // 2 + len(sizes)) % 4
    forward_and_back(ctx, dtype, scope, sizes, C, groups, ACTS[k], ACTS[k - 1])


# Rows of every kind of set: runs of lanes, several warps' lanes, within a unit, sharing units in a warp and in several, and the rest
RUNS = [(70_000, 512, 8), (70_000, 512, 1), (70_000, 384, 8), (70_000, 300, 3), (300_000, 64, 8), (300_000, 64, 32), (300_000, 90, 9), (300_000, 60, 20),
        (300_000, 100, 4), (1_000_000, 16, 2), (20_000, 2048, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("n,C,groups", RUNS)
def test_runs_that_are_many_loads_deep(ctx, dtype, scope, n, C, groups):
    sizes = [n // 2 + 77, 0, 13, n - n // 2 - 90]
    k = (C // 2 + groups) % 4
    forward_and_back(ctx, dtype, scope, sizes, C, groups, ACTS[k], ACTS[k - 1])
    torch.cuda.empty_cache()


@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("C,groups", [(512, 8), (64, 32), (300, 3)])
def test_deep_runs_far_from_zero(ctx, scope, C, groups):
    """A mean of a thousand deviations keeps its digits over many joined batches."""
    forward_and_back(ctx, torch.float32, scope, [90_000, 20_000], C, groups, "none", "none", mean=1500.0)
