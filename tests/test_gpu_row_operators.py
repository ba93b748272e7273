"""Dropout, group norm and grouped products on the rows of many parts, against their definitions in 64 bits.

Tolerances are worst cases of the arithmetic.  h = eps / 2 of the rows' type is what one rounding of a result costs.  A sum of k
products in fp32, rounded or truncated at every step, is off by at most (k + c) 2^-23 of the sum of the products' magnitudes, c for
the few steps that join partial sums.
"""
import math

import numpy as np
import pytest
import torch

import row_reference as ref
from paper_2305_09887_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
F64 = torch.float64


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounding(y, dtype):
    """Half a step of every value (the smallest step of the type for tiny ones)."""
    return half_step(dtype) * y.abs() * 1.001 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def make_rows(n, d, dtype, seed, pad=0, shift=0, scale=1.0, mean=0.0):
    """Rows on the GPU whose distance is d + pad elements, `shift` elements behind an aligned address; everything else is NaN."""
    host = (torch.randn(n, d, generator=gen(seed)) * scale + mean).to(dtype)
    flat = torch.full((n * (d + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    view = flat[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
    view.copy_(host)
    return host, view, flat


def offsets_of(sizes, first=0):
    o = [first]
    for s in sizes:
        o.append(o[-1] + s)
    return o, torch.tensor(o, dtype=torch.int64, device="cuda")


def assert_close(got, want, tol, what=""):
    got, want = got.detach().cpu().to(F64), want.detach()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}: " \
                          f"{got[bad][0].item()} for {want[bad][0].item()}, off by {((got - want).abs() / tol)[bad].max().item():.3g} tolerances"


# ---- dropout --------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,pad,shift", [(1, 1, 0, 0), (1, 8, 0, 0), (33, 7, 0, 0), (257, 64, 0, 0), (100, 47, 1, 3), (64, 128, 8, 8), (5, 1030, 0, 1)])
@pytest.mark.parametrize("p", [0.0, 0.3, 1.0])
def test_dropout(ctx, dtype, n, d, pad, shift, p):
    host, x, _ = make_rows(n, d, dtype, 1, pad, shift)
    rhost, res, _ = make_rows(n, d, dtype, 2, shift, 0)
    ids = torch.randint(-2**31, 2**31 - 1, (n,), generator=gen(3), dtype=torch.int64).to(torch.int32)
    y = ctx.dropout(x, p, 99)
    want = ref.dropout(host, p, 99)
    assert_close(y, want, 2.01 * rounding(want, dtype), "plain")  # the product in fp32, then the type
    y = ctx.dropout(x, p, -5, row_ids=ids.cuda(), residual=res)
    want = ref.dropout(host, p, -5, ids.numpy())
    both = want + rhost.to(F64)
    assert_close(y, both, rounding(both, dtype) + 4 * U * (want.abs() + rhost.to(F64).abs()), "ids, residual")


def test_dropout_keeps_the_share_and_drops_nan(ctx):
    x = torch.ones(4096, 256, device="cuda")
    y = ctx.dropout(x, 0.25, 7)
    kept = (y != 0).double().mean().item()
    assert abs(kept - 0.75) < 6 * math.sqrt(0.75 * 0.25 / x.numel())
    assert set(y.unique().tolist()) == {0.0, np.float32(65536 / 49152).item()}
    x.fill_(float("nan"))
    y = ctx.dropout(x, 0.25, 7)
    assert torch.equal(y.isnan(), ctx.dropout(torch.ones_like(x), 0.25, 7) != 0)


@pytest.mark.parametrize("d", [13, 64])
def test_dropout_in_place_and_beside_it(ctx, d):
    host, x, flat = make_rows(300, d, torch.bfloat16, 4, pad=3)
    want = ctx.dropout(x, 0.5, 11)
    around = flat.clone()
    ctx.dropout(x, 0.5, 11, out=x)
    assert torch.equal(x, want)
    around[:300 * (d + 3)].view(300, d + 3)[:, :d] = want
    assert torch.equal(around.view(torch.int16), flat.view(torch.int16))  # the padding between rows is as it was


def test_a_node_has_the_same_mask_in_every_partition(ctx):
    n, d = 5_000, 40
    x = torch.randn(n, d, device="cuda")
    whole = ctx.dropout(x, 0.4, 5)
    for M, seed in ((3, 1), (8, 2)):
        _, _, perm, _ = ctx.partition(n, None, seed, M)
        assert torch.equal(ctx.dropout(ctx.gather_rows(x, perm), 0.4, 5, row_ids=perm), ctx.gather_rows(whole, perm))


# ---- group norm -----------------------------------------------------------------------------------------

NORM_CASES = [
    # sizes of the parts, C, groups
    ([1], 8, 1), ([1], 2, 1), ([7, 0, 1, 30], 64, 8), ([130, 3], 47, 47), ([130, 3], 47, 1), ([64, 200], 100, 4), ([33, 0], 90, 9),
    ([37, 0, 90], 240, 10), ([61, 5], 250, 2), ([3, 300], 54, 6), ([40, 1], 27, 3), ([200], 144, 16), ([9, 50], 300, 3), ([20, 30], 12, 3),
    ([50, 3], 384, 2), ([41], 384, 32), ([30, 1], 2040, 3), ([17, 40], 1020, 17), ([25], 1100, 100), ([19, 2], 700, 2),
    ([30, 7], 1536, 3), ([21], 1000, 1), ([40, 0, 9], 2048, 8), ([25, 3], 600, 1), ([90, 4], 64, 32), ([33], 36, 9), ([5, 70], 12, 12),
    ([50, 60], 256, 32), ([70], 512, 1), ([9, 12], 1024, 8), ([5, 9], 2048, 2), ([0, 0], 32, 4), ([2500], 24, 3), ([40, 50], 384, 1),
]


def norm_inputs(sizes, C, dtype, seed, pad, shift, behind=3):
    o, off = offsets_of(sizes, 2)
    n = o[-1] + behind
    host, x, _ = make_rows(n, C, dtype, seed, pad, shift, scale=1.5, mean=0.7)
    G = len(sizes)
    gamma = 1 + 0.3 * torch.randn(G, C, generator=gen(seed + 1))
    beta = 0.3 * torch.randn(G, C, generator=gen(seed + 2))
    slope = torch.linspace(0.1, 0.4, G)
    return o, off, n, host, x, gamma, beta, slope


def norm_bounds(host, o, groups, scope, stats, xhat):
    """What fp32 costs xhat, for every value: the mean (sums of at most `deep` steps), the difference, and 1 / std."""
    n, C = host.shape
    x = host.to(F64).abs().view(n, groups, C // groups)
    per = C // groups
    deep = 0
    size = torch.zeros(n, groups, 1, dtype=F64)
    rstd = torch.zeros(n, groups, 1, dtype=F64)
    row = 0
    for g, (a, b) in enumerate(zip(o, o[1:])):
        m = x[a:b]
        size[a:b] = m.amax(2, keepdim=True) if scope == "row" else (m.amax(dim=(0, 2))[None, :, None] if b > a else 0)
        rstd[a:b] = stats[row:row + b - a, :, 1:] if scope == "row" else stats[g:g + 1, :, 1:]
        row += b - a
        deep = max(deep, b - a)
    # a set's values are summed by lanes: at most per + 8 steps in a row, the rows of a part at most so many more
    steps = per + 16 + (deep if scope == "part" else 0)
    return (U * ((steps + 2) * size * rstd + (steps + 6) * xhat.abs().view(n, groups, per))).view(n, C)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("sizes,C,groups", NORM_CASES)
def test_group_norm(ctx, dtype, scope, sizes, C, groups):
    act = ["none", "relu", "prelu", "silu"][(C + len(sizes)) % 4]
    pad, shift = [(0, 0), (5, 3), (8, 0)][(C // 2 + groups) % 3]
    o, off, n, host, x, gamma, beta, slope = norm_inputs(sizes, C, dtype, C + groups, pad, shift)
    for p in (0.0, 0.4):
        kept, scale = ref.mask(31, np.arange(n), C, p)
        want, stats, u, xhat = ref.group_norm(host.to(F64), o, groups, gamma.to(F64), beta.to(F64), scope, act, slope.to(F64), 1e-5, kept, scale)
        out = torch.full((n, C + 1), 7.0, dtype=dtype, device="cuda")[:, :C]
        st = torch.full((n if scope == "row" else len(sizes), groups, 2), 5.0, device="cuda")
        y, _ = ctx.group_norm(x, off, groups, gamma.cuda(), beta.cuda(), scope=scope, act=act, slope=slope.cuda(), p=p, seed=31, out=out, stats=st)
        tol_x = norm_bounds(host, o, groups, scope, stats, xhat)
        big = max(gamma.abs().max().item(), 1.0)
        # a Lipschitz constant of 1.1 (SiLU), the fast exponential's relative error of (2 + |u|) 2^-22, dropout's product
        tol = scale * (1.1 * (big * tol_x + 4 * U * (xhat.abs() * big + 1.5)) + (2 + u.abs()) * 2.0 ** -22 * u.abs()) + 2 * U * want.abs()
        inside = slice(o[0], o[-1])
        assert_close(y[inside], want[inside], (tol + rounding(want, dtype))[inside], f"p={p} {act}")
        assert (y[:o[0]] == 7).all() and (y[o[-1]:] == 7).all()
        got = st.cpu().to(F64)
        if scope == "row":
            assert (got[:o[0]] == 5).all() and (got[o[-1]:] == 5).all()
            got = got[inside]
        magnitude = host.to(F64)[inside].abs().max() if o[-1] > o[0] else torch.tensor(0.0)
        steps = C // groups + 16 + max(sizes)
        assert_close(got[..., 0], stats[..., 0], U * (steps + 4) * magnitude + 1e-30, "mean")
        assert_close(got[..., 1], stats[..., 1], U * (steps + 8) * 2 * stats[..., 1] + 1e-30, "1 / std")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("sizes,C,groups", NORM_CASES)
def test_group_norm_grad(ctx, dtype, scope, sizes, C, groups):
    act = ["none", "relu", "prelu", "silu"][(C + len(sizes) + 1) % 4]
    pad, shift = [(0, 0), (5, 3), (8, 0)][(C // 2 + groups) % 3]
    o, off, n, host, x, gamma, beta, slope = norm_inputs(sizes, C, dtype, C + groups + 50, pad, shift)
    p = 0.3 if C % 3 else 0.0
    kept, scale = ref.mask(8, np.arange(n), C, p)
    X, ga, be, sl = (t.to(F64).requires_grad_() for t in (host, gamma, beta, slope))
    want, stats, u, xhat = ref.group_norm(X, o, groups, ga, be, scope, act, sl, 1e-5, kept, scale)
    dhost, _, _ = make_rows(n, C, dtype, C + 77)
    # the derivative jumps where u = 0: nothing flows through values so near to it that fp32 may see the other side
    dhost = torch.where(u.detach().abs() < 1e-3, torch.zeros((), dtype=dtype), dhost)
    if act in ("none", "silu"):
        dhost = make_rows(n, C, dtype, C + 77)[0]
    want.backward(dhost.to(F64))
    st = stats.detach().float()
    if scope == "row":
        full = torch.full((n, groups, 2), float("nan"))
        full[o[0]:o[-1]] = st
        st = full
    out = torch.full((n, C), 7.0, dtype=dtype, device="cuda")
    dx, dg, db, ds = ctx.group_norm_grad(x, dhost.cuda(), st.cuda(), off, groups, gamma.cuda(), beta.cuda(), scope=scope, act=act,
                                         slope=slope.cuda(), p=p, seed=8, out=out)
    # magnitudes that the sums are made of
    a = dhost.to(F64).abs() * scale
    xh, big = xhat.detach().abs(), gamma.abs().max().item() + 0.1
    s64 = stats.detach()
    tol_x = norm_bounds(host, o, groups, scope, s64, xhat.detach()) + 4 * U * xh  # the statistics given are rounded as well
    tol_du = a * (1.1 * big * tol_x + 2.0 ** -20 * (2 + u.detach().abs()) + 4 * U)
    per = C // groups
    for g, (lo, hi) in enumerate(zip(o, o[1:])):
        rows = slice(lo, hi)
        steps = (hi - lo) + 24
        tb, tg = tol_du[rows].sum(0), (tol_du * xh + 1.1 * a * tol_x)[rows].sum(0)
        sum_b, sum_g = (1.1 * a)[rows].sum(0), (1.1 * a * xh)[rows].sum(0)
        assert_close(db[g], be.grad[g], tb + U * steps * sum_b + 1e-30, "dbeta")
        assert_close(dg[g], ga.grad[g], tg + U * steps * sum_g + 1e-30, "dgamma")
        if act == "prelu":
            ud = (a * u.detach().abs())[rows].sum()
            tu = (a * big * tol_x + 4 * U * a * (xh * big + 1.5))[rows].sum()
            assert_close(ds[g], sl.grad[g], tu + U * (steps + C) * ud + 1e-30, "dslope")
        if hi == lo:
            assert not dg[g].any() and not db[g].any()
            continue
        r = (s64[lo - o[0]:hi - o[0], :, 1:] if scope == "row" else s64[g:g + 1, :, 1:]).expand(hi - lo, groups, per).reshape(hi - lo, C)
        over = (2,) if scope == "row" else (0, 2)
        mean_of = lambda t: t[rows].reshape(hi - lo, groups, per).mean(dim=over, keepdim=True).expand(hi - lo, groups, per).reshape(hi - lo, C)  # noqa: E731
        deep = per + 24 + (hi - lo if scope == "part" else 0)
        m1, m2 = mean_of(1.1 * big * a), mean_of(1.1 * big * a * xh)
        tol = r * (big * tol_du[rows] + mean_of(big * tol_du) + xh[rows] * mean_of(big * (tol_du * xh + 1.1 * a * tol_x)) + tol_x[rows] * m2
                   + U * (deep * m1 + deep * xh[rows] * m2 + 8 * big * 1.1 * a[rows]))
        assert_close(dx[rows], X.grad[rows], tol + rounding(X.grad[rows], dtype), "dx")
    assert (dx[:o[0]] == 7).all() and (dx[o[-1]:] == 7).all()


@pytest.mark.parametrize("scope", ["row", "part"])
def test_group_norm_shared_parameters_views_and_in_place(ctx, scope):
    sizes, C, groups, M = [40, 0, 75], 64, 4, 3
    o, off = offsets_of(sizes)
    x = torch.randn(o[-1], C, generator=gen(1)).cuda()
    dy = torch.randn(o[-1], C, generator=gen(2)).cuda()
    gamma, beta, slope = (torch.randn(s, generator=gen(3)).cuda() for s in (C, C, 1))
    how = dict(scope=scope, act="prelu", p=0.2, seed=3)
    y, st = ctx.group_norm(x, off, groups, gamma, beta, slope=slope, **how)
    each = dict(gamma=gamma.expand(M, C).contiguous(), beta=beta.expand(M, C).contiguous(), slope=slope.expand(M).contiguous())
    y2, st2 = ctx.group_norm(x, off, groups, **each, **how)
    assert torch.equal(y, y2) and torch.equal(st, st2)
    shared = ctx.group_norm_grad(x, dy, st, off, groups, gamma, beta, slope=slope, **how)
    parts = ctx.group_norm_grad(x, dy, st, off, groups, **each, **how)
    assert torch.equal(shared[0], parts[0])
    for s, t in zip(shared[1:], parts[1:]):
        want = (t[0] + t[1]) + t[2]
        assert torch.equal(s.reshape(want.shape if want.dim() else ()), want)
    # parameters and gradients where they lie in a replica's flat vector
    P = 3 * C + 7
    flat, grads = torch.full((M, P), float("nan"), device="cuda"), torch.full((M, P), 9.0, device="cuda")
    flat[:, 5:5 + C], flat[:, 5 + C:5 + 2 * C], flat[:, 5 + 2 * C] = gamma, beta, slope
    cut = lambda t: dict(gamma=t[:, 5:5 + C], beta=t[:, 5 + C:5 + 2 * C], slope=t[:, 5 + 2 * C])  # noqa: E731
    y3, _ = ctx.group_norm(x, off, groups, **cut(flat), **how)
    assert torch.equal(y, y3)
    ctx.group_norm_grad(x, dy, st, off, groups, **cut(flat), **how, **{"d" + k: v for k, v in cut(grads).items()})
    for mine, want in zip(cut(grads).values(), parts[1:]):
        assert torch.equal(mine, want)
    assert (grads[:, :5] == 9).all() and (grads[:, 6 + 2 * C:] == 9).all()
    # in place
    z = x.clone()
    ctx.group_norm(z, off, groups, gamma, beta, slope=slope, out=z, **how)
    assert torch.equal(z, y)
    for keep in (0, 1):
        a, b = x.clone(), dy.clone()
        ctx.group_norm_grad(a, b, st, off, groups, gamma, beta, slope=slope, out=(a, b)[keep], **how)
        assert torch.equal((a, b)[keep], shared[0])
    # no parameters at all
    y4, st4 = ctx.group_norm(x, off, groups, scope=scope)
    y5, _ = ctx.group_norm(x, off, groups, torch.ones(C, device="cuda"), torch.zeros(C, device="cuda"), scope=scope)
    assert torch.equal(y4, y5)
    dx, dg, db, ds = ctx.group_norm_grad(x, dy, st4, off, groups, scope=scope)
    assert dg is None and db is None and ds is None and dx.isfinite().all()


@pytest.mark.parametrize("scope", ["row", "part"])
def test_group_norm_far_from_zero_and_outliers(ctx, scope):
    """A mean a thousand times the deviation, a first row far off, a constant part: statistics hold their digits."""
    C, groups = 32, 2
    o, off = offsets_of([3000, 500, 200])
    x = torch.randn(o[-1], C, generator=gen(1)) + 1000
    x[o[1]] = 1e4  # the second part's first row
    x[o[2]:] = 3.25
    y, st = ctx.group_norm(x.cuda(), off, groups, scope=scope)
    want, stats, _, xhat = ref.group_norm(x.to(F64), o, groups, torch.ones(3, C, dtype=F64), torch.zeros(3, C, dtype=F64), scope, "none", None, 1e-5)
    assert_close(st[..., 1], stats[..., 1], 2e-5 * stats[..., 1], "1 / std")
    tol = norm_bounds(x, o, groups, "row", st.cpu().to(F64) if scope == "row" else stats.repeat_interleave(torch.tensor([3000, 500, 200]), 0), xhat)
    assert_close(y, want, tol + 2e-5 * xhat.abs(), "y")
    assert not y[o[2]:].any()


@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_group_norm_of_values_that_are_not_finite(ctx, scope, bad):
    """They stay within their set: a row's set, or a part's."""
    C, groups = 48, 3
    o, off = offsets_of([20, 30])
    x = torch.randn(50, C, generator=gen(5)).cuda()
    clean, _ = ctx.group_norm(x, off, groups, scope=scope, act="relu")
    x[25, 17] = bad
    y, _ = ctx.group_norm(x, off, groups, scope=scope, act="relu")
    hit = torch.zeros_like(x, dtype=torch.bool)
    if scope == "row":
        hit[25, 16:32] = True
    else:
        hit[20:, 16:32] = True
    assert torch.equal(y[~hit], clean[~hit]) and y[hit].isnan().all()


# ---- grouped products -----------------------------------------------------------------------------------

LINEAR_CASES = [
    # sizes of the parts, d_in, d_out
    ([1], 1, 1), ([1], 64, 64), ([5, 0, 3], 7, 13), ([130, 64, 1], 64, 47), ([300], 100, 256), ([127, 129, 0, 256], 256, 130),
    ([64, 40], 33, 300), ([500, 1, 200], 71, 90), ([200], 512, 2), ([90, 30], 2, 512), ([0, 0], 16, 16), ([10] * 70, 24, 40),
    ([700, 300], 128, 128), ([50], 1030, 65),
]


def linear_inputs(sizes, d_in, d_out, dtype, seed):
    pad, shift = [(0, 0), (1, 1), (8, 8), (3, 0)][(d_in + d_out) % 4]
    o, off = offsets_of(sizes, 1)
    n = o[-1] + 2
    X = make_rows(n, d_in, dtype, seed, pad, shift)
    dY = make_rows(n, d_out, dtype, seed + 1, shift, pad)
    W = (torch.randn(len(sizes), d_in, d_out, generator=gen(seed + 2)) / math.sqrt(d_in)).to(dtype)
    b = torch.randn(len(sizes), d_out, generator=gen(seed + 3)).to(dtype)
    return o, off, n, X, dY, W, b


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", LINEAR_CASES)
def test_grouped_linear(ctx, dtype, sizes, d_in, d_out):
    o, off, n, (host, x, _), _, W, b = linear_inputs(sizes, d_in, d_out, dtype, d_in)
    for bias in (b, None):
        want = ref.linear(host, o, W, bias)
        size = ref.linear(host.abs(), o, W.abs(), None if bias is None else bias.abs())
        out = torch.full((n, d_out + 3), 7.0, dtype=dtype, device="cuda")
        ctx.grouped_linear(x, off, W.cuda(), None if bias is None else bias.cuda(), out=out[:, :d_out])
        inside = slice(o[0], o[-1])
        assert_close(out[inside, :d_out], want[inside], (rounding(want, dtype) + (d_in + 16) * 2 * U * size)[inside], "y")
        assert (out[:o[0]] == 7).all() and (out[o[-1]:] == 7).all() and (out[:, d_out:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", LINEAR_CASES)
def test_grouped_linear_dx(ctx, dtype, sizes, d_in, d_out):
    o, off, n, _, (host, dy, _), W, _ = linear_inputs(sizes, d_in, d_out, dtype, d_in + 5)
    want, size = ref.linear(host, o, W.mT), ref.linear(host.abs(), o, W.mT.abs())
    out = torch.full((n, d_in + 1), 7.0, dtype=dtype, device="cuda")
    ctx.grouped_linear_dx(dy, off, W.cuda(), out=out[:, :d_in])
    inside = slice(o[0], o[-1])
    assert_close(out[inside, :d_in], want[inside], (rounding(want, dtype) + (d_out + 16) * 2 * U * size)[inside], "dx")
    assert (out[:o[0]] == 7).all() and (out[o[-1]:] == 7).all() and (out[:, d_in:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", LINEAR_CASES)
def test_grouped_linear_dw(ctx, dtype, sizes, d_in, d_out):
    o, off, n, (host, x, _), (dhost, dy, _), _, _ = linear_inputs(sizes, d_in, d_out, dtype, d_in + 9)
    want_w, want_b = ref.linear_dw(host, dhost, o)
    size_w, size_b = ref.linear_dw(host.abs(), dhost.abs(), o)
    dw, db = ctx.grouped_linear_dw(x, dy, off)
    steps = (max(sizes) + 16) * 2 * U
    assert_close(dw, want_w, steps * size_w, "dW")
    assert_close(db, want_b, steps * size_b, "db")
    sw, sb = ctx.grouped_linear_dw(x, dy, off, shared=True)
    steps = (sum(sizes) + 16) * 2 * U
    assert_close(sw, want_w.sum(0), steps * size_w.sum(0), "dW of all parts")
    assert_close(sb, want_b.sum(0), steps * size_b.sum(0), "db of all parts")
    alone, none = ctx.grouped_linear_dw(x, dy, off, bias=False)
    assert none is None and torch.equal(alone, dw)


def test_grouped_linear_shared_matrix_and_replicas(ctx):
    """One matrix for all parts, and matrices and gradients where they lie in params [M, P]."""
    M, d_in, d_out = 5, 60, 36
    o, off = offsets_of([100, 0, 37, 129, 4])
    x, dy = (torch.randn(o[-1], d, generator=gen(d)).cuda() for d in (d_in, d_out))
    W, b = torch.randn(d_in, d_out, generator=gen(1)).cuda(), torch.randn(d_out, generator=gen(2)).cuda()
    each = W.expand(M, d_in, d_out).contiguous(), b.expand(M, d_out).contiguous()
    assert torch.equal(ctx.grouped_linear(x, off, W, b), ctx.grouped_linear(x, off, *each))
    assert torch.equal(ctx.grouped_linear_dx(dy, off, W), ctx.grouped_linear_dx(dy, off, each[0]))
    P = 3 + d_in * d_out + d_out + 2
    params, grads = torch.full((M, P), float("nan"), device="cuda"), torch.full((M, P), 9.0, device="cuda")
    w_of = lambda t: t[:, 3:3 + d_in * d_out].view(M, d_in, d_out)  # noqa: E731
    b_of = lambda t: t[:, 3 + d_in * d_out:3 + d_in * d_out + d_out]  # noqa: E731
    w_of(params).copy_(torch.randn(M, d_in, d_out, generator=gen(7)))
    b_of(params).copy_(torch.randn(M, d_out, generator=gen(8)))
    assert torch.equal(ctx.grouped_linear(x, off, w_of(params), b_of(params)),
                       ctx.grouped_linear(x, off, w_of(params).contiguous(), b_of(params).contiguous()))
    dw, db = ctx.grouped_linear_dw(x, dy, off)
    ctx.grouped_linear_dw(x, dy, off, dw=w_of(grads), db=b_of(grads))
    assert torch.equal(w_of(grads), dw) and torch.equal(b_of(grads), db)
    assert (grads[:, :3] == 9).all() and (grads[:, -2:] == 9).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_grouped_linear_of_values_that_are_not_finite(ctx, dtype, bad):
    """They reach their own row, and the gradient of their own part and column, and nothing else."""
    o, off = offsets_of([40, 30])
    x, dy = (torch.randn(70, d, generator=gen(d)).to(dtype).cuda() for d in (50, 20))
    W = torch.randn(2, 50, 20, generator=gen(3)).to(dtype).cuda()
    clean, clean_dx = ctx.grouped_linear(x, off, W), ctx.grouped_linear_dx(dy, off, W)
    clean_dw, clean_db = ctx.grouped_linear_dw(x, dy, off)
    x[40, 3] = bad
    dy[40, 4] = bad
    y, dx = ctx.grouped_linear(x, off, W), ctx.grouped_linear_dx(dy, off, W)
    others = torch.arange(70, device="cuda") != 40
    assert torch.equal(y[others], clean[others]) and not y[40].isfinite().any()
    assert torch.equal(dx[others], clean_dx[others]) and not dx[40].isfinite().any()
    dw, db = ctx.grouped_linear_dw(x, dy, off)
    assert torch.equal(dw[0], clean_dw[0]) and torch.equal(db[0], clean_db[0])
    hit = torch.zeros(50, 20, dtype=torch.bool, device="cuda")
    hit[3], hit[:, 4] = True, True
    assert torch.equal(dw[1][~hit], clean_dw[1][~hit]) and not dw[1][hit].isfinite().any()
    assert not db[1][4].isfinite() and torch.equal(db[1][torch.arange(20) != 4], clean_db[1][torch.arange(20) != 4])


@pytest.mark.parametrize("K", [256, 1024])
def test_products_of_fp32_rows_are_fp32_products(ctx, K):
    """Values of one sign, so that a systematic rounding shows in the mean error.  Sums rounded to nearest have none; a kernel whose
    sums are truncated has half a step of the running sum per addition, K / 2 of them half steps of the result on average: 8 half
    steps allow 16 such additions.  Any single sum of K terms, each addition off by at most a step, is within K steps."""
    n, N = 512, 192
    x = torch.rand(n, K, generator=gen(1)) + 0.5
    W = torch.rand(K, N, generator=gen(2)) + 0.5
    want = x.to(F64) @ W.to(F64)
    off = (ctx.grouped_linear(x.cuda(), None, W.cuda()).cpu().to(F64) - want) / want
    assert off.mean().abs() < 8 * U and off.abs().max() < (K + 16) * 2 * U
    y = torch.rand(n, N, generator=gen(3)) + 0.5
    want = x.to(F64).T @ y.to(F64)
    off = (ctx.grouped_linear_dw(x.cuda(), y.cuda(), None)[0][0].cpu().to(F64) - want) / want
    assert off.mean().abs() < 8 * U and off.abs().max() < (n + 16) * 2 * U


# Enough rows that every block works on several tiles and chunks, and that unaligned 16-bit matrices are laid out first.
# d_in, d_out, elements between the rows of X and of dY: rows on 16-byte boundaries with a width that does not end on one, off them, ...
MANY_CASES = [(256, 47, 0, 0), (47, 90, 0, 6), (100, 256, 4, 0), (101, 256, 3, 8), (512, 512, 0, 0), (33, 300, 0, 4), (130, 62, 6, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_in,d_out,pad,pad_out", MANY_CASES)
def test_grouped_products_of_many_rows(ctx, dtype, d_in, d_out, pad, pad_out):
    sizes = [21_000, 0, 17, 33_333, 128, 6_000]
    o, off = offsets_of(sizes, 3)
    n, G = o[-1] + 5, len(sizes)
    host, x, _ = make_rows(n, d_in, dtype, 1, pad)
    dhost, dy, _ = make_rows(n, d_out, dtype, 2, pad_out)
    W = (torch.randn(G, d_in, d_out, generator=gen(3)) / math.sqrt(d_in)).to(dtype).cuda()
    b = torch.randn(G, d_out, generator=gen(4)).to(dtype).cuda()
    X, D, W64, b64 = host.cuda().to(F64), dhost.cuda().to(F64), W.to(F64), b.to(F64)
    y = torch.full((n, d_out), 7.0, dtype=dtype, device="cuda")
    dx = torch.full((n, d_in), 7.0, dtype=dtype, device="cuda")
    ctx.grouped_linear(x, off, W, b, out=y)
    ctx.grouped_linear_dx(dy, off, W, out=dx)
    dw, db = ctx.grouped_linear_dw(x, dy, off)
    for t in (y, dx):
        assert (t[:o[0]] == 7).all() and (t[o[-1]:] == 7).all()

    def close(got, want, size, steps, what, rounded):
        tol = steps * 2 * U * size + (rounding(want, dtype) if rounded else 0)
        worst = ((got.to(F64) - want).abs() / tol.clamp_min(1e-300)).max() if got.numel() else torch.zeros(())
        assert worst <= 1, f"{what}: {worst.item():.3g} tolerances"

    for g, (lo, hi) in enumerate(zip(o, o[1:])):
        xs, ds = X[lo:hi], D[lo:hi]
        close(y[lo:hi], xs @ W64[g] + b64[g], xs.abs() @ W64[g].abs() + b64[g].abs(), d_in + 16, f"y {g}", True)
        close(dx[lo:hi], ds @ W64[g].T, ds.abs() @ W64[g].T.abs(), d_out + 16, f"dx {g}", True)
        close(dw[g], xs.T @ ds, xs.T.abs() @ ds.abs(), hi - lo + 16, f"dW {g}", False)
        close(db[g], ds.sum(0), ds.abs().sum(0), hi - lo + 16, f"db {g}", False)
    ctx.check()


def test_a_captured_product_keeps_its_laid_out_matrices():
    """A matrix that is laid out first lies in the scratch: a capture without it is refused, a replay follows the matrix."""
    ctx = binding.Context(0)
    x = torch.randn(40_000, 64, generator=gen(1)).half().cuda()
    W = torch.randn(64, 47, generator=gen(2)).half().cuda()
    with pytest.raises(binding.RtmaError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            ctx.grouped_linear(x, None, W)
    ctx.grouped_linear(x, None, W)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ctx.grouped_linear(x, None, W)
    W.mul_(2)
    ctx.grouped_linear_dw(x, x, None)  # other contents, and more of them
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, ctx.grouped_linear(x, None, W))
    ctx.check()


@pytest.mark.parametrize("direction", ["y", "dx"])
def test_deep_products_in_a_graph_and_on_two_streams(direction):
    """Deep contractions of 16-bit rows run on pairs of blocks; the same bits in a graph, and beside another context's."""
    one, two = binding.Context(0), binding.Context(0)
    o, off = offsets_of([12_000, 0, 300, 17_701])
    x = torch.randn(o[-1], 512, generator=gen(1)).bfloat16().cuda()
    W = (torch.randn(4, 512, 512, generator=gen(2)) / 20).bfloat16().cuda()
    b = torch.randn(4, 512, generator=gen(3)).bfloat16().cuda()
    call = (lambda c, **k: c.grouped_linear(x, off, W, b, **k)) if direction == "y" else (lambda c, **k: c.grouped_linear_dx(x, off, W, **k))
    want = call(one).clone()
    x32, W32 = x.float(), W.float()
    want32 = two.grouped_linear(x32, off, W32).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(one)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    outs, outs32 = [torch.empty_like(want) for _ in range(6)], [torch.empty_like(want32) for _ in range(6)]
    torch.cuda.synchronize()
    for a, c in zip(outs, outs32):
        call(one, out=a, stream=streams[0])
        two.grouped_linear(x32, off, W32, out=c, stream=streams[1])
        call(two, out=a, stream=streams[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, want) for a in outs) and all(torch.equal(c, want32) for c in outs32)
    one.check()
    two.check()


def test_more_than_two_to_the_31_elements(ctx):
    """The rows of the last part lie behind 2^31 elements and give what they give alone."""
    d, few = 512, 700
    n = 2 ** 31 // d + 300 + few
    last = torch.randn(few, d, generator=gen(1)).half().cuda()
    x = torch.zeros(n, d, dtype=torch.float16, device="cuda")
    x[-few:] = last
    off = torch.tensor([0, n - few, n], dtype=torch.int64, device="cuda")
    W = torch.randn(2, d, 24, generator=gen(2)).half().cuda()
    y = ctx.grouped_linear(x, off, W)
    assert torch.equal(y[-few:], ctx.grouped_linear(last, None, W[1])) and not y[:-few].any()
    ones = torch.ones_like(y)
    dw, _ = ctx.grouped_linear_dw(x, ones, off)
    alone, _ = ctx.grouped_linear_dw(last, ones[-few:], None)
    assert not dw[0].any() and (dw[1] - alone[0]).abs().max() <= (few + 16) * 2 * U * last.abs().float().sum(0).max()
    out = ctx.grouped_linear_dx(y, off, W)
    assert torch.equal(out[-few:], ctx.grouped_linear_dx(y[-few:].contiguous(), None, W[1])) and not out[:-few].any()
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")  # one id many times: one mask
    ids[-few:] = torch.arange(few, dtype=torch.int32, device="cuda")
    ctx.dropout(x, 0.5, 9, row_ids=ids, out=out)
    assert torch.equal(out[-few:], ctx.dropout(last, 0.5, 9)) and not out[:-few].any()
    ctx.group_norm(x, off, 4, act="silu", out=out)
    assert torch.equal(out[-few:], ctx.group_norm(last, None, 4, act="silu")[0]) and not out[:-few].any()
    ctx.group_norm(x, off, 4, scope="part", out=out)
    want = ctx.group_norm(last, None, 4, scope="part")[0]
    assert (out[-few:].float() - want.float()).abs().max() <= 2 * half_step(torch.float16) * want.abs().max() and not out[:-few].any()
    ctx.check()


# ---- all of them ----------------------------------------------------------------------------------------


def operators(ctx, dtype=torch.float32, n=700, stream=None):
    """Name -> a call of every operator on inputs of its own."""
    o, off = offsets_of([n // 2, 0, n - n // 2])
    x, dy = (torch.randn(n, d, generator=gen(d)).to(dtype).cuda() for d in (72, 40))
    W, b = (torch.randn(3, *s, generator=gen(1)).to(dtype).cuda() for s in ((72, 40), (40,)))
    gamma, beta = torch.randn(72, generator=gen(2)).cuda(), torch.randn(3, 72, generator=gen(3)).cuda()
    how = dict(act="silu", p=0.25, seed=1)
    kept = {s: ctx.group_norm(x, off, 8, gamma, beta, scope=s, **how)[1] for s in ("row", "part")}
    torch.cuda.synchronize()
    calls = {
        "dropout": lambda **k: ctx.dropout(x, 0.5, 3, residual=x, **k),
        "linear": lambda **k: ctx.grouped_linear(x, off, W, b, **k),
        "dx": lambda **k: ctx.grouped_linear_dx(dy, off, W, **k),
        "dw": lambda **k: ctx.grouped_linear_dw(x, dy, off, **k),
    }
    for s in ("row", "part"):
        calls["norm " + s] = lambda s=s, **k: ctx.group_norm(x, off, 8, gamma, beta, scope=s, **how, **k)
        calls["norm grad " + s] = lambda s=s, **k: ctx.group_norm_grad(x, x, kept[s], off, 8, gamma, beta, scope=s, **how, **k)
    return calls


def tensors(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


NAMES = ["dropout", "linear", "dx", "dw", "norm row", "norm grad row", "norm part", "norm grad part"]


@pytest.mark.parametrize("name", NAMES)
def test_same_bits_every_time_on_any_stream_and_in_a_graph(name):
    ctx = binding.Context(0)
    call = operators(ctx, n=3000)[name]
    want = [t.clone() for t in tensors(call())]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t, w in zip(tensors(call()), want):
            side.synchronize()
            assert torch.equal(t, w)
    for t, w in zip(tensors(call(stream=side)), want):
        side.synchronize()
        assert torch.equal(t, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = tensors(call())
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(out, want))
    # the scratch grows behind the graph's back: the graph keeps its own
    before = ctx.workspace_bytes
    big = operators(ctx, n=400_000)["norm grad part"]
    big()
    ctx.grouped_linear_dw(torch.ones(50_000, 300, device="cuda"), torch.ones(50_000, 300, device="cuda"), None)
    torch.cuda.synchronize()
    assert ctx.workspace_bytes > before
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(out, want))
    ctx.check()


def test_a_capture_does_not_grow_the_scratch():
    ctx = binding.Context(0)
    x = torch.randn(2000, 64, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(binding.RtmaError, match="before the capture"):
        with torch.cuda.graph(graph):
            ctx.group_norm(x, None, 4, scope="part")
    y, _ = ctx.group_norm(x, None, 4, scope="part")  # the context works on
    assert y.isfinite().all()


@pytest.mark.parametrize("name", NAMES)
def test_no_rows(ctx, name):
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    x, dy = torch.empty(0, 16, device="cuda"), torch.empty(0, 8, device="cuda")
    W = torch.ones(2, 16, 8, device="cuda")
    one = torch.ones(2, 16, device="cuda")
    if name == "dropout":
        assert ctx.dropout(x, 0.5, 1).shape == (0, 16)
    elif name == "linear":
        assert ctx.grouped_linear(x, off, W).shape == (0, 8)
    elif name == "dx":
        assert ctx.grouped_linear_dx(dy, off, W).shape == (0, 16)
    elif name == "dw":
        dw, db = ctx.grouped_linear_dw(x, dy, off)
        assert not dw.any() and not db.any()
    else:
        scope = name.split()[-1]
        y, st = ctx.group_norm(x, off, 4, one, one, scope=scope)
        assert y.shape == (0, 16)
        if scope == "part":
            assert torch.allclose(st, torch.tensor([0.0, 1e-5 ** -0.5], device="cuda").expand(2, 4, 2))
        if "grad" in name:
            dx, dg, db, _ = ctx.group_norm_grad(x, x, st, off, 4, one, one, scope=scope)
            assert dx.shape == (0, 16) and not dg.any() and not db.any()


@pytest.mark.parametrize("name", NAMES)
def test_offsets_that_are_none_reach_no_other_memory(name):
    """Beyond the rows, backwards, overlapping, negative: every access stays within the rows (here: within guard rows)."""
    n, d_in, d_out = 300, 24, 16
    for checked in (False, True):
        ctx = binding.Context(0, checked=checked)
        for values in ([0, n + 500, n + 900], [200, 100, 300], [0, 300, 0, 300, 0, 300], [-50, 10, 2**40], [2**62, -2**62, 5]):
            off = torch.tensor(values, dtype=torch.int64, device="cuda")
            G = len(values) - 1
            outer = [torch.full((n + 600, d), 7.0, device="cuda") for d in (d_in, d_out, d_in)]
            x, y, dx = (t[300:300 + n] for t in outer)
            W = torch.ones(G, d_in, d_out, device="cuda")
            one = torch.ones(G, d_in, device="cuda")
            if name == "dropout":
                return
            if name == "linear":
                ctx.grouped_linear(x, off, W, out=y)
            elif name == "dx":
                ctx.grouped_linear_dx(y, off, W, out=dx)
            elif name == "dw":
                ctx.grouped_linear_dw(x, y, off)
            else:
                scope = name.split()[-1]
                st = torch.ones(n if scope == "row" else G, 4, 2, device="cuda")
                if "grad" in name:
                    ctx.group_norm_grad(x, x, st, off, 4, one, one, scope=scope, out=dx)
                else:
                    ctx.group_norm(x, off, 4, one, one, scope=scope, out=dx, stats=st)
            torch.cuda.synchronize()
            for t in outer:
                assert (t[:300] == 7).all() and (t[300 + n:] == 7).all()
            if checked:
                with pytest.raises(binding.RtmaError, match="part offset"):
                    ctx.check()
            else:
                ctx.check()


def test_refusals(ctx):
    x, y = torch.ones(10, 16, device="cuda"), torch.ones(10, 8, device="cuda")
    off = torch.tensor([0, 4, 10], dtype=torch.int64, device="cuda")
    W = torch.ones(2, 16, 8, device="cuda")
    g = torch.ones(2, 16, device="cuda")
    many = torch.zeros(binding.MAX_GROUPS + 2, dtype=torch.int64, device="cuda")
    refused = [
        (TypeError, lambda: ctx.dropout(x.double(), 0.5, 1)),
        (ValueError, lambda: ctx.dropout(x.cpu(), 0.5, 1)),
        (ValueError, lambda: ctx.dropout(x[0], 0.5, 1)),
        (ValueError, lambda: ctx.dropout(x.t(), 0.5, 1)),
        (ValueError, lambda: ctx.dropout(x, 0.5, 1, residual=y)),
        (TypeError, lambda: ctx.dropout(x, 0.5, 1, residual=x.half())),
        (TypeError, lambda: ctx.dropout(x, 0.5, 1, row_ids=torch.arange(10, device="cuda"))),
        (ValueError, lambda: ctx.dropout(x, 0.5, 1, row_ids=torch.arange(9, device="cuda", dtype=torch.int32))),
        (ValueError, lambda: ctx.dropout(x, 0.5, 1, out=torch.ones(16, device="cuda").expand(10, 16))),
        (binding.RtmaError, lambda: ctx.dropout(x, -0.1, 1)),
        (binding.RtmaError, lambda: ctx.dropout(x, 1.5, 1)),
        (binding.RtmaError, lambda: ctx.dropout(x, float("nan"), 1)),
        (TypeError, lambda: ctx.grouped_linear(x, off.int(), W)),
        (ValueError, lambda: ctx.grouped_linear(x, off.cpu(), W)),
        (ValueError, lambda: ctx.grouped_linear(x, off[:1], W)),
        (ValueError, lambda: ctx.grouped_linear(x, off, torch.ones(3, 16, 8, device="cuda"))),
        (ValueError, lambda: ctx.grouped_linear(x, off, torch.ones(2, 8, 16, device="cuda").mT)),
        (TypeError, lambda: ctx.grouped_linear(x, off, W.half())),
        (ValueError, lambda: ctx.grouped_linear(x, off, W, torch.ones(2, 9, device="cuda"))),
        (ValueError, lambda: ctx.grouped_linear(x, off, W, out=x)),
        (binding.RtmaError, lambda: ctx.grouped_linear(x, many, W[0])),
        (binding.RtmaError, lambda: ctx.grouped_linear(torch.ones(1, 16385, device="cuda"), None, torch.ones(16385, 1, device="cuda"))),
        (binding.RtmaError, lambda: ctx.grouped_linear(x, off, torch.ones(2, 16, 16, device="cuda"), out=x)),
        (ValueError, lambda: ctx.grouped_linear_dx(x, off, W)),
        (ValueError, lambda: ctx.grouped_linear_dw(x, y[:9], off)),
        (TypeError, lambda: ctx.grouped_linear_dw(x, y.half(), off)),
        (TypeError, lambda: ctx.grouped_linear_dw(x, y, off, dw=W.half())),
        (ValueError, lambda: ctx.grouped_linear_dw(x, y, off, shared=True, dw=W)),
        (binding.RtmaError, lambda: ctx.grouped_linear_dw(x, y, off, dw=torch.ones(16, 8, device="cuda").expand(2, 16, 8))),
        (ValueError, lambda: ctx.group_norm(x, off, 4, g, scope="batch")),
        (ValueError, lambda: ctx.group_norm(x, off, 4, g, act="tanh")),
        (ValueError, lambda: ctx.group_norm(x, off, 4, g[:, :8])),
        (TypeError, lambda: ctx.group_norm(x, off, 4, g.half())),
        (binding.RtmaError, lambda: ctx.group_norm(x, off, 5, g)),
        (binding.RtmaError, lambda: ctx.group_norm(x, off, 4, g, act="prelu")),
        (binding.RtmaError, lambda: ctx.group_norm(x, off, 4, g, eps=0.0)),
        (binding.RtmaError, lambda: ctx.group_norm(x, off, 4, g, p=2.0)),
        (ValueError, lambda: ctx.group_norm(x, off, 4, g, act="prelu", slope=torch.ones(3, device="cuda"))),
        (binding.RtmaError, lambda: ctx.group_norm(torch.ones(2, 2049, device="cuda"), None, 1)),
        (ValueError, lambda: ctx.group_norm_grad(x, x, torch.ones(10, 2, 2, device="cuda"), off, 4, g)),
        (binding.RtmaError, lambda: ctx.group_norm_grad(x, x, torch.ones(10, 4, 2, device="cuda"), off, 4, g, dslope=torch.ones(2, device="cuda"))),
        (binding.RtmaError, lambda: ctx.group_norm_grad(x, x, torch.ones(10, 4, 2, device="cuda"), off, 4, g, dgamma=torch.ones(20, device="cuda").as_strided((2, 16), (4, 1)))),
    ]
    for i, (error, call) in enumerate(refused):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    assert ctx.dropout(x, 0.0, 1).equal(x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scope", ["row", "part"])
def test_two_layers_of_replicas_forward_and_backward(ctx, dtype, scope):
    """Product, norm with PReLU and dropout by node id, product, over the parts of a partition, and back; against autograd in 64 bits."""
    n, M, d, h, c = 1_500, 4, 36, 64, 10
    _, off, perm, _ = ctx.partition(n, None, 7, M)
    o = off.cpu().tolist()
    r = lambda *s, seed: torch.randn(*s, generator=gen(seed))  # noqa: E731
    x = r(n, d, seed=1).to(dtype)
    W1, W2 = (r(M, d, h, seed=2) / d ** 0.5).to(dtype), (r(M, h, c, seed=3) / h ** 0.5).to(dtype)
    b1, b2 = r(M, h, seed=4).to(dtype), r(M, c, seed=5).to(dtype)
    gamma, beta, slope = 1 + 0.2 * r(M, h, seed=6), 0.2 * r(M, h, seed=7), torch.full((M,), 0.25)
    dout = r(n, c, seed=8).to(dtype)
    kept, scale = ref.mask(3, perm.cpu().numpy(), h, 0.5)
    leaves = [t.to(F64).requires_grad_() for t in (x, W1, b1, gamma, beta, slope, W2, b2)]
    z = ref.linear(leaves[0], o, leaves[1], leaves[2])
    a, _, _, _ = ref.group_norm(z, o, 4, leaves[3], leaves[4], scope, "prelu", leaves[5], 1e-5, kept, scale)
    want = ref.linear(a, o, leaves[6], leaves[7])
    want.backward(dout.to(F64))
    cu = lambda t: t.cuda()  # noqa: E731
    how = dict(scope=scope, act="prelu", slope=cu(slope), p=0.5, seed=3, row_ids=perm)
    Z = ctx.grouped_linear(cu(x), off, cu(W1), cu(b1))
    A, st = ctx.group_norm(Z, off, 4, cu(gamma), cu(beta), **how)
    Y = ctx.grouped_linear(A, off, cu(W2), cu(b2))
    dA = ctx.grouped_linear_dx(cu(dout), off, cu(W2))
    dW2, db2 = ctx.grouped_linear_dw(A, cu(dout), off)
    dZ, dg, db, ds = ctx.group_norm_grad(Z, dA, st, off, 4, cu(gamma), cu(beta), **how)
    dX = ctx.grouped_linear_dx(dZ, off, cu(W1))
    dW1, db1 = ctx.grouped_linear_dw(cu(x), dZ, off)
    # Every stage rounds its rows once; errors of the stages before are passed on by maps of norm about one (products of random
    # matrices, normalisation, dropout's factor of two): eight roundings of half a step, with a factor of 4 for those maps.  A value
    # of u within rounding of zero takes the other slope: a share of about half_step of the values, each off by 0.75.
    h2 = half_step(dtype)
    tol = 8 * 4 * h2 + 0.75 * 2 * math.sqrt(4 * h2) if dtype != torch.float32 else 8 * 4 * h2 + 1e-3
    got = dict(Y=Y, dX=dX, dW1=dW1, db1=db1, dg=dg, db=db, ds=ds, dW2=dW2, db2=db2)
    exact = dict(Y=want, dX=leaves[0].grad, dW1=leaves[1].grad, db1=leaves[2].grad, dg=leaves[3].grad, db=leaves[4].grad, ds=leaves[5].grad,
                 dW2=leaves[6].grad, db2=leaves[7].grad)
    for k in got:
        e, g = exact[k].detach(), got[k].cpu().to(F64)
        # normalised columns that add up to zero over a part leave a gradient of the first bias that is a difference of large numbers
        size = e.norm() if k != "db1" else max(e.norm(), dZ.double().norm().cpu())
        assert (g - e).norm() <= tol * size, (k, ((g - e).norm() / size).item(), tol)


def test_two_contexts_side_by_side():
    """Two calls at once on two streams, each on its own context's scratch."""
    a, b = binding.Context(0), binding.Context(0)
    calls = [operators(c, n=60_000) for c in (a, b)]
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = {k: [t.clone() for t in tensors(f())] for k, f in calls[0].items()}
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for k in want:
            for c, st in zip(calls, s):
                with torch.cuda.stream(st):
                    got.append((k, tensors(c[k]())))
        torch.cuda.synchronize()
        for k, ts in got:
            assert all(torch.equal(t, w) for t, w in zip(ts, want[k])), k
