"""The operators on the rows of many parts where their arguments are at an end: the most rows, expanded and overlapping tensors,
runs of rows of every length, values whose squares do not fit.  Tolerances as in test_gpu_row_operators.py."""
import numpy as np
import pytest
import torch

import row_reference as ref
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


@pytest.mark.parametrize("dtype,d_out,stride", [(torch.float32, 300, 112), (torch.float32, 300, 224), (torch.bfloat16, 600, 416), (torch.float16, 600, 208)])
def test_parameters_of_parts_that_overlap(ctx, dtype, d_out, stride):
    """Parameters are only read, so those of two parts may share memory (strides smaller than a part's): columns of one part's bias that
    another part has at the same address are still that part's, and as many as it has."""
    G, d_in = 9, 16
    g = torch.Generator().manual_seed(d_out + stride)
    sizes = torch.randint(3_000, 14_000, (G,), generator=g)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), sizes.cumsum(0)]).cuda()
    x = torch.randn(int(off[-1]), d_in, generator=g).to(dtype).cuda()
    flat = torch.randn(G * max(stride, 5) + d_in * d_out, generator=g).to(dtype).cuda()
    bias = flat.as_strided((G, d_out), (stride, 1))
    W = flat.as_strided((G, d_in, d_out), (5, d_out, 1))
    assert torch.equal(ctx.grouped_linear(x, off, W, bias), ctx.grouped_linear(x, off, W.contiguous(), bias.contiguous()))
    dy = torch.randn(len(x), d_out, generator=g).to(dtype).cuda()
    assert torch.equal(ctx.grouped_linear_dx(dy, off, W), ctx.grouped_linear_dx(dy, off, W.contiguous()))


NORM_KINDS = [(64, 8), (64, 32), (60, 20), (100, 4), (384, 1), (300, 3), (1024, 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("C,groups", NORM_KINDS)
def test_norm_of_equal_values_far_from_zero(ctx, dtype, C, groups):
    """x - mean is 0 whatever 1 / std is: y is beta, and gamma's gradient 0 however many rows there are."""
    n = 5_000
    x = torch.full((n, C), 1000.0, dtype=dtype, device="cuda")
    g = torch.Generator().manual_seed(C)
    gamma, beta = torch.randn(C, generator=g).cuda(), torch.randn(C, generator=g).cuda()
    dy = torch.ones_like(x)
    y, st = ctx.group_norm(x, None, groups, gamma, beta, scope="part")
    assert torch.equal(y, beta.to(dtype).expand(n, C)) and (st[..., 0] == 1000).all()
    for scope, rows in (("part", 1), ("row", n)):
        stats = st.expand(rows, groups, 2).contiguous()
        _, dg, db, _ = ctx.group_norm_grad(x, dy, stats, None, groups, gamma, beta, scope=scope)
        assert not dg.any() and (db == n).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("C,groups", NORM_KINDS)
def test_norm_of_values_whose_squares_do_not_fit(ctx, dtype, scope, C, groups):
    """1 / std is 0 then, so that y is beta, and no gradient comes through; other rows (parts) are not touched."""
    g = torch.Generator().manual_seed(C)
    n, half = 120, 60
    x = torch.randn(n, C, generator=g).to(dtype).cuda()
    gamma, beta = torch.randn(2, C, generator=g).cuda(), torch.randn(2, C, generator=g).cuda()
    dy = torch.randn(n, C, generator=g).to(dtype).cuda()
    off = torch.tensor([0, half, n], dtype=torch.int64, device="cuda")
    clean, _ = ctx.group_norm(x, off, groups, gamma, beta, scope=scope)
    x[half:] = (x[half:].float() * 1e25).to(dtype)
    y, st = ctx.group_norm(x, off, groups, gamma, beta, scope=scope)
    assert torch.equal(y[:half], clean[:half])
    assert torch.equal(y[half:], beta[1].to(dtype).expand(n - half, C))
    huge = st[half:] if scope == "row" else st[1:]
    # (two rounded values of a row's set may be equal: such a set has no squares to speak of)
    sets = x[half:].view(half, groups, C // groups) if scope == "row" else x[half:].view(half, groups, C // groups).transpose(0, 1).reshape(1, groups, -1)
    equal = sets.amax(2) == sets.amin(2)
    assert (huge[..., 1] == 0)[~equal].all() and (huge[..., 0].abs() < 1e26).all()
    dx, dg, db, _ = ctx.group_norm_grad(x, dy, st, off, groups, gamma, beta, scope=scope)
    assert not dx[half:].view(half, groups, -1)[~equal.expand(half, groups)].any() and not dg[1].any() and dx.isfinite().all()
    want = dy[half:].to(F64).sum(0)
    assert ((db[1].to(F64) - want).abs() <= n * 2 * U * dy[half:].to(F64).abs().sum(0)).all()


@pytest.mark.parametrize("scope", ["row", "part"])
@pytest.mark.parametrize("C,groups", NORM_KINDS)
@pytest.mark.parametrize("eps", [1e-42, 1e-30])
def test_norm_of_equal_values_with_a_tiny_eps(ctx, scope, C, groups, eps):
    """1 / sqrt(eps), of an eps below the smallest normal number too: three roundings, and that of eps itself."""
    x = torch.full((40, C), 2.0, device="cuda")
    y, st = ctx.group_norm(x, None, groups, scope=scope, eps=eps)
    want = torch.tensor(eps).to(F64).item() ** -0.5
    assert not y.any() and (st[..., 0] == 2).all()
    assert ((st[..., 1].to(F64) / want - 1).abs() <= 4 * 2 * U).all()


def test_a_result_is_not_in_memory_that_another_stream_still_writes(ctx):
    """A tensor is freed while its stream has yet to write it; a call on another stream, which runs first, keeps out of its memory."""
    n, d = 4096, 1024
    x = torch.randn(n, d, device="cuda")
    want = ctx.dropout(x, 0.5, 3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        freed = torch.empty(n, d, device="cuda")
        torch.cuda._sleep(100_000_000)
        freed.fill_(7)
        del freed
        y = ctx.dropout(x, 0.5, 3, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("direction", ["y", "dx"])
def test_deep_products_beside_another_contexts(direction):
    """Products on pairs of blocks while another context's run on another stream: every one its own result, all of them right."""
    one, two = binding.Context(0), binding.Context(0)
    g = torch.Generator().manual_seed(4)
    off = torch.tensor([0, 12_000, 12_000, 12_300, 30_001], device="cuda")
    x = torch.randn(30_001, 512, generator=g).bfloat16().cuda()
    W = (torch.randn(4, 512, 512, generator=g) / 20).bfloat16().cuda()
    call = (lambda c, **k: c.grouped_linear(x, off, W, **k)) if direction == "y" else (lambda c, **k: c.grouped_linear_dx(x, off, W, **k))
    want = call(one).clone()
    W64 = W.double() if direction == "y" else W.double().mT
    for k in range(4):
        r = slice(int(off[k]), int(off[k + 1]))
        exact, size = x[r].double() @ W64[k], x[r].double().abs() @ W64[k].abs()
        assert ((want[r].double() - exact).abs() <= 2.0 ** -8 * 1.001 * exact.abs() + (512 + 16) * 2 * U * size).all()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [[torch.zeros_like(want) for _ in range(6)] for _ in streams]
    torch.cuda.synchronize()
    for k in range(6):
        for c, s, o in zip((one, two), streams, outs):
            call(c, out=o[k], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for side in outs for o in side)
    one.check()
    two.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sign", [False, True])
def test_the_longest_contractions(ctx, dtype, sign):
    """16,384 terms.  Sums of 16-bit rows stay in the accumulator, truncated every 16 terms (a step, 2^-23 of the sum so far at most, towards zero):
    with terms of one sign that is a drift of up to 1024 steps, a quarter of a rounding to fp16."""
    K, N, n = 16384, 40, 300
    g = torch.Generator().manual_seed(5)
    draw = (lambda *s: torch.randn(*s, generator=g)) if sign else (lambda *s: torch.rand(*s, generator=g) + 0.5)
    x, W = draw(n, K).to(dtype).cuda(), (draw(K, N) / 128).to(dtype).cuda()
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for got, a, b in ((ctx.grouped_linear(x, None, W), x, W), (ctx.grouped_linear_dx(x, None, W.mT.contiguous()), x, W)):
        exact, size = a.double() @ b.double(), a.double().abs() @ b.double().abs()
        # sums within 16 terms are exact or truncated as well: 2 steps for each of the K / 16 additions
        tol = torch.finfo(dtype).eps / 2 * 1.001 * exact.abs() + tiny + (2 * K / 16 + 16) * 2 * U * size
        assert ((got.double() - exact).abs() <= tol).all()


@pytest.mark.parametrize("d", [2 ** 31 - 1, 2 ** 31 - 9])
def test_dropout_of_the_widest_row(ctx, d):
    """One row of as many columns as an int32 counts: the mask of its last columns, and nothing behind them."""
    def step(z):
        z = z + np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    x = torch.ones(1, d + 9, dtype=torch.float16, device="cuda")[:, :d]
    y = torch.full((1, d + 9), 7.0, dtype=torch.float16, device="cuda")
    ctx.dropout(x, 0.5, 11, out=y[:, :d])
    assert (y[:, d:] == 7).all()
    last = 4096
    first = (d - last) // 4 * 4
    with np.errstate(over="ignore"):
        key = step(np.array([11], dtype=np.uint64))[0]
        col = np.arange(first, d, dtype=np.uint64)
        lane = (step(key ^ (col // np.uint64(4))) >> (np.uint64(16) * (col % np.uint64(4)))) & np.uint64(0xFFFF)
    assert torch.equal(y[0, first:d].cpu(), torch.from_numpy(lane >= 32768).half() * 2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("deviations", [0.0, 60.0, 63.9, 64.1, 70.0, 500.0])
def test_norm_of_a_part_with_means_on_both_sides_of_the_folding(ctx, dtype, deviations):
    """The mean folded into the shift, 2^-24 of up to 64 deviations off, or subtracted: both within a few roundings of the result, and mixed within a row."""
    n, C, groups = 30_000, 64, 8
    g = torch.Generator().manual_seed(6)
    x = torch.randn(n, C, generator=g)
    x[:, :24] += deviations  # three of the eight sets
    x = x.to(dtype).cuda()
    gamma, beta = torch.randn(C, generator=g).cuda(), torch.randn(C, generator=g).cuda()
    y, st = ctx.group_norm(x, None, groups, gamma, beta, scope="part")
    want, stats, u, xhat = ref.group_norm(x.to(F64), [0, n], groups, gamma.to(F64)[None], beta.to(F64)[None], "part", "none", None, 1e-5)
    # statistics: sums at most 8 (channels) + 16 + 240 steps deep, three roundings each; the folding: 64 deviations at 2^-24, times gamma
    size, rstd = x.to(F64).abs().view(n, groups, 8).amax(dim=(0, 2)), stats[0, :, 1]
    tol_x = (3 * U * 270 * (size * rstd)).repeat_interleave(8) + 3 * U * 270 * xhat.abs() + 64 * U
    tol = gamma.to(F64).abs() * tol_x + 4 * U * (want.abs() + beta.to(F64).abs()) + torch.finfo(dtype).eps / 2 * 1.001 * want.abs() + 2.0 ** -24
    assert ((y.to(F64) - want).abs() <= tol).all()


@pytest.mark.parametrize("exponent", [-100, -110, -115, -120, -126, -130])
def test_fp32_products_of_tiny_values(ctx, exponent):
    """A factor's three bf16 numbers add up to it to within the smallest of them, 2^-133 (the last is cut off, the second rounded: once each)."""
    g = torch.Generator().manual_seed(9)
    K, n = 64, 300
    small = ((torch.rand(n, K, generator=g) + 0.5).to(F64) * 2.0 ** exponent).float().cuda()
    W = (torch.rand(K, 40, generator=g) + 0.5).cuda()
    ones = torch.ones(n, 40, device="cuda")

    def check(got, a, b, tiny_is_a, steps):
        a, b = a.to(F64), b.to(F64)
        size = a.abs() @ b.abs()
        lost = 2 * 2.0 ** -133 * (torch.ones_like(a) @ b.abs() if tiny_is_a else a.abs() @ torch.ones_like(b))
        assert ((got.to(F64) - a @ b).abs() <= (steps + 16) * 2 * U * size + lost + 2.0 ** -149).all()

    check(ctx.grouped_linear(small, None, W), small, W, True, K)
    check(ctx.grouped_linear_dx(small, None, W.mT.contiguous()), small, W, True, K)
    check(ctx.grouped_linear(ones[:, :K // 2].contiguous(), None, small[:K // 2].contiguous()), ones[:, :K // 2], small[:K // 2], False, K)
    check(ctx.grouped_linear_dw(small, ones, None)[0][0], small.mT, ones, True, n)
