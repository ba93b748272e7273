"""Whole layers and clipping at the ends of their ranges: widest matrices, most parts, rows far apart, long sums, two calls at once, captures."""
import pytest
import torch

from paper_2305_09887_b200 import binding
from test_gpu_layers import TYPES, Case, normal

pytestmark = pytest.mark.gpu
WIDEST = 16384


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


@pytest.mark.parametrize("d_in,d_out,gated", [(WIDEST, 40, False), (40, WIDEST, False), (40, WIDEST // 2, True), (WIDEST - 1, 9, True),
                                              (9, WIDEST // 2 - 1, True)])
@pytest.mark.parametrize("dtype", TYPES)
def test_widest(ctx, dtype, d_in, d_out, gated):
    case = Case(dtype, [150, 3], d_in, d_out, "silu", gated, residual=True, seed=51)
    case.check_forward(ctx)
    case.residual = None
    case.check_gradient(ctx)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_most_parts(ctx, dtype, gated):
    sizes = [(7 * g) % 11 for g in range(binding.MAX_GROUPS)]
    sizes[3], sizes[-1] = 700, 0
    case = Case(dtype, sizes, 24, 10, "prelu", gated, seed=53)
    case.check_forward(ctx)
    case.check_gradient(ctx, grad_dtype=torch.float32)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_far_apart(ctx, dtype, gated, shift):
    """Offsets that pass 32 bits: the same bits as of rows side by side."""
    n, far, d_in, d_out = 40000, 60000, 40, 24
    buffer = torch.empty(n * far + 8, dtype=dtype, device="cuda")
    rows = buffer[shift:shift + n * far].view(n, far)
    X, side, out, dz, dx = rows[:, 64:64 + d_in], rows[:, 128:128 + d_out], rows[:, 200:200 + d_out], buffer[:n * far].view(n, far)[:, 256:256 + 2 * d_out], rows[:, 408:408 + d_in]
    X.copy_(normal(55, n, d_in))
    side.copy_(normal(56, n, d_out))
    if not gated:
        dz = dz[:, :d_out]
    W, b = normal(57, d_in, 2 * d_out if gated else d_out).to(dtype), normal(58, 2 * d_out if gated else d_out).to(dtype)
    forward, back = (ctx.grouped_gated_linear, ctx.grouped_gated_linear_grad) if gated else (ctx.grouped_linear_act, ctx.grouped_linear_act_grad)
    near_X, near_side = X.contiguous(), side.contiguous()
    forward(X, None, W, b, act="silu", residual=side, out=out)
    assert torch.equal(out, forward(near_X, None, W, b, act="silu", residual=near_side))
    got, want = back(X, side, None, W, b, act="silu", out=dx, dz=dz), back(near_X, near_side, None, W, b, act="silu")
    for a, c in zip(got[:3], want[:3]):
        assert torch.equal(a, c)
    ctx.check()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_long_column_sums(ctx, dtype, gated):
    """Sums of twelve million values of one sign.  The tensor cores truncate, by 2^-23 of a sum of 64 tiles of 256 rows at most for every 16 of a warp's 32
    rows; those are added up in fp32 (twelve of them: 2^-24 each), then in 64 bits, and rounded once."""
    n, d = 12_000_000, 8
    dY = 0.5 + torch.rand(n, d, generator=torch.Generator("cuda").manual_seed(59), device="cuda").to(dtype)
    X = torch.zeros(n, d, dtype=dtype, device="cuda")
    X[:, 0] = 1
    W = torch.zeros(d, 2 * d if gated else d, dtype=dtype, device="cuda")
    W[0] = 1
    b = torch.zeros_like(W[0])
    back = ctx.grouped_gated_linear_grad if gated else ctx.grouped_linear_act_grad  # Z is one everywhere: dZ is dY, in both halves
    _, dw, db, _ = back(X, dY, None, W, b, act="relu", need_dx=False, grad_dtype=torch.float32)
    want = dY.sum(0, dtype=torch.float64).repeat(2 if gated else 1)
    tol = (2 * 64 * 2.0**-23 + 13 * 2.0**-24) * want
    assert ((db.double() - want).abs() <= tol).all(), ((db.double() - want).abs() / want).max()


@pytest.mark.parametrize("dtype", TYPES)
def test_two_calls_at_once(dtype):
    """Two contexts on two streams: the same bits as alone."""
    contexts, streams = [binding.Context(0), binding.Context(0)], [torch.cuda.Stream(), torch.cuda.Stream()]
    cases = [Case(dtype, [20000, 0, 9000], 200, 264, "silu", True, seed=61), Case(dtype, [25000, 3000], 256, 100, "relu", False, seed=67)]
    alone = [[t.clone() for t in (c.forward(x), *c.gradient(x)[:3])] for c, x in zip(cases, contexts)]
    torch.cuda.synchronize()
    together = [[], []]
    for _ in range(4):
        for k, (c, x, s) in enumerate(zip(cases, contexts, streams)):
            with torch.cuda.stream(s):
                together[k].append((c.forward(x), *c.gradient(x)[:3]))
    torch.cuda.synchronize()
    for k, c in enumerate(cases):
        a, b = c.o[0], c.o[-1]
        for got in together[k]:
            for t, want in zip(got, alone[k]):
                assert torch.equal(t[a:b], want[a:b]) if t.shape[0] == c.X.shape[0] else torch.equal(t, want)
        contexts[k].check()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_capture_does_not_grow_the_scratch(dtype):
    """Refused with nothing enqueued; after one call outside, it can be captured."""
    ctx = binding.Context(0)
    case = Case(dtype, [300], 33, 47, "silu", True, seed=71)
    with pytest.raises(binding.RtmaError, match="before the capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            case.gradient(ctx)
    want = case.gradient(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = case.gradient(ctx)
    graph.replay()
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a[1:301], b[1:301]) if a.shape[0] == case.X.shape[0] else torch.equal(a, b)


def test_two_graphs_share_the_scratch():
    """Replayed by turns on one stream."""
    ctx = binding.Context(0)
    cases = [Case(torch.bfloat16, [2000, 500], 100, 140, "silu", True, seed=73), Case(torch.float32, [900], 47, 90, "prelu", False, seed=79)]
    wants = [c.gradient(ctx)[1] for c in cases]
    graphs, gots = [torch.cuda.CUDAGraph() for _ in cases], []
    for c, g in zip(cases, graphs):
        with torch.cuda.graph(g):
            gots.append(c.gradient(ctx)[1])
    for _ in range(3):
        for g, got in zip(graphs, gots):
            got.zero_()
            g.replay()
        for got, want in zip(gots, wants):
            assert torch.equal(got, want)


def test_clipping_beyond_32_bits(ctx):
    n = 2**31 + 100
    t = torch.ones(n, dtype=torch.float16, device="cuda")
    norm = n**0.5
    assert abs(ctx.clip_gradients([t], norm / 2)[0].item() - norm) <= 2.0**-23 * norm
    assert t.min() == 0.5 and t.max() == 0.5
    del t
    rows = torch.empty(3 * 1_200_000_000, dtype=torch.bfloat16, device="cuda").as_strided((3, 1001), (1_200_000_000, 1))
    rows.copy_(normal(83, 3, 1001))
    near = rows.contiguous()
    assert torch.equal(ctx.clip_gradients([rows], 1.0, parts=3), ctx.clip_gradients([near], 1.0, parts=3))
    assert torch.equal(rows, near)


def test_most_parts_clipped(ctx):
    t = normal(89, binding.MAX_GROUPS, 37)
    want = t.double().norm(dim=1)
    norms = ctx.clip_gradients([t], 3.0, parts=binding.MAX_GROUPS)
    assert ((norms.double() - want).abs() <= 8 * 2.0**-24 * want).all()
    assert (t.double().norm(dim=1) <= 3.0 * (1 + 2.0**-22)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_stream_of_its_own(dtype):
    """stream=: everything the call makes and launches is on that stream."""
    ctx, stream = binding.Context(0), torch.cuda.Stream()
    case = Case(dtype, [5000, 0, 700], 100, 90, "prelu", True, seed=97)
    want = [t.clone() for t in (case.forward(ctx), *case.gradient(ctx))]
    stream.wait_stream(torch.cuda.current_stream())
    got = (case.forward(ctx, stream=stream), *case.gradient(ctx, stream=stream))
    stream.synchronize()
    a, b = case.o[0], case.o[-1]
    for x, y in zip(got, want):
        assert torch.equal(x[a:b], y[a:b]) if x.shape[0] == case.X.shape[0] else torch.equal(x, y)
