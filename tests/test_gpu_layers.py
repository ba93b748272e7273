"""Whole layers on the rows of many parts (product with bias, activation and residual; gated product) and their gradients, against their
definitions in 64 bits.  layer_reference says where the tolerances come from."""
import pytest
import torch

from layer_reference import F64, Layer, half_step, rounding
from paper_2305_09887_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = ["none", "relu", "prelu", "silu"]


@pytest.fixture(scope="module")
def ctx():
    return binding.Context(0)


def normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


def rows_of(values, dtype, pad=0, shift=0, behind=2):
    """The values as rows whose distance is d + pad elements, `shift` elements behind an aligned address, `behind` rows of NaN after them;
    everything else is NaN."""
    n, d = values.shape
    flat = torch.full(((n + behind) * (d + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    view = flat[shift:shift + (n + behind) * (d + pad)].view(n + behind, d + pad)[:, :d]
    view[:n].copy_(values.to(dtype))
    return view


def offsets_of(sizes, first):
    o = [first]
    for s in sizes:
        o.append(o[-1] + s)
    return o, torch.tensor(o, dtype=torch.int64, device="cuda")


def assert_close(got, want, tol, what=""):
    bad = ~((got.to(F64) - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}: " \
                          f"{got[bad][0].item()} for {want[bad][0].item()}, off by {((got.to(F64) - want).abs() / tol)[bad].max().item():.3g} tolerances"


def assert_near(got, want, dtype, what, kink=0.0):
    """As a whole: independent roundings, of the rows' type at most two, are off by less than two half steps of the 2-norm (a rounding's
    rms is below half a step).  kink: the 2-norm of what entries that may lie on either side of a kink change (one such entry of 1,500 x 1,024
    moves dW of 264 columns by sqrt(264) |x dY U (1 - slope)|, 1e-3 of its norm: above 2^-10)."""
    most = 2 * half_step(dtype) if dtype != torch.float32 else 2e-6
    off, size = (got.to(F64) - want).norm().item(), want.norm().item()
    assert off <= most * size + kink + 1e-30, f"{what}: {off / size if size else off:.3g} of the norm off, {most:.3g} allowed"


class Case:
    """A call's tensors: parts of the sizes, rows before the first part and behind the last that belong to none and hold NaN."""

    def __init__(self, dtype, sizes, d_in, d_out, act, gated, bias=True, residual=False, pad=0, shift=0, seed=0, shared=False, before=1):
        self.dtype, self.act, self.gated, self.sizes = dtype, act, gated, sizes
        n, G, wide = sum(sizes), len(sizes), 2 * d_out if gated else d_out
        self.o, self.offsets = offsets_of(sizes, before)
        lead = torch.full((before, max(d_in, d_out)), float("nan"), device="cuda")
        put = lambda v: rows_of(torch.cat([lead[:, :v.shape[1]], v]), dtype, pad, shift)  # noqa: E731
        self.X, self.dY = put(normal(seed, n, d_in) + 0.1), put(normal(seed + 1, n, d_out))
        self.residual = put(normal(seed + 2, n, d_out)) if residual else None
        lead_W = () if shared else (G,)
        self.W = (normal(seed + 3, *lead_W, d_in, wide) / d_in**0.5).to(dtype)
        self.b = (0.3 * normal(seed + 4, *lead_W, wide)).to(dtype) if bias else None
        self.slope = torch.linspace(0.1, 0.4, G, device="cuda") if act == "prelu" else None
        self.d_in, self.d_out, self.wide, self.shared = d_in, d_out, wide, shared

    def how(self):
        return dict(bias=self.b, act=self.act, slope=self.slope)

    def parts(self, grad=False):
        for g, (a, b) in enumerate(zip(self.o, self.o[1:])):
            w, bias = (self.W, self.b) if self.shared else (self.W[g], None if self.b is None else self.b[g])
            yield g, a, b, Layer(self.X[a:b], w, bias, self.act, 0.0 if self.slope is None else self.slope[g].item(), self.gated, self.dtype,
                                 None if self.residual is None else self.residual[a:b], self.dY[a:b] if grad else None)

    def forward(self, ctx, **more):
        return (ctx.grouped_gated_linear if self.gated else ctx.grouped_linear_act)(self.X, self.offsets, self.W, residual=self.residual, **self.how(), **more)

    def gradient(self, ctx, **more):
        return (ctx.grouped_gated_linear_grad if self.gated else ctx.grouped_linear_act_grad)(self.X, self.dY, self.offsets, self.W, **self.how(), **more)

    def check_forward(self, ctx):
        n = self.X.shape[0]
        out = rows_of(torch.full((n - 2, self.d_out), 7.0, device="cuda"), self.dtype, 3)
        out[n - 2:] = 7.0
        got = self.forward(ctx, out=out)
        ctx.check()
        assert got is out
        for g, a, b, want in self.parts():
            assert_close(out[a:b], want.y, want.y_off, f"part {g}")
        assert (out[:self.o[0]] == 7).all() and (out[self.o[-1]:] == 7).all(), "rows of no part were written"

    def check_gradient(self, ctx, grad_dtype=None):
        n = self.X.shape[0]
        out = rows_of(torch.full((n - 2, self.d_in), 7.0, device="cuda"), self.dtype, 3)
        up = (self.d_out + 7) // 8 * 8  # halves are rounded up, with zeros behind
        dz = rows_of(torch.full((n - 2, self.wide // self.d_out * up), 7.0, device="cuda"), self.dtype)
        out[n - 2:] = dz[n - 2:] = 7.0
        made = self.gated or self.act != "none"
        dx, dw, db, dslope = self.gradient(ctx, out=out, dz=dz if made else None, grad_dtype=grad_dtype)
        ctx.check()
        kind = grad_dtype or self.dtype
        assert dx is out and dw.shape == self.W.shape and dw.dtype == kind and (db is None) == (self.b is None) and (dslope is None) == (self.slope is None)
        total = 0
        for g, a, b, want in self.parts(grad=True):
            assert_close(dx[a:b], want.dx, want.dx_off, f"dX of part {g}")
            if made:
                for h in range(self.wide // self.d_out):
                    real = slice(h * self.d_out, (h + 1) * self.d_out)
                    assert_close(dz[a:b, h * up:h * up + self.d_out], want.dz[:, real], want.dz_off[:, real], f"dZ of part {g}")
                    assert not dz[a:b, h * up + self.d_out:(h + 1) * up].any()
            if self.slope is not None:
                assert_close(dslope[g], want.dslope, want.dslope_off + rounding(want.dslope, torch.float32), f"dslope of part {g}")
            if self.shared:
                total = [x + y for x, y in zip(total, (want.dw, want.dw_off, want.db, want.db_off))] if total else [want.dw, want.dw_off, want.db, want.db_off]
                continue
            assert_close(dw[g], want.dw, want.dw_off + rounding(want.dw.abs() + want.dw_off, kind), f"dW of part {g}")
            assert_near(dw[g], want.dw, self.dtype, f"dW of part {g}", want.dw_kink)
            if db is not None:
                assert_close(db[g], want.db, want.db_off + rounding(want.db.abs() + want.db_off, kind), f"db of part {g}")
        if self.shared:
            assert_close(dw, total[0], total[1] + rounding(total[0].abs() + total[1], kind), "dW")
            if db is not None:
                assert_close(db, total[2], total[3] + rounding(total[2].abs() + total[3], kind), "db")
        for t in (dx, dz) if made else (dx,):
            assert (t[:self.o[0]] == 7).all() and (t[self.o[-1]:] == 7).all(), "rows of no part were written"


# (part sizes, d_in, d_out): one row, none, edges of tiles of 128 rows, of 16, 32, 64, 128 and 256 columns, of 16-byte boundaries
SHAPES = [
    ([1], 1, 1), ([0], 5, 3), ([2, 0, 1], 2, 2), ([31, 33], 7, 13), ([127, 1, 128], 33, 47), ([129, 0, 300], 64, 64), ([200], 100, 266), ([65, 190], 47, 90),
    ([300, 5], 128, 128), ([140], 256, 130), ([64, 64], 130, 256), ([257], 72, 272), ([100, 0, 0, 28], 300, 33), ([1, 1, 1, 1, 1, 1, 1], 64, 8), ([500], 16, 24),
]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_forward(ctx, dtype, sizes, d_in, d_out, gated):
    act = ACTS[(d_in + d_out) % 4]
    Case(dtype, sizes, d_in, d_out, act, gated, bias=d_in != 64, residual=d_out % 2 == 0).check_forward(ctx)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,d_in,d_out", SHAPES)
def test_gradient(ctx, dtype, sizes, d_in, d_out, gated):
    act = ACTS[(d_in + d_out + 1) % 4]
    Case(dtype, sizes, d_in, d_out, act, gated, bias=d_in != 64).check_gradient(ctx)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_every_activation(ctx, dtype, gated, act):
    case = Case(dtype, [90, 0, 150], 48, 80, act, gated, residual=True, seed=5)
    case.check_forward(ctx)
    case.check_gradient(ctx, torch.float32)


@pytest.mark.parametrize("pad,shift", [(1, 0), (0, 1), (4, 4), (8, 0), (3, 2)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_on_any_boundary(ctx, dtype, gated, pad, shift):
    case = Case(dtype, [150, 61], 64, 96, "silu", gated, residual=True, pad=pad, shift=shift, seed=9)
    case.check_forward(ctx)
    case.check_gradient(ctx)


@pytest.mark.parametrize("gated,d_out", [(True, 1024), (False, 2048)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_pairs_of_blocks(ctx, dtype, gated, d_out):
    """Deep contractions over whole tiles: parts that end in either half of a pair's 256 rows, and before it."""
    case = Case(dtype, [700, 100, 0, 256, 1500, 129], 256, d_out, "silu", gated, residual=True, seed=13)
    case.check_forward(ctx)
    case.check_gradient(ctx)
    Case(dtype, [1100, 1500, 129], 264, d_out, "prelu", gated, seed=14).check_gradient(ctx)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_matrix_for_all_parts_and_no_parts_at_all(ctx, dtype, gated):
    case = Case(dtype, [70, 0, 200], 40, 56, "silu", gated, seed=17, shared=True)
    case.check_forward(ctx)
    case.check_gradient(ctx, torch.float32)
    call = ctx.grouped_gated_linear if gated else ctx.grouped_linear_act
    X = case.X[1:271].contiguous()
    whole = call(X, None, case.W, bias=case.b, act="silu")
    assert torch.equal(whole, case.forward(ctx, out=torch.empty_like(case.dY))[1:271].contiguous())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_slope_for_all_parts(ctx, dtype, gated):
    case = Case(dtype, [70, 0, 200], 40, 56, "prelu", gated, seed=19)
    case.slope = torch.full((1,), 0.25, device="cuda").expand(3)
    want = [w.dslope for *_, w in case.parts(grad=True)], [w.dslope_off for *_, w in case.parts(grad=True)]
    case.slope = torch.tensor(0.25, device="cuda")
    *_, dslope = case.gradient(ctx)
    assert dslope.shape == ()
    assert_close(dslope, sum(want[0]), sum(want[1]) + rounding(sum(want[0]), torch.float32), "dslope")


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_what_is_not_wanted(ctx, dtype, gated):
    case = Case(dtype, [150, 80], 64, 64, "silu", gated, residual=True, seed=21)
    want = case.forward(ctx)
    again = case.residual
    assert case.forward(ctx, out=again) is again
    assert torch.equal(again[1:231], want[1:231])
    dx, dw, db, _ = case.gradient(ctx)
    only = case.gradient(ctx, need_dw=False)
    assert torch.equal(only[0][1:231], dx[1:231]) and only[1] is only[2] is only[3] is None
    only = case.gradient(ctx, need_dx=False)
    assert only[0] is None and torch.equal(only[1], dw) and torch.equal(only[2], db)
    if not gated:  # dZ in dY's place
        assert torch.equal(case.gradient(ctx, dz=case.dY)[0][1:231], dx[1:231])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_stays_in_its_row(ctx, dtype, gated, bad):
    case = Case(dtype, [130, 60], 40, 48, "silu", gated, seed=23)
    clean, grads = case.forward(ctx), case.gradient(ctx)
    case.X[100, 3] = bad
    y, (dx, dw, db, _) = case.forward(ctx), case.gradient(ctx)
    keep = [r for r in range(1, 191) if r != 100]
    assert torch.equal(y[keep], clean[keep]) and torch.equal(dx[keep], grads[0][keep])
    assert not torch.isfinite(y[100]).all()
    assert torch.equal(dw[1], grads[1][1]) and torch.equal(db[1], grads[2][1])


def test_relu_of_what_is_not_finite(ctx):
    """ReLU keeps NaN and plus infinity, and its gradient lets nothing through where the product is not positive."""
    X = torch.tensor([[1.0], [float("inf")], [-1.0], [float("nan")]], device="cuda", dtype=torch.bfloat16)
    W = torch.ones(1, 8, device="cuda", dtype=torch.bfloat16)
    y = ctx.grouped_linear_act(X, None, W, act="relu")
    assert y[0].eq(1).all() and y[1].isinf().all() and y[2].eq(0).all() and y[3].isnan().all()
    dY = torch.full((4, 8), float("inf"), device="cuda", dtype=torch.bfloat16)
    dz = torch.empty_like(dY)
    ctx.grouped_linear_act_grad(X, dY, None, W, act="relu", dz=dz, need_dw=False)
    assert dz[0].isinf().all() and dz[2].eq(0).all()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_against_differences(ctx, dtype, gated):
    """The slope of the sum of dY * Y along a direction: the forward pass in 64 bits at either side, the gradient from the kernel."""
    case = Case(dtype, [40, 23], 24, 32, "silu", gated, seed=29)
    dx, dw, db, _ = case.gradient(ctx, grad_dtype=torch.float32)
    step = 1e-4
    for name, grad in (("X", dx[1:64]), ("W", dw), ("b", db)):
        base = getattr(case, name)
        held = base if name != "X" else base[1:64]
        direction = normal(31, *held.shape).to(F64)

        def at(t):
            moved = held.to(F64) + t * direction
            total = 0.0
            for g, (a, b) in enumerate(zip(case.o, case.o[1:])):
                x = moved[a - 1:b - 1] if name == "X" else case.X[a:b]
                w, bias = (moved[g] if name == "W" else case.W[g]), (moved[g] if name == "b" else case.b[g])
                y = Layer(x, w, bias, "silu", 0.0, gated, dtype).y
                total += (y * case.dY[a:b].to(F64)).sum().item()
            return total

        slope = (at(step) - at(-step)) / (2 * step)
        got = (grad.to(F64) * direction).sum().item()
        # two roundings to the rows' type at most on the way to a gradient, of independent signs; the difference itself is good to step^2
        most = 2 * half_step(dtype) * grad.to(F64).norm().item() * direction.norm().item() / (direction.numel() ** 0.5) * 4 + 1e-5 * grad.to(F64).norm().item() + 1e-5
        assert abs(got - slope) <= most, (name, got, slope, most)


def chain(ctx, dtype, n=900, streams=None):
    """A block as it is used, there and back and to the step: a gated layer, the product back into the residual stream, the
    gradients of both, clipped for each replica into the rows that the averaging step takes.  Returns everything that is computed."""
    G, d, f = 3, 96, 160
    offsets = torch.tensor([0, 400, 400, n], dtype=torch.int64, device="cuda")
    X, dY = normal(41, n, d).to(dtype), normal(42, n, d).to(dtype)
    params = 0.1 * normal(43, G, d * 2 * f + 2 * f + f * d + d)
    shapes = [(d, 2 * f), (2 * f,), (f, d), (d,)]
    ends = [0]
    for s in shapes:
        ends.append(ends[-1] + (s[0] * s[1] if len(s) == 2 else s[0]))
    views = lambda t: [t[:, a:b].unflatten(1, s) for a, b, s in zip(ends, ends[1:], shapes)]  # noqa: E731
    W1, b1, W2, b2 = (p.to(dtype) for p in views(params))
    H = ctx.grouped_gated_linear(X, offsets, W1, b1)
    Y = ctx.grouped_linear_act(H, offsets, W2, b2, residual=X)
    dH, dW2, db2, _ = ctx.grouped_linear_act_grad(H, dY, offsets, W2, b2)
    dX, dW1, db1, _ = ctx.grouped_gated_linear_grad(X, dH, offsets, W1, b1)
    grads = torch.empty_like(params)
    norms = ctx.clip_gradients([dW1, db1, dW2, db2], 5.0, parts=G, out=views(grads))
    stepped = params.clone()
    ctx.sgd_aggregate(stepped, grads, 0.1)
    return dict(X=X, dY=dY, params=params, H=H, Y=Y, dH=dH, dX=dX, dW1=dW1, db1=db1, dW2=dW2, db2=db2, norms=norms, grads=grads, stepped=stepped,
                parts=(W1, b1, W2, b2), offsets=[0, 400, 400, n])


@pytest.mark.parametrize("dtype", TYPES)
def test_a_block_there_and_back_and_its_step(ctx, dtype):
    r = chain(ctx, dtype)
    ctx.check()
    W1, b1, W2, b2 = r["parts"]
    most = 4 * half_step(dtype) if dtype != torch.float32 else 4e-6  # four roundings to the rows' type at most lie on a way
    f = W2.shape[1]
    for g, (a, b) in enumerate(zip(r["offsets"], r["offsets"][1:])):
        p = [t[g].to(F64).requires_grad_() for t in (W1, b1, W2, b2)]
        x = r["X"][a:b].to(F64).requires_grad_()
        z = x @ p[0] + p[1]
        h = z[:, :f] * torch.sigmoid(z[:, :f]) * z[:, f:]
        y = x + h @ p[2] + p[3]
        (y * r["dY"][a:b].to(F64)).sum().backward()
        near = lambda got, want: (got.to(F64) - want).norm() <= most * want.norm() + 1e-30  # noqa: E731
        assert near(r["H"][a:b], h.detach()) and near(r["Y"][a:b], y.detach())
        assert near(r["dX"][a:b] + r["dY"][a:b].to(torch.float32), x.grad)  # the residual's gradient is dY itself
        flat = []
        for got, want in zip((r["dW1"], r["db1"], r["dW2"], r["db2"]), p):
            assert near(got[g], want.grad)
            flat.append(got[g].to(F64).flatten())
        flat = torch.cat(flat)
        norm = flat.norm().item()
        assert abs(r["norms"][g].item() - norm) <= 1e-6 * norm
        assert_close(r["grads"][g], flat * min(1.0, 5.0 / norm if norm else 1.0), 2e-7 * flat.abs(), "clipped")
    want = (r["params"].to(F64) - 0.1 * r["grads"].to(F64)).mean(0)
    assert_close(r["stepped"], want.expand_as(r["stepped"]), 1e-6 * (1 + want.abs()), "step")


@pytest.mark.parametrize("dtype", TYPES)
def test_the_block_in_a_graph_and_on_another_stream(dtype):
    ctx = binding.Context(0)
    want = chain(ctx, dtype)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        beside = chain(ctx, dtype)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    X, dY = want["X"], want["dY"]
    offsets = torch.tensor(want["offsets"], dtype=torch.int64, device="cuda")
    W1, b1, W2, b2 = want["parts"]
    with torch.cuda.graph(graph):
        H = ctx.grouped_gated_linear(X, offsets, W1, b1)
        Y = ctx.grouped_linear_act(H, offsets, W2, b2, residual=X)
        dH, dW2, db2, _ = ctx.grouped_linear_act_grad(H, dY, offsets, W2, b2)
        dX, dW1, db1, _ = ctx.grouped_gated_linear_grad(X, dH, offsets, W1, b1)
        norms = ctx.clip_gradients([dW1, db1, dW2, db2], 5.0, parts=3)
    for _ in range(2):
        for t in (H, Y, dH, dX, dW1, dW2, norms):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in dict(H=H, Y=Y, dH=dH, dX=dX, norms=norms).items():
            assert torch.equal(t, want[name]), name
            assert torch.equal(t, beside[name]), name
    ctx.check()
    # the replay follows its inputs, and offsets that have moved
    X.mul_(0.5)
    offsets.copy_(torch.tensor([0, 100, 500, 900], dtype=torch.int64))
    graph.replay()
    assert torch.equal(H, ctx.grouped_gated_linear(X, offsets, W1, b1))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(ctx, dtype, gated):
    X = torch.empty(0, 12, dtype=dtype, device="cuda")
    W = torch.ones(2, 12, 16, dtype=dtype, device="cuda")
    d_out = 8 if gated else 16
    offsets = torch.zeros(3, dtype=torch.int64, device="cuda")
    dY = torch.empty(0, d_out, dtype=dtype, device="cuda")
    slope = torch.ones(2, device="cuda")
    bias = torch.ones(2, 16, dtype=dtype, device="cuda")
    forward, back = (ctx.grouped_gated_linear, ctx.grouped_gated_linear_grad) if gated else (ctx.grouped_linear_act, ctx.grouped_linear_act_grad)
    assert forward(X, offsets, W, bias, act="prelu", slope=slope).shape == (0, d_out)
    dx, dw, db, dslope = back(X, dY, offsets, W, bias, act="prelu", slope=slope)
    assert dx.shape == (0, 12) and not dw.any() and not db.any() and not dslope.any()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_same_bits_every_time(ctx, dtype, gated):
    case = Case(dtype, [3000, 0, 1700], 100, 140, "prelu", gated, seed=37)
    first = [t.clone() for t in (case.forward(ctx), *case.gradient(ctx))]
    for _ in range(3):
        again = (case.forward(ctx), *case.gradient(ctx))
        for a, b in zip(first, again):
            assert torch.equal(a[1:4701] if a.shape[0] == case.X.shape[0] else a, b[1:4701] if a.shape[0] == case.X.shape[0] else b)


def test_replicas_where_they_lie(ctx):
    """Matrices and gradients as views of params [M, P] and grads [M, P], at odd places."""
    M, d, f, P = 4, 30, 21, 3001
    params, grads = normal(47, M, P), torch.full((M, P), 5.0, device="cuda")
    views = lambda t: (t[:, 7:7 + d * 2 * f].unflatten(1, (d, 2 * f)), t[:, 2000:2000 + 2 * f])  # noqa: E731
    W, b = views(params)
    dw, db = views(grads)
    X, dH = normal(48, 500, d), normal(49, 500, f)
    offsets = torch.tensor([0, 100, 100, 333, 500], dtype=torch.int64, device="cuda")
    same = ctx.grouped_gated_linear(X, offsets, W.contiguous(), b.contiguous())
    assert torch.equal(ctx.grouped_gated_linear(X, offsets, W, b), same)
    want = ctx.grouped_gated_linear_grad(X, dH, offsets, W.contiguous(), b.contiguous())
    got = ctx.grouped_gated_linear_grad(X, dH, offsets, W, b, dw=dw, db=db)
    assert torch.equal(got[0], want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])
    rest = grads.clone()
    for v in views(rest):
        v.fill_(5.0)
    assert (rest == 5).all()
