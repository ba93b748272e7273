"""The operators of a whole layer and its step over the rows of many parts, measured by themselves.

A program that trains layers of its own next to the library's partition, sampler and averaging calls has the rows of all parts
(or experts, or relation types) behind one another, the parts' row offsets on the device as the partition leaves them, and one
replica of the parameters per part.  Three operators take such a layer from its rows to the step that trains it:

  linear  a product with bias, activation and a residual branch in its epilogue, and its gradient from the inputs alone: what
          lay in front of the activation is worked out again
  gated   the gated half of a feed-forward block, act(X Wg + bg) * (X Wu + bu) with the two matrices side by side, and its gradient
  clip    the norm of every replica's gradients over all their tensors, and the gradients scaled down to a largest norm

Shapes are those of the named workloads (feature and hidden widths, classes, trainers, nodes) and ragged ones.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SLOPE = 0.25


def listed():
    return [
        # a hidden layer of the Tiny workload with its residual branch: launches and host work are all there is
        _layer("linear_tiny", "linear", "forward", "f32", 2_000, 4, 64, 64, "silu", residual=True),
        # Medium's hidden layer as a residual one, all nodes of its 8 trainers, in the library's own precision
        _layer("linear_residual_f32", "linear", "forward", "f32", 200_000, 8, 256, 256, "relu", residual=True),
        # the way back into the residual stream behind a gated layer: no activation, trainers of unequal size
        _layer("linear_down", "linear", "forward", "bf16", 500_000, 16, 512, 256, "none", residual=True, ragged=True),
        # backward of SuperTMA's hidden layer with the paper's PReLU, a quarter of its nodes
        _layer("linear_gradient", "linear", "grad", "bf16", 500_000, 16, 256, 256, "prelu"),
        # backward of a 47-class head on 100 features: rows that lie on odd boundaries
        _layer("linear_head_gradient", "linear", "grad", "f16", 300_000, 8, 100, 47, "silu", ragged=True),
        # a gated layer on the Tiny workload's nodes
        _layer("gated_tiny", "gated", "forward", "f32", 2_000, 4, 64, 128, "silu"),
        # a gated layer twice as wide as SuperTMA's hidden layer, a quarter of its nodes
        _layer("gated_wide", "gated", "forward", "bf16", 500_000, 16, 256, 512, "silu", ragged=True),
        # its backward pass
        _layer("gated_gradient", "gated", "grad", "bf16", 500_000, 16, 256, 512, "silu"),
        # the same of half of Medium's nodes in full precision
        _layer("gated_gradient_f32", "gated", "grad", "f32", 100_000, 8, 128, 256, "silu"),
        # two thirds of four widths, as gated layers are often cut: 266 columns, rows of odd length
        _layer("gated_odd", "gated", "forward", "f16", 200_000, 5, 100, 266, "silu", ragged=True),
        # the gradients of a Tiny model's layers, clipped into the rows that the averaging step takes
        dict(name="clip_tiny", kind="clip", dtype="f32", M=4, layers=2, d=64, f=128, whole=False),
        # sixteen replicas of a deep model with 16-bit gradients, clipped into the 32-bit gradients that the step takes
        dict(name="clip_large", kind="clip", dtype="bf16", M=16, layers=6, d=512, f=1_024, whole=False),
    ]


def _layer(name, kind, direction, dtype, n, M, d_in, d_out, act, residual=False, ragged=False):
    return dict(name=name, kind=kind, direction=direction, dtype=dtype, n=n, M=M, d_in=d_in, d_out=d_out, act=act, residual=residual,
                ragged=ragged)


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    most_bytes, most_flops = 1.0e9, 7.8e11  # those of clip_large and of gated_gradient
    while True:
        kind = rng.choice(("linear", "linear", "linear", "gated", "gated", "clip"))
        dtype = rng.choice(("f32", "bf16", "f16"))
        M = rng.choice((1, 2, 3, 4, 5, 8, 16, 23, 32, 64))
        if kind == "clip":
            case = dict(kind="clip", dtype=dtype, M=M, layers=rng.randint(1, 12), d=_width(rng), f=_width(rng), whole=rng.random() < 0.3)
        else:
            direction = rng.choice(("forward", "grad"))
            # a kink under a gradient lets the last bit of what is in front of it decide between two answers: fp32 gradients take the smooth ones
            smooth = direction == "grad" and dtype == "f32"
            act = rng.choice(("none", "silu", "silu") if smooth else ("none", "relu", "prelu", "silu"))
            case = _layer("", kind, direction, dtype, _log(rng, 40, 1_000_000), M, _width(rng), _width(rng), act,
                          kind == "linear" and direction == "forward" and rng.random() < 0.5, rng.random() < 0.5)
            case.pop("name")
        w = work(case)
        if w["bytes"] <= most_bytes and w["flops"] <= (most_flops / 12 if dtype == "f32" else most_flops):
            return case


def _width(rng):
    return rng.choice((2, 7, 13, 33, 47, 64, 71, 90, 100, 128, 200, 256, 256, 266, 384, 512))


# ---- inputs ---------------------------------------------------------------------------------------------


def _offsets(n, M, ragged, seed):
    """Row offsets of M parts of n nodes: nodes assigned one by one, or (ragged) parts of very unequal size, one of them empty."""
    rng = np.random.default_rng(seed)
    share = np.full(M, 1.0 / M)
    if ragged and M > 1:
        share = rng.dirichlet(np.full(M, 0.7))
        share[rng.integers(0, M)] = 0.0
        share /= share.sum()
    return [0] + np.cumsum(rng.multinomial(n, share)).tolist()


def _shapes(case):
    """The parameters of one replica: a norm, a gated layer and the product behind it, for every layer."""
    d, f = case["d"], case["f"]
    return [(d,), (d,), (d, 2 * f), (2 * f,), (f, d), (d,)] * case["layers"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case=case)
    M = case["M"]
    if case["kind"] == "clip":
        shapes = _shapes(case)
        # replicas on different parts have gradients of different size; some are above the largest norm, some below
        size = 0.2 + torch.rand(M, generator=g, device="cuda") * 2.0
        s["grads"] = [(normal(M, *shape) * size.view(M, *[1] * len(shape))).to(dtype) for shape in shapes]
        P = sum(math.prod(shape) for shape in shapes)
        s["max_norm"] = math.sqrt(P * (M if case["whole"] else 1.0))
        # where the step takes them from: one row of 32-bit gradients for every replica
        s["flat"] = torch.empty(M, P, device="cuda")
        ends = np.cumsum([math.prod(shape) for shape in shapes]).tolist()
        s["out"] = [s["flat"][:, a:b].unflatten(1, shape) for a, b, shape in zip([0] + ends, ends, shapes)]
        return s
    n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
    wide = 2 * d_out if case["kind"] == "gated" else d_out
    s["host"] = _offsets(n, M, case["ragged"], seed)
    s["offsets"] = torch.tensor(s["host"], dtype=torch.int64, device="cuda")
    s["X"] = (normal(n, d_in) + 0.1).to(dtype)
    s["W"] = (normal(M, d_in, wide) / math.sqrt(d_in)).to(dtype)
    s["b"] = (0.1 * normal(M, wide)).to(dtype)
    s["slope"] = torch.full((M,), SLOPE, device="cuda") if case["act"] == "prelu" else None
    s["residual"] = normal(n, d_out).to(dtype) if case["residual"] else None
    s["dY"] = normal(n, d_out).to(dtype) if case["direction"] == "grad" else None
    return s


# ---- one pass -------------------------------------------------------------------------------------------

_held = {}


def _context():
    if "context" not in _held:
        from paper_2305_09887_b200 import binding
        _held["context"] = binding.Context(0)
    return _held["context"]


def run(s):
    c = s["case"]
    if own:
        ctx = _context()
        if c["kind"] == "clip":
            return ctx.clip_gradients(s["grads"], s["max_norm"], parts=1 if c["whole"] else c["M"], out=s["out"]), s["flat"]
        if c["kind"] == "linear":
            if c["direction"] == "forward":
                return ctx.grouped_linear_act(s["X"], s["offsets"], s["W"], s["b"], act=c["act"], slope=s["slope"], residual=s["residual"])
            grads = ctx.grouped_linear_act_grad(s["X"], s["dY"], s["offsets"], s["W"], s["b"], act=c["act"], slope=s["slope"])
        else:
            if c["direction"] == "forward":
                return ctx.grouped_gated_linear(s["X"], s["offsets"], s["W"], s["b"], act=c["act"], slope=s["slope"])
            grads = ctx.grouped_gated_linear_grad(s["X"], s["dY"], s["offsets"], s["W"], s["b"], act=c["act"], slope=s["slope"])
        return grads if c["act"] == "prelu" else grads[:3]
    if c["kind"] == "clip":
        return _plain_clip(s)
    return (_plain_forward if c["direction"] == "forward" else _plain_grad)(s)


def _parts(s, x):
    """The rows of every part of x (the offsets are the program's own numbers too)."""
    return [x[a:b] for a, b in zip(s["host"], s["host"][1:])]


def _front(s):
    """X W + b in 32 bits, all columns."""
    W, b = s["W"].float(), s["b"].float()
    return torch.cat([torch.addmm(b[g], x.float(), W[g]) for g, x in enumerate(_parts(s, s["X"]))])


def _slopes(s):
    """The slope of every row's part, in a column."""
    h = s["host"]
    return torch.repeat_interleave(s["slope"], torch.tensor([b - a for a, b in zip(h, h[1:])], device="cuda"), output_size=h[-1])[:, None]


def _act(s, z):
    act = s["case"]["act"]
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "prelu":
        return torch.where(z > 0, z, z * _slopes(s))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _derivative(s, z):
    act = s["case"]["act"]
    if act == "relu":
        return (z > 0).float()
    if act == "prelu":
        return torch.where(z > 0, torch.ones_like(z), _slopes(s))
    if act == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    return torch.ones_like(z)


def _plain_forward(s):
    c = s["case"]
    z = _front(s)
    if c["kind"] == "gated":
        f = c["d_out"]
        return (_act(s, z[:, :f]) * z[:, f:]).to(s["X"].dtype)
    y = _act(s, z)
    return (y + s["residual"].float() if s["residual"] is not None else y).to(s["X"].dtype)


def _plain_grad(s):
    c = s["case"]
    dtype = s["X"].dtype
    z, dy = _front(s), s["dY"].float()
    if c["kind"] == "gated":
        f = c["d_out"]
        z, up = z[:, :f], z[:, f:]
        dz = torch.cat([dy * up * _derivative(s, z), dy * _act(s, z)], dim=1)
        dy = dy * up
    else:
        dz = dy * _derivative(s, z)
    W = s["W"].float()
    rows = _parts(s, dz)
    dx = torch.cat([d @ W[g].T for g, d in enumerate(rows)]).to(dtype)
    dw = torch.stack([x.float().T @ d for x, d in zip(_parts(s, s["X"]), rows)]).to(dtype)
    db = torch.stack([d.sum(0) for d in rows]).to(dtype)
    if c["act"] != "prelu":
        return dx, dw, db
    # a sum of terms of either sign, of which next to nothing is left: in 64 bits
    dslope = torch.stack([(y.double() * torch.clamp(t, max=0)).sum() for y, t in zip(_parts(s, dy), _parts(s, z))])
    return dx, dw, db, dslope.float()


def _plain_clip(s):
    c = s["case"]
    squares = torch.stack([(g.float() ** 2).flatten(1).sum(1) for g in s["grads"]]).sum(0)
    if c["whole"]:
        squares = squares.sum(0, keepdim=True)
    norms = torch.sqrt(squares)
    scale = torch.clamp(s["max_norm"] / norms, max=1.0).expand(c["M"])
    return norms, torch.cat([g.float().flatten(1) * scale[:, None] for g in s["grads"]], dim=1)


# ---- work -----------------------------------------------------------------------------------------------


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    M = case["M"]
    if case["kind"] == "clip":
        P = float(M) * sum(math.prod(shape) for shape in _shapes(case))
        return {"bytes": P * (size + 4) + 4.0 * M, "flops": 3.0 * P}
    n, d_in, d_out = float(case["n"]), case["d_in"], case["d_out"]
    wide = 2 * d_out if case["kind"] == "gated" else d_out
    weights = float(M) * (d_in + 1) * wide * size
    if case["direction"] == "forward":
        return {"bytes": n * (d_in + d_out * (2 if case["residual"] else 1)) * size + weights, "flops": 2.0 * n * d_in * wide}
    # what is in front of the activation, the rows' gradient and the weights' (a layer without either activation or gate needs the last two)
    products = 2 if case["act"] == "none" and case["kind"] == "linear" else 3
    return {"bytes": n * (2 * d_in + d_out) * size + 2 * weights, "flops": 2.0 * products * n * d_in * wide}


# ---- the definitions in 64 bits -------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    M = case["M"]
    if case["kind"] == "clip":
        flat = torch.cat([g.to(f64).reshape(M, -1) for g in s["grads"]], dim=1)
        if case["whole"]:
            norms = torch.linalg.vector_norm(flat).reshape(1)
        else:
            norms = torch.linalg.vector_norm(flat, dim=1)
        over = (norms > s["max_norm"]).to(f64)
        return norms, flat * (over * (s["max_norm"] / norms) + (1 - over)).reshape(-1, 1)
    f = case["d_out"]
    grad = case["direction"] == "grad"
    outs = []
    for g, (a, b) in enumerate(zip(s["host"], s["host"][1:])):
        # the definition, and its derivatives by the chain rule that torch applies to it
        x = s["X"][a:b].to(f64).requires_grad_(grad)
        w = s["W"][g].to(f64).requires_grad_(grad)
        bias = s["b"][g].to(f64).requires_grad_(grad)
        slope = torch.tensor(SLOPE, dtype=f64, device="cuda", requires_grad=grad)
        z = torch.einsum("ri,io->ro", x, w) + bias
        front = z[:, :f]
        if case["act"] == "relu":
            y = torch.where(front > 0, front, torch.zeros((), dtype=f64, device="cuda"))
        elif case["act"] == "prelu":
            y = torch.where(front > 0, front, slope * front)
        elif case["act"] == "silu":
            y = front * torch.sigmoid(front)
        else:
            y = front
        if case["kind"] == "gated":
            y = y * z[:, f:]
        if case["residual"]:
            y = y + s["residual"][a:b].to(f64)
        if not grad:
            outs.append(y)
            continue
        wanted = [x, w, bias] + ([slope] if case["act"] == "prelu" else [])
        outs.append([t.detach() for t in torch.autograd.grad((y * s["dY"][a:b].to(f64)).sum(), wanted)])
    if not grad:
        return torch.cat(outs)
    dx, rest = torch.cat([o[0] for o in outs]), [torch.stack(t) for t in zip(*[o[1:] for o in outs])]
    return (dx, *rest)
