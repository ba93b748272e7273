"""The operators of a layer over the rows of many parts, measured by themselves.

A program that writes a layer next to the library's partition, sampler and averaging calls has the rows of all parts (or
experts, or relation types) behind one another, the parts' row offsets on the device as the partition leaves them, and one
replica of the parameters per part.  Three operators work on that:

  linear    the product of every part's rows with the part's own matrix: forward, input gradient, weight and bias gradient
  norm      group norm over the channels of a row ("row") or of a whole part ("part"), channels last, with the activation and
            dropout behind it, forward and gradient
  dropout   dropout whose mask is a hash of (seed, row id, column) and is never stored; its gradient is the same call

Shapes are those of the named workloads (feature and hidden widths, classes, trainers, nodes) and ragged ones.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
SLOPE = 0.25


def listed():
    return [
        # the Tiny workload's first layer: 4 trainers, 2,000 nodes; launches and host work are all there is
        _linear("linear_tiny", "forward", "f32", 2_000, 4, 64, 64),
        # Medium's first layer on all nodes of its 8 trainers, in the library's own precision
        _linear("linear_medium", "forward", "f32", 200_000, 8, 128, 256),
        # the width sweep's hidden layer with rows of half the size
        _linear("linear_sweep", "forward", "bf16", 500_000, 8, 512, 512),
        # backward through SuperTMA's hidden layer at full size, trainers of unequal size
        _linear("linear_input_gradient", "dx", "bf16", 2_000_000, 16, 256, 256, ragged=True),
        # the weight gradient of a 47-class head
        _linear("linear_head_gradient", "dw", "f32", 200_000, 8, 256, 47),
        # the weight gradient of SuperTMA's first layer (100 features), parts of unequal size and one of them empty
        _linear("linear_weight_gradient", "dw", "f16", 1_000_000, 16, 100, 256, ragged=True),
        # per-node normalisation of the Tiny workload
        _norm("norm_tiny", "forward", "f32", 2_000, 4, 64, 1, "row", "prelu"),
        # backward of Medium's hidden layer with per-node statistics and dropout
        _norm("norm_row_gradient", "grad", "f32", 200_000, 8, 256, 8, "row", "silu", p=0.5),
        # statistics over each whole part, SuperTMA's nodes, half-size rows
        _norm("norm_part", "forward", "bf16", 2_000_000, 16, 128, 32, "part", "silu"),
        # and its gradient on a quarter of them
        _norm("norm_part_gradient", "grad", "bf16", 500_000, 16, 256, 32, "part", "silu", ragged=True),
        # the inputs of the Tiny workload's layer
        dict(name="dropout_tiny", kind="dropout", direction="forward", dtype="f32", n=2_000, d=64, p=0.5, ids=False, residual=False),
        # a fifth of the Large workload's nodes in partition order with a residual branch; the mask goes by node id
        dict(name="dropout_large", kind="dropout", direction="forward", dtype="bf16", n=5_000_000, d=128, p=0.1, ids=True, residual=True),
    ]


def _linear(name, direction, dtype, n, M, d_in, d_out, ragged=False):
    return dict(name=name, kind="linear", direction=direction, dtype=dtype, n=n, M=M, d_in=d_in, d_out=d_out, ragged=ragged)


def _norm(name, direction, dtype, n, M, C, groups, scope, act, p=0.0, ragged=False):
    return dict(name=name, kind="norm", direction=direction, dtype=dtype, n=n, M=M, C=C, groups=groups, scope=scope, act=act, p=p,
                ragged=ragged)


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    most_bytes, most_flops = 4.0e9, 2.7e11  # those of dropout_large and of linear_sweep
    while True:
        kind = rng.choice(("linear", "linear", "linear", "norm", "norm", "dropout"))
        dtype = rng.choice(("f32", "bf16", "f16"))
        n = _log(rng, 40, 2_000_000)
        M = rng.choice((1, 2, 3, 4, 5, 8, 16, 23, 32, 64))
        ragged = rng.random() < 0.5
        if kind == "linear":
            case = _linear("", rng.choice(("forward", "dx", "dw")), dtype, n, M, _width(rng), _width(rng), ragged)
        elif kind == "norm":
            # a kink under a gradient lets the last bit of u decide between two answers: gradients take the smooth activations
            direction = rng.choice(("forward", "grad"))
            act = rng.choice(("none", "silu") if direction == "grad" else ("none", "relu", "prelu", "silu"))
            C = _width(rng)
            scope = rng.choice(("row", "part"))
            # two channels a row or more: the normalisation of a single value is zero
            groups = rng.choice([k for k in (1, 2, 4, 8, 16, 32, C) if C % k == 0 and (scope == "part" or C // k >= 2)] or [1])
            case = _norm("", direction, dtype, n, M, C, groups, scope, act, rng.choice((0.0, 0.0, 0.1, 0.5)), ragged)
            if C < 2 or (scope == "part" and n < 40 * M):  # parts of a row or two have next to no variance
                continue
        else:
            case = dict(kind="dropout", direction="forward", dtype=dtype, n=_log(rng, 40, 5_000_000), d=_width(rng),
                        p=rng.choice((0.1, 0.2, 0.5, 0.9)), ids=rng.random() < 0.5, residual=rng.random() < 0.5)
        case.pop("name", None)
        w = work(case)
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops and (dtype != "f32" or kind != "linear" or w["flops"] <= most_flops / 3):
            return case


def _width(rng):
    return rng.choice((2, 7, 13, 33, 47, 64, 71, 90, 100, 128, 200, 256, 256, 384, 512))


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


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    n = case["n"]
    s = dict(case=case)
    if case["kind"] == "dropout":
        s["X"] = normal(n, case["d"]).to(dtype)
        s["residual"] = normal(n, case["d"]).to(dtype) if case["residual"] else None
        # rows in partition order: the ids of the nodes that they are
        s["ids"] = torch.randperm(n, generator=g, device="cuda", dtype=torch.int32) if case["ids"] else None
        s["seed"] = int(seed) * 1_000_003 + 17
        return s
    M = case["M"]
    s["host"] = _offsets(n, M, case["ragged"], seed)
    s["offsets"] = torch.tensor(s["host"], dtype=torch.int64, device="cuda")
    if case["kind"] == "linear":
        d_in, d_out = case["d_in"], case["d_out"]
        if case["direction"] != "dx":
            # activations behind a ReLU and features around zero both occur: normal values with a small mean
            s["X"] = (normal(n, d_in) + 0.1).to(dtype)
        if case["direction"] != "dw":
            s["W"] = (normal(M, d_in, d_out) / math.sqrt(d_in)).to(dtype)
            s["b"] = (0.1 * normal(M, d_out)).to(dtype)
        if case["direction"] != "forward":
            s["dY"] = normal(n, d_out).to(dtype)
        return s
    C = case["C"]
    # products of a layer: every channel has a mean and a scale of its own, every row a little of its own
    s["X"] = (normal(n, C) * (0.5 + torch.rand(C, generator=g, device="cuda")) + 0.5 * normal(C) + 0.1 * normal(n, 1)).to(dtype)
    s["gamma"] = 1.0 + 0.2 * normal(M, C)
    s["beta"] = 0.2 * normal(M, C)
    s["slope"] = torch.full((M,), SLOPE, device="cuda") if case["act"] == "prelu" else None
    s["seed"] = int(seed) * 1_000_003 + 29
    if case["direction"] == "grad":
        s["dY"] = normal(n, C).to(dtype)
        s["stats"] = _stats(s, torch.float64).to(torch.float32)  # kept from the forward pass
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
        if c["kind"] == "dropout":
            return ctx.dropout(s["X"], c["p"], s["seed"], row_ids=s["ids"], residual=s["residual"])
        if c["kind"] == "linear":
            if c["direction"] == "forward":
                return ctx.grouped_linear(s["X"], s["offsets"], s["W"], s["b"])
            if c["direction"] == "dx":
                return ctx.grouped_linear_dx(s["dY"], s["offsets"], s["W"])
            return ctx.grouped_linear_dw(s["X"], s["dY"], s["offsets"])
        how = dict(scope=c["scope"], act=c["act"], slope=s["slope"], p=c["p"], seed=s["seed"])
        if c["direction"] == "forward":
            return ctx.group_norm(s["X"], s["offsets"], c["groups"], s["gamma"], s["beta"], eps=EPS, **how)
        dx, dgamma, dbeta, _ = ctx.group_norm_grad(s["X"], s["dY"], s["stats"], s["offsets"], c["groups"], s["gamma"], s["beta"], **how)
        return dx, dgamma, dbeta
    return {"dropout": _plain_dropout, "linear": _plain_linear, "norm": _plain_norm}[c["kind"]](s)


def _parts(s, x):
    """The rows of every part of x (the offsets are the program's own numbers too)."""
    return [x[a:b] for a, b in zip(s["host"], s["host"][1:])]


def _plain_linear(s):
    c = s["case"]
    dtype = DTYPES[c["dtype"]]
    if c["direction"] == "forward":
        W, b = s["W"].float(), s["b"].float()
        return torch.cat([torch.addmm(b[g], x.float(), W[g]) for g, x in enumerate(_parts(s, s["X"]))]).to(dtype)
    if c["direction"] == "dx":
        W = s["W"].float()
        return torch.cat([y.float() @ W[g].T for g, y in enumerate(_parts(s, s["dY"]))]).to(dtype)
    X, dY = _parts(s, s["X"].float()), _parts(s, s["dY"].float())
    return torch.stack([x.T @ y for x, y in zip(X, dY)]), torch.stack([y.sum(0) for y in dY])


def _mix(z):
    """One SplitMix64 step of 64-bit words held as signed numbers (products wrap; shifts are made logical)."""
    z = z + -7046029254386353131
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * -4658895280553007687
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * -7723592293110705685
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _keep_scale(seed, ids, n, d, p, device):
    """What dropout multiplies by: 0, or one over the share that is kept; float32 [n, d]."""
    t = math.floor(65536 * p + 0.5)
    if t == 0:
        return None
    rows = torch.arange(n, device=device) if ids is None else ids.long()
    quads = torch.arange((d + 3) // 4, device=device)
    key = _mix(torch.tensor(seed, dtype=torch.int64, device=device))
    word = _mix(key ^ ((rows[:, None] << 32) | quads[None, :]))
    lanes = torch.stack([(word >> k) & 65535 for k in (0, 16, 32, 48)], dim=2).reshape(n, -1)[:, :d]
    return (lanes >= t).float() * (65536.0 / (65536 - t) if t < 65536 else 0.0)


def _plain_dropout(s):
    c, X = s["case"], s["X"]
    k = _keep_scale(s["seed"], s["ids"], c["n"], c["d"], c["p"], X.device)
    y = X.float() * k if k is not None else X.float()
    return (y + s["residual"].float() if s["residual"] is not None else y).to(X.dtype)


def _stats(s, dtype):
    """Mean and 1 / sqrt(variance + eps) of every set of channels: [n, groups, 2] or [M, groups, 2]."""
    c = s["case"]
    n, groups = c["n"], c["groups"]
    x = s["X"].to(dtype).view(n, groups, -1)
    if c["scope"] == "row":
        var, mean = torch.var_mean(x, dim=2, correction=0)
    else:
        both = [torch.var_mean(x[a:b], dim=(0, 2), correction=0) if b > a else (x.new_zeros(groups), x.new_zeros(groups))
                for a, b in zip(s["host"], s["host"][1:])]
        var, mean = torch.stack([v for v, _ in both]), torch.stack([m for _, m in both])
    return torch.stack([mean, torch.rsqrt(var + EPS)], dim=2)


def _of_part(s):
    """The part of every row."""
    h = s["host"]
    return torch.repeat_interleave(torch.arange(len(h) - 1, device="cuda"), torch.tensor([b - a for a, b in zip(h, h[1:])], device="cuda"),
                                   output_size=h[-1])


def _plain_norm(s):
    c = s["case"]
    X, n, C, groups = s["X"], c["n"], c["C"], c["groups"]
    part = _of_part(s)
    stats = _stats(s, torch.float32) if c["direction"] == "forward" else s["stats"]
    of = stats if c["scope"] == "row" else stats[part]
    xhat = (X.float().view(n, groups, -1) - of[:, :, :1]) * of[:, :, 1:]
    gamma = s["gamma"][part].view(n, groups, -1)
    u = xhat * gamma + s["beta"][part].view(n, groups, -1)
    keep = _keep_scale(s["seed"], None, n, C, c["p"], X.device)
    if c["direction"] == "forward":
        h = u
        if c["act"] == "relu":
            h = torch.clamp(u, min=0)
        elif c["act"] == "prelu":
            h = torch.where(u > 0, u, u * s["slope"][part][:, None, None])
        elif c["act"] == "silu":
            h = u / (1 + torch.exp(-u))
        h = h.view(n, C)
        return (h * keep if keep is not None else h).to(X.dtype), stats
    du = s["dY"].float()
    du = (du * keep if keep is not None else du).view(n, groups, -1)
    if c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-u))
        du = du * (sig * (1 + u * (1 - sig)))
    dgamma = torch.stack([t.sum(0) for t in _parts(s, (du * xhat).view(n, C))])
    dbeta = torch.stack([t.sum(0) for t in _parts(s, du.view(n, C))])
    t = du * gamma
    if c["scope"] == "row":
        s1, s2 = t.mean(2, keepdim=True), (t * xhat).mean(2, keepdim=True)
    else:
        size = torch.tensor([max(b - a, 1) * (C // groups) for a, b in zip(s["host"], s["host"][1:])], device="cuda")[:, None]
        s1 = ((dbeta * s["gamma"]).view(-1, groups, C // groups).sum(2) / size)[part][:, :, None]
        s2 = ((dgamma * s["gamma"]).view(-1, groups, C // groups).sum(2) / size)[part][:, :, None]
    dx = of[:, :, 1:] * (t - s1 - xhat * s2)
    return dx.view(n, C).to(X.dtype), dgamma, dbeta


# ---- work -----------------------------------------------------------------------------------------------


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    n = case["n"]
    if case["kind"] == "dropout":
        d = case["d"]
        return {"bytes": float(n) * d * size * (3 if case["residual"] else 2) + (4.0 * n if case["ids"] else 0.0), "flops": 2.0 * n * d}
    M = case["M"]
    if case["kind"] == "linear":
        d_in, d_out = case["d_in"], case["d_out"]
        weights = float(M) * (d_in + 1) * d_out * (4 if case["direction"] == "dw" else size)
        return {"bytes": float(n) * (d_in + d_out) * size + weights, "flops": 2.0 * n * d_in * d_out}
    C = case["C"]
    sets = (n if case["scope"] == "row" else M) * case["groups"]
    if case["direction"] == "forward":
        return {"bytes": 2.0 * n * C * size + 8.0 * sets + 8.0 * M * C, "flops": 10.0 * n * C}
    return {"bytes": 3.0 * n * C * size + 8.0 * sets + 16.0 * M * C, "flops": 20.0 * n * C}


# ---- the definitions in 64 bits -------------------------------------------------------------------------


def _exact_mask(seed, ids, n, d, p):
    """The mask times its scale in numpy's unsigned words, a block of rows at a time."""
    t = int(np.floor(np.float64(p) * 65536 + 0.5))
    golden, m1, m2 = np.uint64(0x9E3779B97F4A7C15), np.uint64(0xBF58476D1CE4E5B9), np.uint64(0x94D049BB133111EB)

    def step(z):
        z = z + golden
        z = (z ^ (z >> np.uint64(30))) * m1
        z = (z ^ (z >> np.uint64(27))) * m2
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        key = step(np.array([seed], dtype=np.uint64))[0]
        kept = np.empty((n, d), dtype=bool)
        for a in range(0, n, 1 << 17):
            b = min(n, a + (1 << 17))
            rows = (np.arange(a, b) if ids is None else ids[a:b]).astype(np.uint64)
            word = step(key ^ ((rows << np.uint64(32))[:, None] | np.arange((d + 3) // 4, dtype=np.uint64)[None, :]))
            lane = word.view(np.uint16).reshape(b - a, -1)[:, :d]  # little-endian: the lowest 16 bits come first
            kept[a:b] = lane >= t if t < 65536 else False
    return torch.from_numpy(kept).cuda(), 65536.0 / (65536 - t) if t < 65536 else 0.0


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["kind"] == "dropout":
        if case["n"] * case["d"] > 700_000_000:
            return None
        kept, scale = _exact_mask(s["seed"], None if s["ids"] is None else s["ids"].cpu().numpy(), case["n"], case["d"], case["p"])
        y = torch.where(kept, s["X"].to(f64) * scale, 0.0)
        return y if s["residual"] is None else y + s["residual"].to(f64)
    if case["kind"] == "linear":
        outs = []
        for a, b, g in zip(s["host"], s["host"][1:], range(case["M"])):
            if case["direction"] == "forward":
                outs.append(torch.einsum("ri,io->ro", s["X"][a:b].to(f64), s["W"][g].to(f64)) + s["b"][g].to(f64))
            elif case["direction"] == "dx":
                outs.append(torch.einsum("ro,io->ri", s["dY"][a:b].to(f64), s["W"][g].to(f64)))
            else:
                ones = torch.ones(b - a, dtype=f64, device="cuda")
                dy = s["dY"][a:b].to(f64)
                outs.append((torch.einsum("ri,ro->io", s["X"][a:b].to(f64), dy), torch.einsum("r,ro->o", ones, dy)))
        if case["direction"] == "dw":
            return torch.stack([o[0] for o in outs]), torch.stack([o[1] for o in outs])
        return torch.cat(outs)
    C, groups = case["C"], case["groups"]
    kept = None
    if case["p"] > 0:
        kept, scale = _exact_mask(s["seed"], None, case["n"], C, case["p"])
    outs, stats, dgamma, dbeta = [], [], [], []
    for a, b, g in zip(s["host"], s["host"][1:], range(case["M"])):
        x = s["X"][a:b].to(f64).reshape(b - a, groups, C // groups)
        over = (2,) if case["scope"] == "row" else (0, 2)
        if b > a:
            mean = x.mean(dim=over, keepdim=True)
            rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(dim=over, keepdim=True) + EPS)
        else:
            mean = x.new_zeros(1 if case["scope"] == "part" else 0, groups, 1)
            rstd = mean + 1.0 / math.sqrt(EPS)
        stats.append(torch.stack([mean.reshape(-1, groups), rstd.reshape(-1, groups)], dim=2))
        if case["direction"] == "grad":  # from the statistics that the pass is given
            given = s["stats"][a:b] if case["scope"] == "row" else s["stats"][g:g + 1]
            mean, rstd = given[:, :, :1].to(f64), given[:, :, 1:].to(f64)
        ga, be = s["gamma"][g].to(f64).view(groups, -1), s["beta"][g].to(f64).view(groups, -1)
        xh = (x - mean) * rstd
        u = ga * xh + be
        sig = torch.sigmoid(u)
        if case["direction"] == "forward":
            slope = SLOPE if case["act"] == "prelu" else 0.0
            h = {"none": lambda: u, "silu": lambda: u * sig}.get(case["act"], lambda: u.clamp(min=0) + slope * u.clamp(max=0))()
            h = h.reshape(b - a, C)
            outs.append(torch.where(kept[a:b], h * scale, 0.0) if kept is not None else h)
            continue
        dh = s["dY"][a:b].to(f64)
        if kept is not None:
            dh = torch.where(kept[a:b], dh * scale, 0.0)
        du = dh.reshape(x.shape) * (sig + u * sig * (1 - sig) if case["act"] == "silu" else 1.0)
        dgamma.append((du * xh).sum(0).reshape(-1))
        dbeta.append(du.sum(0).reshape(-1))
        t = du * ga
        count = (C // groups) * (1 if case["scope"] == "row" else max(b - a, 1))
        first, second = t.sum(dim=over, keepdim=True) / count, (t * xh).sum(dim=over, keepdim=True) / count
        outs.append((rstd * (t - first - xh * second)).reshape(b - a, C))
    if case["direction"] == "forward":
        return torch.cat(outs), torch.cat(stats)
    return torch.cat(outs), torch.stack(dgamma), torch.stack(dbeta)
