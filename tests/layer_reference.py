"""Plain 64-bit forms of whole layers on the rows of many parts, with bounds of what fp32 sums and roundings can be off."""
import torch

F64 = torch.float64


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounding(y, dtype):
    """Half a step of every value (the smallest step of the type for tiny ones)."""
    return half_step(dtype) * y.abs() * 1.001 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def sum_error(terms, dtype):
    """What a sum of so many products is off, as a share of the sum of their magnitudes.  16-bit rows: exact products, added 16 at a time
    in an accumulator that truncates (2^-23 for every addition, two for what joins).  fp32 rows: below 2^-22 of a product is left out, the
    twelve additions of 32 terms truncate, the sums of 32 terms are rounded."""
    if dtype == torch.float32:
        return 2.0**-22 + 12 * 2.0**-23 + (terms / 32 + 3) * 2.0**-24
    return (terms / 16 + 3) * 2.0**-23


def activation(z, act, slope):
    """(act(z), act'(z), act''(z) as a bound of its size) in 64 bits."""
    if act == "none":
        return z, torch.ones_like(z), torch.zeros_like(z)
    if act == "silu":
        s = torch.sigmoid(z)
        d = s * (1 + z * (1 - s))
        return z * s, d, torch.full_like(z, 0.5)
    k = slope if act == "prelu" else torch.zeros((), dtype=F64, device=z.device)
    return torch.where(z > 0, z, k * z), torch.where(z > 0, torch.ones_like(z), k + torch.zeros_like(z)), torch.zeros_like(z)


class Layer:
    """One part's rows through the layer and back; every attribute with an _off beside it is a value and how far a kernel's may be from
    it.  x, w, b, dy, residual as the kernel reads them; slope: a number; dtype: the rows' type."""

    def __init__(self, x, w, b, act, slope, gated, dtype, residual=None, dy=None):
        x, w = x.to(F64), w.to(F64)
        k = x.shape[1]
        z = x @ w
        size = x.abs() @ w.abs()
        if b is not None:
            z, size = z + b.to(F64), size + b.to(F64).abs()
        off = sum_error(k, dtype) * size + 2.0**-23 * size
        f = w.shape[1] // 2 if gated else w.shape[1]
        slope = torch.tensor(float(slope), dtype=F64, device=x.device)
        front, front_off = z[:, :f], off[:, :f]
        a, d1, d2 = activation(front, act, slope)
        # the exponential and the reciprocal are good to (2 + |z|) 2^-22; a kink within reach of the error lets either side be taken
        near = ((2 + front.abs()) * 2.0**-22) if act == "silu" else torch.zeros_like(front)
        reach = torch.maximum(d1.abs(), torch.ones_like(d1)) * 1.1
        a_off = reach * front_off + near * a.abs() + 2.0**-23 * a.abs()
        d1_off = d2 * front_off + 3 * near + 2.0**-22
        if act in ("relu", "prelu"):
            d1_off = torch.where(front.abs() <= front_off, (1 - slope if act == "prelu" else torch.ones_like(slope)).abs(), 2.0**-23 * torch.ones_like(front))
        if act == "none":
            d1_off = torch.zeros_like(front)
        u = z[:, f:] if gated else torch.ones_like(front)
        u_off = off[:, f:] if gated else torch.zeros_like(front)
        y = a * u
        y_off = a_off * (u.abs() + u_off) + a.abs() * u_off + 2.0**-23 * y.abs()
        if residual is not None:
            y = y + residual.to(F64)
            y_off = y_off + 2.0**-23 * (y.abs() + y_off)
        self.y, self.y_off = y, y_off + rounding(y.abs() + y_off, dtype)
        if dy is None:
            return
        dy = dy.to(F64)
        dfront = dy * u * d1
        dfront_off = dy.abs() * (u_off * (d1.abs() + d1_off) + u.abs() * d1_off) + 2.0**-22 * dfront.abs()
        if gated:
            dz = torch.cat([dfront, dy * a], 1)
            dz_off = torch.cat([dfront_off, dy.abs() * a_off + 2.0**-23 * (dy * a).abs()], 1)
        else:
            dz, dz_off = dfront, dfront_off
        if not (act == "none" and not gated):
            dz_off = dz_off + rounding(dz.abs() + dz_off, dtype)
        self.dz, self.dz_off = dz, dz_off
        whole = dz.abs() + dz_off
        self.dx = dz @ w.T
        self.dx_off = dz_off @ w.abs().T + sum_error(dz.shape[1], dtype) * (whole @ w.abs().T)
        self.dx_off = self.dx_off + rounding(self.dx.abs() + self.dx_off, dtype)
        # sums over rows: a truncating accumulator of 128 rows at most (fp32: 32), then joined with rounding
        rows = x.shape[0]
        share = sum_error(128, dtype) + (rows / 32 + 40) * 2.0**-24
        self.dw = x.T @ dz
        # What the other side of the kink would change: where |Z| is below its own error the kernel's Z may have the other sign, its derivative is
        # then the other side's, and the entry of dZ is off by |dY U (1 - slope)| whole, which no rounding bounds.
        kink = (front.abs() <= front_off) & (act in ("relu", "prelu"))
        self.dw_kink = (x.abs().T @ torch.where(kink, (dy * u).abs() * (1 - (slope if act == "prelu" else 0.0)), torch.zeros_like(front))).norm().item()
        self.dw_off = x.abs().T @ dz_off + share * (x.abs().T @ whole)
        self.db = dz.sum(0)
        self.db_off = dz_off.sum(0) + share * whole.sum(0)
        low = torch.clamp(front, max=0)
        self.dslope = (dy * u * low).sum()
        self.dslope_off = (dy.abs() * ((u.abs() + u_off) * front_off + u_off * low.abs())).sum() + (rows / 32 + 200) * 2.0**-24 * (dy * u * low).abs().sum()
