"""Plain 64-bit forms of layer norm, the product in 8-bit integers and sampling, and the error bounds that follow from their roundings."""
import numpy as np
import torch

from operator_util import F32, U32


def depth(dim):
    """Roundings that a value goes through in a sum over a row, at most: a lane's elements one after the other (32 where a row stays in
    registers, else dim / 1024 in runs of 8), 6 between lanes, 16 between wavefronts."""
    return (32 if dim <= 8192 else dim // 1024 + 8) + 22


def rows_depth(rows, dim):
    """... in a sum over rows: those of one wavefront, four wavefronts; the workgroups' sums are added in fp64."""
    partials = min(512 if dim <= 2048 else 256, max(8, (1 << 21) // dim))
    return -(-rows // partials) + 4


def layer_norm64(x, w, b, eps):
    """(out, mean, rstd) and their bounds before a rounding to the output's type."""
    x = x.double().cpu()
    n = x.shape[1]
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double().cpu()
    b = torch.zeros(n, dtype=torch.float64) if b is None else b.double().cpu()
    eps = float(torch.tensor(eps, dtype=F32))
    mean = x.mean(1, keepdim=True)
    c = x - mean
    var = (c * c).mean(1, keepdim=True)
    r = 1 / (var + eps).sqrt()
    D = depth(n)
    # the sum, 1 / n and its product
    tm = (D + 3) * U32 * x.abs().mean(1, keepdim=True)
    tc = U32 * c.abs() + tm
    # squares of what is off by tc, their rounding, the sum, 1 / n and its product
    tv = (2 * c.abs() * tc + tc * tc).mean(1, keepdim=True) + (D + 4) * U32 * ((c.abs() + tc) ** 2).mean(1, keepdim=True)
    # eps' sum, the root, the quotient: a rounding each, at most one unit for the root and the quotient
    hi, lo = 1 / ((var - tv).clamp_min(0) + eps).sqrt(), 1 / (var + tv + eps).sqrt()
    tr = torch.maximum(hi - r, r - lo) + 6 * U32 * hi
    y = c * r * w + b
    ty = w.abs() * (tc * (r + tr) + c.abs() * tr + 2 * U32 * (c.abs() + tc) * (r + tr)) * 1.001
    ty = ty + U32 * (y.abs() + ty)
    return y, mean[:, 0], r[:, 0], ty * 1.001 + 1e-44, tm[:, 0] * 1.001 + 1e-44, tr[:, 0] * 1.001


def layer_norm_grad64(dout, x, w, mean, rstd, dw0=None, db0=None):
    """(dx, dweight, dbias) from the given mean and rstd, and their bounds before a rounding to the outputs' types."""
    dy, x, m, r = dout.double().cpu(), x.double().cpu(), mean.double().cpu()[:, None], rstd.double().cpu()[:, None]
    rows, n = x.shape
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double().cpu()
    D, R = depth(n), rows_depth(rows, n)
    xh = (x - m) * r
    g = dy * w
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - c1 - xh * c2)
    # g is rounded, xh twice; the sum, 1 / n and its product
    t1 = (D + 3) * U32 * g.abs().mean(1, keepdim=True)
    t2 = (D + 6) * U32 * (g * xh).abs().mean(1, keepdim=True)
    # g, xh twice, xh c2, two differences, the product with rstd
    tx = r * (t1 + xh.abs() * t2 + 6 * U32 * (g.abs() + c1.abs() + (xh * c2).abs()))
    dw, db = (dy * xh).sum(0), dy.sum(0)
    tw, tb = (R + 4) * U32 * (dy * xh).abs().sum(0), R * U32 * dy.abs().sum(0)
    if dw0 is not None:
        dw, db = dw + dw0.double().cpu(), db + db0.double().cpu()
    # the fp64 sum becomes fp32
    tw, tb = tw + U32 * (dw.abs() + tw), tb + U32 * (db.abs() + tb)
    return dx, dw, db, tx * 1.001 + 1e-44, tw * 1.001 + 1e-44, tb * 1.001 + 1e-44


def token_codes(x):
    """(integers, scales) of tokens by the header's operations in fp32, on the CPU."""
    x = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        a = np.abs(x).max(1)
        finite, zero = np.isfinite(a), a < np.float32(2.0 ** -116)
        inverse = np.where(finite & ~zero, (np.float32(1) / np.where(finite & ~zero, a, 1)).astype(np.float32) * np.float32(127), np.float32(0))
        codes = np.where((inverse != 0)[:, None], np.rint((x * inverse[:, None]).astype(np.float32)), 0)
        scale = np.where(~finite, np.float32(np.nan), np.where(zero, np.float32(0), a * (np.float32(1) / np.float32(127))))
    return torch.from_numpy(np.where(np.isfinite(codes), codes, 0).astype(np.int8)), torch.from_numpy(scale.astype(np.float32))


def linear8(codes, scales, weight, unit, bias, dtype):
    """The product by the header's operations in fp32, on the CPU: exact sums, then one rounding per operation."""
    sums = codes.double().cpu().numpy() @ weight.double().cpu().numpy().T         # whole numbers below 2^31: exact
    with np.errstate(all="ignore"):
        y = sums.astype(np.float32) * scales.cpu().numpy()[:, None]
        y = y * (unit.cpu().numpy()[None, :] if isinstance(unit, torch.Tensor) else np.float32(unit))
        if bias is not None:
            y = y + bias.float().cpu().numpy()[None, :]
    return torch.from_numpy(y).to(dtype)


def sample(logits, u, temperature, top_k, top_p, min_p):
    """The token of one row by the header's definition; -1 where there is none.  Masses are integers."""
    x = logits.float().cpu().numpy()
    f32 = lambda v: float(np.float32(v))  # noqa: E731
    temperature, top_p, min_p = f32(temperature), f32(top_p), f32(min_p)
    if np.isnan(x).any() or not (0 <= temperature < np.inf) or x.max() == -np.inf:
        return -1
    x = np.minimum(x, np.finfo(np.float32).max)
    order = np.argsort(-x, kind="stable")
    if temperature == 0:
        return int(order[0])
    y = x[order].astype(np.float64)
    with np.errstate(over="ignore"):
        mass = np.rint(np.exp((y - y[0]) / temperature) * 2.0 ** 40).astype(np.uint64)
    if 0 < top_k < mass.size:
        mass = mass[:top_k]
    run = np.cumsum(mass)
    end = mass.size
    if top_p < 1:
        end = 1 + int(np.argmax(run.astype(np.float64) >= max(top_p, 0.0) * float(run[-1])))
    if min_p > 0:
        end = min(end, int((mass.astype(np.float64) >= min(min_p, 1.0) * 2.0 ** 40).sum()))
    u = f32(u)
    u = 0.0 if not u > 0 else min(u, float(np.nextafter(np.float32(1), np.float32(0))))
    return int(order[int(np.argmax(run[:end].astype(np.float64) > u * float(run[end - 1])))])
