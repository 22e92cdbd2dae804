"""Plain 64-bit forms of the operators beside the step, and the error bounds that follow from their roundings."""
import numpy as np
import torch

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U32 = 2.0 ** -24
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}          # half a unit of the last place, relative
LEAST = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}      # smallest positive values


def rounded(bound, value, dtype):
    """Bound of a value that is within `bound` of `value` and then rounded to dtype."""
    if dtype == F32:
        return bound
    return bound + (value.abs() + bound) * UNIT[dtype] + LEAST[dtype]


def close(got, want, bound, what=""):
    """|got - want| <= bound for every element, in 64 bits."""
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.cpu()
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of a bound %.3g, at %d" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound[bad].max()), int(bad.flatten().nonzero()[0]))


def adamw64(x, g, m, v, step, lr, decay, c=1.0, beta1=0.9, beta2=0.999, eps=1e-8):
    """AdamW by its definition in 64 bits: (x, m, v) and the bounds of their fp32 evaluation."""
    x, g, m, v = x.double(), g.double() * c, m.double(), v.double()
    am = beta1 * m.abs() + (1 - beta1) * g.abs()
    m2, v2 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    # m: rounded are the constant, c g, the product, the sum; v: the constant, c g twice, its square, the product, the sum
    tm, tv = 5 * U32 * am, 6 * U32 * v2
    den = torch.sqrt(v2) / (1 - beta2 ** step) ** 0.5 + eps
    lr1 = lr / (1 - beta1 ** step)
    update = lr1 * m2 / den
    # den: half of v's, the root, the constant, the product, the sum (and eps): 7; lr, the constant, the product, the quotient: 4
    tu = lr1 * tm / den + update.abs() * 11 * U32
    kept = x - lr * decay * x
    x2 = kept - update
    tx = tu + U32 * (2 * kept.abs() + x2.abs()) + 4 * U32 * (lr * decay * x).abs()
    tiny = 8 * LEAST[F32]           # products of subnormals
    return x2, m2, v2, tx * 1.001 + tiny, tm * 1.001 + tiny, tv * 1.001 + tiny


def adamw32(x, g, m, v, step, lr, decay, c=None, beta1=0.9, beta2=0.999, eps=1e-8):
    """The same in fp32 on the CPU, one rounding per operation in the order of the header: (x, m, v, sqrt(v))."""
    f = lambda a: torch.tensor(a, dtype=F32)  # noqa: E731
    x, g, m, v = x.float().cpu(), g.float().cpu(), m.cpu(), v.cpu()
    if c is not None:
        g = g * c.cpu()
    m = m * f(beta1) + g * f(1 - beta1)
    v = v * f(beta2) + (g * g) * f(1 - beta2)
    r = torch.from_numpy(np.sqrt(v.numpy()))        # correctly rounded, which torch.sqrt is not
    lr32 = float(f(lr))
    x = x - x * (f(lr) * f(decay))
    x = x - (m * f(lr32 / (1 - beta1 ** step))) / (r * f(1 / (1 - beta2 ** step) ** 0.5) + f(eps))
    return x, m, v, r


def fp8_blocks(x, positive, block=256):
    """Blocks of a vector as (8-bit floats, scales), by the header's formula in fp32."""
    n = x.numel()
    y = torch.zeros(-(-n // block) * block)
    y[:n] = x
    y = y.view(-1, block)
    big = y.abs().amax(1, keepdim=True)
    big = torch.where(big < 2.0 ** -116, torch.zeros_like(big), big)
    q = y * torch.where(big > 0, (torch.ones_like(big) / big) * 448, torch.zeros_like(big))
    if positive:
        q = torch.where((y > 0) & (big > 0), q.clamp_min(2.0 ** -9), q)
    return q.to(torch.float8_e4m3fn).view(-1)[:n], (big * (torch.ones(1) / 448)).view(-1)


def embedding_grad64(tokens, dout, rows, scale, padding=None):
    """(gradient, bound of its fp32 evaluation) in 64 bits."""
    tok = tokens.reshape(-1).long().cpu()
    x = dout.reshape(tok.numel(), -1).double().cpu() * scale
    keep = (tok >= 0) & (tok < rows)
    if padding is not None:
        keep &= tok != padding
    g, a = (torch.zeros(rows, x.shape[1], dtype=torch.float64) for _ in range(2))
    g.index_add_(0, tok[keep], x[keep])
    a.index_add_(0, tok[keep], x[keep].abs())
    n = torch.zeros(rows, dtype=torch.float64).index_add_(0, tok[keep], torch.ones(int(keep.sum()), dtype=torch.float64))
    # a sum of n in any order: n - 1 roundings, the scale, the product
    return g, a * ((n + 2) * U32)[:, None] * 1.001 + 4 * LEAST[F32]
