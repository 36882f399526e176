"""The dense side's operators in 64 bits, for tests: AdamW, packed moments, layer norm of rows."""
import torch

BLOCK = 128
HALF32 = 2.0 ** -24                      # half a step of fp32, relative to the value


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def padded(n):
    return -(-n // BLOCK) * BLOCK


def adamw(p, g, m, v, t, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, factor=1.0):
    """One step in float64 (t: its number).  Returns p, m, v and how far fp32 arithmetic may be off
    in each, counting half a step for every constant, product, sum, root and quotient."""
    p, g, m, v = (x.double() for x in (p, g, m, v))
    g = factor * g
    a, b = beta1 * m, (1 - beta1) * g
    c, d = beta2 * v, (1 - beta2) * g * g
    m1, v1 = a + b, c + d
    tol_m = HALF32 * (3 * a.abs() + 4 * b.abs()) + 1e-44
    tol_v = HALF32 * (3 * c + 7 * d) + 1e-44
    size = lr / (1 - beta1 ** t)
    den = (v1 / (1 - beta2 ** t)).sqrt() + eps
    up = size * m1 / den
    p1 = p * (1 - lr * weight_decay) - up
    # v1 is a sum of two terms >= 0: its relative error, halved by the root, is among the 16
    tol_p = HALF32 * (4 * p.abs() + 16 * up.abs()) + size / den * tol_m + 1e-44
    return p1, m1, v1, tol_p, tol_m, tol_v


def decode(code, exps, top, signed):
    """Values (float64) of codes of whole blocks; exps: one byte per block."""
    c = code.double().view(-1, BLOCK)
    sign = torch.ones_like(c)
    if signed:
        sign = torch.where(c >= 128, -1.0, 1.0).double()
        c = c % 128
    field = torch.floor(c / 8)
    mant = c - 8 * field
    two = torch.tensor(2.0, dtype=torch.float64)
    value = torch.where(field > 0, (1 + mant / 8) * two ** (field - 127), mant / 8 * two ** -126.0)
    return (sign * value * (two ** (exps.double() - top))[:, None]).view(-1)


def dither(first, n, t, turn):
    h = t * 0x9E3779B9 % 2 ** 32
    h = (h ^ h >> 15) * 0x6A09E667 % 2 ** 32
    h = (h ^ h >> 13) * 0x9E3779B9 % 2 ** 32
    h ^= h >> 16
    i = torch.arange(first, first + n, dtype=torch.int64)
    return ((i * 0x6A09E667 + h + turn) % (1 << 32) // 4096).double() / (1 << 20)


def exponents(x, top):
    """The exponent fields that whole blocks of x >= 0 (float64) go by."""
    most = x.view(-1, BLOCK).amax(1)
    return torch.where(most > 0, torch.frexp(most)[1] + 126, 0).clamp(min=top)


def encode(x, e, top, t, turn, first):
    """Codes without sign of x >= 0 (float64, whole blocks, element `first` of the arrays on) under
    their blocks' exponents e, and the place between two codes: position + dither, whose floor
    decides."""
    b = x.view(-1, BLOCK)
    two = torch.tensor(2.0, dtype=torch.float64)
    y = b / (two ** (e - top).double())[:, None]
    field = torch.where(y > 0, torch.frexp(y)[1] + 126, 1).clamp(min=1)
    place = y / two ** (field - 130).double()              # 8 .. 16, below 8 in the lowest field
    total = place + dither(first, x.numel(), t, turn).view_as(y)
    code = torch.floor(total) + 8 * (field - 1)
    return code.view(-1).long(), total.view(-1)


def layernorm(x, gamma, beta, eps):
    x = x.double()
    mu = x.mean(1, keepdim=True)
    rstd = 1 / ((x - mu).square().mean(1, keepdim=True) + eps).sqrt()
    return (x - mu) * rstd * gamma.double() + beta.double(), mu[:, 0], rstd[:, 0]


def layernorm_backward(dy, x, gamma, eps):
    x, dy = x.double(), dy.double()
    mu = x.mean(1, keepdim=True)
    rstd = 1 / ((x - mu).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (x - mu) * rstd
    g = dy * gamma.double()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), xh, rstd[:, 0]
