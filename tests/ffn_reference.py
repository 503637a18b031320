"""The operators around a feed-forward block in binary64 on the host, from their formulas: what the device's results are held to.
Nothing here is shared with the package or the oracle."""
import math

import numpy as np
import torch

QMAX = {0: 127.0, 1: 448.0, 2: 57344.0}            # by the library's format numbers: INT8, E4M3, E5M2
EPS32 = 2.0 ** -24                                  # a binary32 rounding, relative


def rounding(dtype):
    """A rounding to `dtype`, relative to the value."""
    return torch.finfo(dtype).eps / 2


def norm(x, residual, weight, eps):
    """h (rounded to x's type), y and 1 / rms of the rows of x."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype) if x.dtype != torch.float64 else x + residual
    v = h.double()
    rstd = 1.0 / torch.sqrt((v * v).mean(-1) + eps)
    w = torch.ones(v.shape[-1], dtype=torch.float64) if weight is None else weight.double()
    return h, v * rstd.unsqueeze(-1) * w, rstd


def norm_grad(dy, h, rstd, weight, dresidual):
    """dx, dw and the sums of magnitudes that the errors of both are relative to."""
    w = torch.ones(h.shape[-1], dtype=torch.float64) if weight is None else weight.double()
    r = rstd.double().reshape(*h.shape[:-1], 1)
    n, a = h.double() * r, dy.double() * w
    dx = r * (a - n * (a * n).mean(-1, keepdim=True))
    size = r * (a.abs() + n.abs() * (a * n).abs().mean(-1, keepdim=True))
    if dresidual is not None:
        dx, size = dx + dresidual.double(), size + dresidual.double().abs()
    flat = (dy.double() * n).reshape(-1, h.shape[-1])
    return dx, flat.sum(0), size, flat.abs().sum(0)


def phi(g):
    return 0.5 * torch.special.erfc(-g / math.sqrt(2.0))


def act(g, kind):
    """act(g) and its slope; kind 0 is SiLU, 1 is GELU."""
    if kind == 0:
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    return g * phi(g), phi(g) + g * torch.exp(-g * g / 2) / math.sqrt(2.0 * math.pi)


def grid_error(values, t, fmt):
    """How far code values are from t, in units of the most that rounding to nearest may be off there (t within the format's range)."""
    half = {0: torch.full_like(t, 0.5), 1: t.abs().clamp_min(2.0 ** -6) * 2.0 ** -4, 2: t.abs().clamp_min(2.0 ** -14) * 2.0 ** -3}[fmt]
    return (values - t).abs() / half


def decode(codes, fmt):
    c = codes.cpu()
    return (c.view(torch.int8) if fmt == 0 else c.view(torch.float8_e4m3fn if fmt == 1 else torch.float8_e5m2)).double()


def check_codes(codes, delta, y, fmt, rel):
    """codes and delta of the rows of y (binary64), which the device has to `rel` (relative): the step size to that and the division's
    rounding, every code the nearest one to its quotient up to that."""
    d = delta.cpu().double()
    rows = y.reshape(-1, y.shape[-1])
    want = rows.abs().amax(-1) / QMAX[fmt]
    want = torch.where(want == 0, torch.ones_like(want), want.clamp_min(2.0 ** -126))
    assert torch.all((d - want).abs() <= (rel + 2 * EPS32) * want)
    t = rows / d.unsqueeze(-1)
    # the quotient is a product with a rounded reciprocal: two more roundings; above the largest value it is cut off
    off = grid_error(decode(codes, fmt).reshape(rows.shape), t.clamp(-QMAX[fmt], QMAX[fmt]), fmt)
    slack = 1.0 + (rel + 4 * EPS32) * (t.abs() / 0.5 if fmt == 0 else 2.0 ** (4 if fmt == 1 else 3)) + 1e-12
    assert torch.all(off <= slack), (off - slack).max()


def same_bits(a, b):
    a, b = a.cpu(), b.cpu()
    return a.dtype == b.dtype and a.shape == b.shape and np.array_equal(a.contiguous().view(torch.uint8).numpy(), b.contiguous().view(torch.uint8).numpy())
