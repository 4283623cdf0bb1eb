"""The head's operators in 64 bits, written from their formulas, and how far 32-bit and 16-bit arithmetic may end from
them.  Used by the tests of gosh_linear, gosh_layer_norm and the 8-bit form."""
from __future__ import annotations

import math

import torch

F32 = 2.0 ** -24  # half a unit in the last place, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}  # rounding below the normal range
TYPES = (torch.float32, torch.bfloat16, torch.float16)
NONE, RELU, GELU, SILU = range(4)


def act(z, kind):
    if kind == RELU:
        return z.clamp(min=0)
    if kind == GELU:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if kind == SILU:
        return z * torch.sigmoid(z)
    return z


def slope(z, kind):
    if kind == RELU:
        return (z > 0).to(z.dtype)
    if kind == GELU:
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if kind == SILU:
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def linear(x, w, b, kind, r):
    """(y, z, bound of y's error in 32 bits, bound of z's).

    A sum of k products in 32 bits is off by at most (k + 8) 2^-24 of the sum of magnitudes, the 8 for the bias and for
    products that are themselves rounded.  No activation's slope exceeds 1.13; its own evaluation (an exponential whose
    argument is rounded, a reciprocal) is off by less than 2^-20 (1 + |z|); the residual's sum is rounded once."""
    z = x @ w.t() + (0 if b is None else b)
    dz = (x.shape[1] + 8) * F32 * (x.abs() @ w.abs().t() + (0 if b is None else b.abs()))
    y = act(z, kind)
    dy = 1.13 * dz + (0 if kind in (NONE, RELU) else 2.0 ** -20 * (1 + z.abs()))
    if r is not None:
        y = y + r
        dy = dy + F32 * y.abs()
    return y, z, dy, dz


def linear_backward(dy, x, w, z, kind, dtype):
    """(dx, dw, db) and bounds of their errors before they are rounded to their type: dz is rounded to `dtype` (not where
    the activation is none or only passes or drops dy, nor in db), its slope is off by at most 2^-19."""
    dz = dy * slope(z, kind) if kind != NONE else dy
    off = dy.abs() * (2.0 ** -19 if kind in (GELU, SILU) else 0)
    off16 = off + HALF[dtype] * dz.abs() * (1 if kind in (GELU, SILU) else 0) + TINY[dtype] * (kind != NONE)
    n, rows = dy.shape[1], dy.shape[0]
    dx = dz @ w
    ex = off16 @ w.abs() + (n + 8) * F32 * (dz.abs() @ w.abs())
    dw = dz.t() @ x
    ew = off16.t() @ x.abs() + (rows + 8) * F32 * (dz.abs().t() @ x.abs())
    db = dz.sum(dim=0)
    eb = off.sum(dim=0) + (rows + 8) * F32 * dz.abs().sum(dim=0)
    return (dx, dw, db), (ex, ew, eb)


def norm(x, gamma, beta, eps):
    """(y, mean, rstd, xhat) and bounds of the errors in 32 bits.

    The mean is off by at most k 2^-24 of the mean magnitude; what that and the rounding of x - mean do to xhat is that
    times rstd; rstd's relative error is at most (k / 2 + 4) 2^-24, plus twice the mean's effect on the centred rows
    (second order in the variance, first order here to be safe)."""
    k = x.shape[1]
    mean = x.mean(dim=1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(dim=1, keepdim=True) + eps)
    xhat = (x - mean) * rstd
    emean = k * F32 * x.abs().mean(dim=1, keepdim=True)
    rel = (k / 2 + 4) * F32 + 2 * emean * rstd
    exhat = (emean + F32 * (x.abs() + mean.abs())) * rstd + xhat.abs() * (rel + 2 * F32)
    y = xhat * gamma + beta
    ey = exhat * gamma.abs() + 2 * F32 * (xhat * gamma).abs() + F32 * y.abs()
    return (y, mean[:, 0], rstd[:, 0], xhat), (ey, emean[:, 0], rstd[:, 0] * rel[:, 0], exhat)


def norm_backward(dy, xhat, gamma, rstd, add, exhat):
    """(dx, dgamma, dbeta) and bounds: exhat is how far the xhat of the pass may be off."""
    rows, k = dy.shape
    g = dy * gamma
    m0, m1 = g.mean(dim=1, keepdim=True), (g * xhat).mean(dim=1, keepdim=True)
    r = rstd[:, None]
    dx = r * (g - m0 - xhat * m1)
    e0 = (k + 2) * F32 * g.abs().mean(dim=1, keepdim=True)
    e1 = (k + 3) * F32 * (g * xhat).abs().mean(dim=1, keepdim=True) + (g.abs() * exhat).mean(dim=1, keepdim=True)
    ex = r.abs() * (e0 + xhat.abs() * e1 + exhat * (m1.abs() + e1) + 6 * F32 * (g.abs() + m0.abs() + (xhat * m1).abs()))
    if add is not None:
        dx = dx + add
        ex = ex + F32 * (dx.abs() + add.abs())
    dgamma = (dy * xhat).sum(dim=0)
    eg = (dy.abs() * exhat).sum(dim=0) + (rows + 4) * F32 * (dy * xhat).abs().sum(dim=0)
    dbeta = dy.sum(dim=0)
    eb = (rows + 4) * F32 * dy.abs().sum(dim=0)
    return (dx, dgamma, dbeta), (ex, eg, eb)


def rounded(bound, want, dtype):
    """The bound of an output that is rounded to `dtype` once."""
    return bound + (HALF[dtype] * (want.abs() + bound) if dtype != torch.float32 else F32 * want.abs()) + TINY[dtype]


def eight_bits(x, dtype):
    """(q, exponent byte) of the 8-bit form, entry by entry as it is defined; x in 64 bits, of values of `dtype`."""
    rows, k = x.shape
    q = torch.zeros(rows, k, dtype=torch.int64)
    exps = torch.zeros(rows, -(-k // 32), dtype=torch.int64)
    low = -24 if dtype == torch.float16 else -126
    largest = torch.finfo(dtype).max
    for r in range(rows):
        for g in range(exps.shape[1]):
            part = x[r, 32 * g:32 * g + 32]
            if not torch.isfinite(part).all():
                exps[r, g] = 255
                continue
            most = float(part.abs().max())
            e = low
            while most > 127 * 2.0 ** e:
                e += 1
            v = torch.round(part / 2.0 ** e)  # ties to even
            if 64 * 2.0 ** e > largest:
                v = v.clamp(-63, 63)
            q[r, 32 * g:32 * g + 32] = v.to(torch.int64)
            exps[r, g] = e + 127
    return q, exps


def values(q, exps):
    """What an 8-bit form stands for, in 64 bits."""
    e = exps.to(torch.float64).repeat_interleave(32, dim=1)[:, :q.shape[1]]
    return torch.where(e == 255, torch.full_like(e, math.nan), q.to(torch.float64) * 2.0 ** (e - 127))


def group_most(x):
    """The largest magnitude of each entry's group."""
    pad = -x.shape[1] % 32
    most = torch.nn.functional.pad(x.abs(), (0, pad)).reshape(x.shape[0], -1, 32).amax(dim=2)
    return most.repeat_interleave(32, dim=1)[:, :x.shape[1]]
