"""Matrices in 8-bit floating point, AdamW with its 8-bit moments and the softmax loss in 64 bits, written from their
definitions, and how far 32-bit arithmetic may end from them.  Used by the tests of gosh_pack_fp8, gosh_linear_fp8,
gosh_adamw_step and gosh_softmax_loss."""
from __future__ import annotations

import bisect
import math

import torch

from tests import head_model as H

F32 = H.F32
NUMBERS = [(e and 1) * 2.0 ** (e - 7) * (1 + m / 8) or 2.0 ** -6 * m / 8 for e in range(16) for m in range(8)][:127]  # e4m3


def _by_blocks(x, tall):
    """(row blocks, rows of a block, column blocks, 128) with zeros past the ends."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x, (0, -k % 128, 0, -rows % tall))
    return x.reshape(x.shape[0] // tall, tall, -1, 128)


def two(e):
    """2^e by its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def fp8(x, tall):
    """(bytes with columns padded to 128, exponent bytes, values) of x in 64 bits."""
    rows, k = x.shape
    b = _by_blocks(x, tall)
    fine = torch.isfinite(b)
    most = torch.where(fine, b.abs(), torch.zeros_like(b)).amax(dim=(1, 3), keepdim=True)
    e = torch.full_like(most, -126.0)
    for power in range(-126, 120):
        e = torch.where(most > 448 * 2.0 ** power, torch.full_like(e, power + 1.0), e)
    unit = two(e)
    v = torch.where(fine, b, torch.zeros_like(b)) / unit
    table = torch.tensor(NUMBERS, dtype=torch.float64, device=x.device)
    low = torch.clamp(torch.searchsorted(table, v.abs().contiguous(), right=True) - 1, max=125)
    down, up = v.abs() - table[low], table[low + 1] - v.abs()
    code = low + ((down > up) | ((down == up) & (low % 2 == 1))).long()
    value = torch.where(fine, torch.sign(v) * table[code] * unit, torch.full_like(b, math.nan))
    code = torch.where(fine, code, torch.full_like(code, 127)) + 128 * torch.signbit(b).long()
    flat = lambda t: t.reshape(-1, t.shape[2] * 128)[:rows]  # noqa: E731
    return flat(code), (e[:, 0, :, 0] + 127).long(), flat(value)[:, :k]


def fp8_values(q, exps, rows, cols, tall):
    """What a form stands for, in 64 bits."""
    v = q.view(torch.float8_e4m3fn).double()[:rows]
    e = exps.double().repeat_interleave(tall, dim=0)[:rows].repeat_interleave(128, dim=1)
    return v[:, :cols] * two(e[:, :cols] - 127)


def product_bound(a, b, dtype, kind=H.NONE):
    """How far the sum over the columns of a and b of products may be off before it is rounded to `dtype`, values that 8 bits
    stand for: a product of two e4m3 numbers and powers of two is exact in 32 bits, and the matrix cores may cut a sum of them
    off where 32 bits would round it, 2^-23 a term.  For bfloat16 (not with ReLU) they take eight products at a time, of which
    seven may lose what is below 2^-13 of the largest: 7 * 2^-13 of the magnitudes."""
    size = a.abs() @ b.abs().t()
    return size * (2 * (a.shape[1] + 8) * F32 + (7 * 2.0 ** -13 if dtype == torch.bfloat16 and kind != H.RELU else 0))


def linear_fp8(x, w, b, kind, r, dtype):
    """As H.linear, of values that 8 bits stand for, with the bound of their products."""
    y, z, ey, ez = H.linear(x, w, b, kind, r)
    more = product_bound(x, w, dtype, kind)
    return y, z, ey + 1.13 * more, ez + more


def linear_fp8_backward(dy, xt, w, z, kind, dtype, dw_type):
    """(dx, dw, db) and bounds.  dz, in 32 bits, is off by its rounding and by the slope's 2^-19 (GELU, SiLU); a value that
    close to the middle between two 8-bit numbers may go to either, and a block's unit may be the next where its largest
    magnitude is that close to 448 units: both are counted for the entries that they can happen to."""
    dz = dy * H.slope(z, kind) if kind != H.NONE else dy
    off = dy.abs() * (2.0 ** -19 if kind in (H.GELU, H.SILU) else 0) + 2 * F32 * dz.abs() * (kind != H.NONE)

    def eight(v, o):
        here = fp8(v, 1)[2]
        ends = (fp8(v + s * o, 1)[2] for s in (1, -1, torch.sign(v), -torch.sign(v)))
        return here, torch.stack([(t - here).abs() for t in ends]).amax(dim=0)

    rows, n = dz.shape
    a, ea = eight(dz, off)
    t, et = eight(dz.t().contiguous(), off.t().contiguous())
    dx, dw, db = a @ w, t @ xt.t(), dz.sum(dim=0)
    ex = ea @ w.abs() + product_bound(a, w.t(), dtype)
    ew = et @ xt.t().abs() + product_bound(t, xt, dw_type)
    eb = off.sum(dim=0) + (rows + 8) * F32 * dz.abs().sum(dim=0)
    return (dx, dw, db), (ex, ew, eb)


# ---- AdamW ---------------------------------------------------------------------------------------


def moments32(m, v, g, beta1, beta2):
    """The new moments in 32 bits, each operation rounded: what the 8-bit ones are made of."""
    f = lambda s: torch.tensor(s, dtype=torch.float32)  # noqa: E731  a double rounded once
    return f(beta1) * m + f(1 - beta1) * g, f(beta2) * v + (f(1 - beta2) * g) * g


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay):
    """(p, m, v) after step t, in 64 bits."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps), m, v


def adamw_bound(p, g, m, v, t, lr, beta1, beta2, eps, decay):
    """How far 32 bits may be off: the parameter's product and difference are rounded, 1 - lr decay too; the moments are
    rounded three times each (terms of m may cancel), the bias corrections once or, from a device's step, by 2^-21; root,
    quotient and sum of the update add six roundings."""
    new, m1, v1 = adamw(p, g, m, v, t, lr, beta1, beta2, eps, decay)
    root = torch.sqrt(v1 / (1 - beta2 ** t)) + eps
    em = 3 * F32 * (beta1 * m.abs() + (1 - beta1) * g.abs()) / (1 - beta1 ** t)
    update = lr * ((m1 / (1 - beta1 ** t)).abs() * (12 * F32 + 2.0 ** -20) + em) / torch.where(root > 0, root, torch.ones_like(root))
    return 4 * F32 * p.abs() + F32 * new.abs() + update


def moment_codes(x, second, add):
    """(codes, exponent bytes, values) of a flat tensor of 32-bit numbers; add: 20 bits for each entry, or None for the
    nearest (ties to even).  Entry by entry, in whole numbers and 64 bits."""
    n = x.numel()
    bits, bias = (5, 31) if second else (4, 15)
    number = [2.0 ** (1 - bias) * (c % 8) / 8 if c < 8 else 2.0 ** (c // 8 - bias) * (1 + c % 8 / 8) for c in range(1 << (bits + 3))]
    codes, exps, values = [], [], []
    for at in range(0, n, 128):
        block = [float(f) for f in x[at:at + 128]]
        most = max((abs(f) for f in block), default=0.0) if all(math.isfinite(f) for f in block) else math.inf
        if most > 1.875 * 2.0 ** 126:
            exps.append(255)
            codes += [-1] * len(block)
            values += [math.nan] * len(block)
            continue
        e = -95
        while most > 1.875 * 2.0 ** e:
            e += 1
        exps.append(e + 127)
        for i, f in enumerate(block):
            y = abs(f) / 2.0 ** e
            c = bisect.bisect_right(number, y) - 1
            if y > number[c]:
                # the bits of a float: 20 below the third of the mantissa; what is smaller than they hold is rounded to them
                cut = round((y - number[c]) / (number[c + 1] - number[c]) * 2 ** 20)
                if add is None:
                    c += cut > 2 ** 19 or (cut == 2 ** 19 and c % 2 == 1)
                else:
                    c += cut + int(add[at + i]) >= 2 ** 20
                if second and c == 0:
                    c = 1
            codes.append(c + (128 if not second and math.copysign(1, f) < 0 else 0))
            values.append(math.copysign(number[c] * 2.0 ** e, f))
    return codes, exps, values


def sequence(n, t, second):
    h = [(i * 2654435769 + t * 1779033703) % 2 ** 32 for i in range(n)]
    return [((2 ** 32 - 1 - v) if second else v) >> 12 for v in h]


# ---- the loss ------------------------------------------------------------------------------------


def softmax_loss(x, target, weight, scale):
    """(loss, gradient) in 64 bits."""
    rows, classes = x.shape
    w = torch.ones(rows, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    none = (target < 0) | (w == 0) | (x == -math.inf).all(dim=1)
    wrong = ~none & (target >= classes)
    at = target.clamp(0, classes - 1).long()[:, None]
    x = x - x.amax(dim=1, keepdim=True)  # logits of the type's lowest value leave no digits for the logarithm
    lse = torch.logsumexp(x, dim=1)
    loss = w * (lse - x.gather(1, at)[:, 0])
    grad = torch.exp(x - lse[:, None]) - torch.zeros_like(x).scatter_(1, at, 1.0)
    grad = grad * (scale * w)[:, None]
    for t, dim in ((loss, 0), (grad, 1)):
        shape = (-1,) + (1,) * dim
        t.copy_(torch.where(none.reshape(shape), torch.zeros_like(t), torch.where(wrong.reshape(shape), torch.full_like(t, math.nan), t)))
    return loss, grad


def softmax_loss_bound(x, target, weight, scale):
    """x - max is rounded once; its exponential takes its argument times log2 e, rounded twice more, in steps of 2^-24 of
    its magnitude, and is off by 2^-22 itself: together d * 2^-22 + 2^-21 relative for d = max - x, of which nothing is left
    where exp(-d) ends.  The sum of c terms is off by c 2^-24 at most, the logarithm by 2^-22 of it or of 1."""
    rows, classes = x.shape
    w = torch.ones(rows, dtype=torch.float64, device=x.device) if weight is None else weight.double().abs()
    finite = torch.where(torch.isfinite(x), x, torch.full_like(x, -1e4))
    most = finite.amax(dim=1, keepdim=True)
    d = (most - finite).clamp(max=110.0)
    rel = d * 2.0 ** -22 + 2.0 ** -21
    e = torch.exp(-d)
    total = e.sum(dim=1, keepdim=True)
    esum = (e * rel).sum(dim=1, keepdim=True) / total + (classes + 2) * F32
    at = target.clamp(0, classes - 1).long()[:, None]
    far = (most - finite.gather(1, at)).abs()
    eloss = w * (esum + 4 * F32 * (1 + torch.log(total) + far))[:, 0]
    p = e / total
    egrad = (scale * w)[:, None] * (p * (rel + esum + 6 * F32) + torch.zeros_like(x).scatter_(1, at, 4 * F32)) + 1e-38
    return eloss, egrad
