"""The training operators' definitions in 64 bits, and the bounds that their results are held to.

Bounds are elementwise and follow from the arithmetic: a stored result is off by
half a unit of its type's last place (U), a sum of fp32 products by its length
times 2^-24 of the sum of their magnitudes at most, taken here as the growth of
sums joined in pieces (GROWTH of its length)."""

import math

import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}   # results near the type's smallest
E32 = 2.0 ** -24


def growth(n):
    """fp32 error of a sum of n products, in units of 2^-24 of the sum of magnitudes: pieces of 32 are
    summed by the matrix cores (cut, not rounded: a whole unit each), then added one after another."""
    return 8.0 + n / 16.0


def act64(name, z):
    """(act(z), act'(z))"""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 0.134145 * z * z)
    p = torch.sigmoid(z)
    return z * p, p * (1 + z * (1 - p))


def act_error(z):
    """Of act and act' in fp32: the normal distribution function to 1.5e-7 (half of erf's), the
    exponential and the reciprocal to a few units, times |z|."""
    return 4e-7 * (1 + z.abs())


def pack64(x):
    """(q, s) of a matrix, by the definition, in 64 bits (exact for fp32 values)."""
    rows, cols = x.shape
    v = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=x.device)
    v[:, :cols] = x.double()
    v = v.view(rows, -1, 32)
    m = v.abs().amax(2)
    e = torch.full_like(m, -126)
    for t in range(-126, 123):   # the smallest power that covers the group
        e = torch.where(m > 127 * 2.0 ** t, torch.full_like(m, t + 1), e)
    bad = ~torch.isfinite(v).all(2)
    q = torch.round(v / torch.exp2(e)[:, :, None])
    q = torch.where(e[:, :, None] == 122, q.clamp(-63, 63), q)   # 64 * 2^122 is past fp32's largest value
    q = torch.where(bad[:, :, None], torch.zeros_like(q), q)
    s = torch.where(bad, torch.full_like(e, 255), e + 127)
    return q.reshape(rows, -1)[:, :cols].to(torch.int8), s.to(torch.uint8)


def unpack64(q, s):
    scale = torch.exp2(s.double() - 127)
    scale = torch.where(s == 255, torch.full_like(scale, float("nan")), scale)
    return q.double() * scale.repeat_interleave(32, 1)[:, :q.shape[1]]


def off(got, want, bound):
    """The largest error in units of its bound (infinite where only one side is finite)."""
    got = got.double()
    if got.shape != want.shape:
        return math.inf
    fine = torch.isfinite(want)
    if not torch.equal(fine, torch.isfinite(got)):
        return math.inf
    d = (got - want).abs()[fine] / bound.expand_as(want)[fine]
    return float(d.max()) if d.numel() else 0.0
