"""The operators of a gated block in 64 bits, and bounds that their results are held to (see train_ref for the units).

Row sums: a thread adds its eight values and the waves' sums by twos, at most 8 + 6 + 16 additions in a row and a few
roundings beside them: ROW units of 2^-24 of the sum of magnitudes. Rows past 8192 columns: four times eight values."""

import numpy as np
import torch

from train_ref import E32, U, act64, act_error

ROW = 40.0


def philox(counter, key):
    """Philox 4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011) of counters (4, ...) and two key words, as uint32 words."""
    x = [np.array(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), b & np.uint64(0xFFFFFFFF),
             (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), a & np.uint64(0xFFFFFFFF)]
        k = [k[0] + 0x9E3779B9 & 0xFFFFFFFF, k[1] + 0xBB67AE85 & 0xFFFFFFFF]
    return np.stack(np.broadcast_arrays(*x))


def drop_factor(rows, cols, p, at):
    """What dropout multiplies each element by, by the definition, on the host."""
    seed, offset = (int(v) & (1 << 64) - 1 for v in at)
    group = np.arange(-(-cols // 8), dtype=np.uint64)[None, :]
    row = np.arange(rows, dtype=np.uint64)[:, None]
    w = philox([group, row, offset & 0xFFFFFFFF, offset >> 32], [seed & 0xFFFFFFFF, seed >> 32])
    w = np.broadcast_to(w, (4, rows, group.shape[1]))
    halves = np.stack([v for word in w for v in (word & np.uint64(0xFFFF), word >> np.uint64(16))], -1)
    t = int(65536 * p + 0.5)
    keep = halves.reshape(rows, -1)[:, :cols].astype(np.int64) >= t
    return torch.from_numpy(keep * (65536 / (65536 - t) if t < 65536 else 0.0))


def gated64(act, zg, zu, eg, eu):
    """(y, its error before rounding) of act(zg) zu, where zg and zu are off by eg and eu."""
    a, _ = act64(act, zg)
    ea = 1.2 * eg + (act_error(zg) if act != "none" else 0)
    y = a * zu
    return y, ea * (zu.abs() + eu) + a.abs() * eu + 2 * E32 * y.abs()


def gate_slopes64(act, zg, zu, da, ed):
    """((dg, error), (du, error), (a, error)) where da is off by ed."""
    a, slope = act64(act, zg)
    ea = act_error(zg) if act != "none" else torch.zeros_like(zg)
    dg, du, y = da * zu * slope, da * a, a * zu
    d = da.abs() + ed
    return ((dg, zu.abs() * (d * ea + ed * slope.abs()) + 4 * E32 * dg.abs()),
            (du, d * ea + ed * a.abs() + 4 * E32 * du.abs()), (y, ea * zu.abs() + 4 * E32 * y.abs()))


def norm64(x, e, kind, eps):
    """(xhat, its error, mean, rstd) of rows x that are off by e."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    c = x - mean
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    xh = c * rstd
    own = ROW * E32 * xh.abs() + rstd * E32 * (2 * x.abs() + ROW * x.abs().mean(1, keepdim=True)) * (kind == "layer")
    through = rstd * (e + (e.mean(1, keepdim=True) if kind == "layer" else 0) + xh.abs() * e.square().mean(1, keepdim=True).sqrt())
    return xh, own + 1.1 * through, mean, rstd


def affine64(xh, e, w, b):
    y = xh * w + b
    return y, e * w.abs() + 2 * E32 * (y.abs() + b.abs())


def residual64(y, r, post, pre, gate, scale, factor, kind, eps):
    """The forward pass: a dict of (value, error before rounding). Weights are given whole."""
    out, v, e = {}, y, torch.zeros_like(y)
    if post is not None:
        v, e, out["mean1"], out["rstd1"] = norm64(v, e, kind, eps)
        v, e = affine64(v, e, *post)
    v, e = v * gate * factor, (e + 4 * E32 * v.abs()) * gate.abs() * factor
    if r is not None:
        e = e + 2 * E32 * (v.abs() + (scale * r).abs())
        v = v + scale * r
    out["s"] = v, e
    if pre is not None:
        xh, e, out["mean2"], out["rstd2"] = norm64(v, e, kind, eps)
        out["xhat"] = xh, e
        out["h"] = affine64(xh, e, *pre)
    return out


def norm_back64(g, eg, w, xh, exh, rstd, kind):
    """(dx, error) of a norm whose output's gradient g is off by eg, with xhat off by exh."""
    h, eh = g * w, eg * w.abs() + E32 * (g * w).abs()
    mean = lambda t: t.mean(1, keepdim=True)   # noqa: E731
    layer = kind == "layer"
    m1, em1 = (mean(h), mean(eh) + ROW * E32 * mean(h.abs())) if layer else (0, 0)
    m2 = mean(h * xh)
    em2 = mean(eh * (xh.abs() + exh) + h.abs() * exh) + ROW * E32 * mean((h * xh).abs())
    dx = rstd * (h - m1 - xh * m2)
    size = h.abs() + (m1.abs() if layer else 0) + (xh * m2).abs()
    return dx, rstd * (eh + em1 + xh.abs() * em2 + exh * (m2.abs() + em2) + 5 * E32 * size)


def xhat64(x, mean, rstd):
    """((x - mean) rstd, its error in fp32)."""
    xh = (x - mean) * rstd
    return xh, 3 * E32 * xh.abs() + E32 * rstd * (x.abs() + mean.abs() if isinstance(mean, torch.Tensor) else 0 * x)


def sums64(t, e, parts):
    """Column sums over the rows and their error: a work-group's rows one after another, then the parts by sixteens."""
    return t.sum(0), E32 * (-(-t.shape[0] // parts) + parts / 16 + 40) * t.abs().sum(0) + e.sum(0)


def residual_back64(ds, dh, y, s, stats, post, pre, gate, full, scale, factor, kind, copy=None):
    """The gradients: a dict of (value, error). stats: mean1, rstd1, mean2, rstd2 as columns (means 0 where there are none).
    full: the gate has a value for each element."""
    out = {}
    mean1, rstd1, mean2, rstd2 = stats
    like = dh if dh is not None else ds
    d, e = torch.zeros_like(like), torch.zeros_like(like)
    parts = 1024
    if pre is not None:
        xh, exh = (copy, torch.zeros_like(like)) if copy is not None else xhat64(s, mean2, rstd2)
        d, e = norm_back64(dh, torch.zeros_like(dh), pre[0], xh, exh, rstd2, kind)
        out["dpre_w"] = sums64(dh * xh, dh.abs() * exh, parts)
        out["dpre_b"] = sums64(dh, torch.zeros_like(dh), parts)
    if ds is not None:
        e = e + 2 * E32 * (d.abs() + ds.abs())
        d = d + ds
    out["dr"] = scale * d, abs(scale) * e + 2 * E32 * (scale * d).abs()
    t, et = d * factor, (e + 3 * E32 * d.abs()) * factor
    if y is not None:
        xh, exh = y, torch.zeros_like(y)
        n, en = xh, exh
        if post is not None:
            xh, exh = xhat64(y, mean1, rstd1)
            n, en = affine64(xh, exh, *post)
        dg = t * n
        eg = et * (n.abs() + en) + t.abs() * en + 3 * E32 * dg.abs()
        # through the sums of t xhat and t, by the weight and the bias
        if full:
            out["dgate"] = dg, eg
        else:
            big = (t * xh).abs() * (post[0].abs() if post is not None else 1) + t.abs() * (post[1].abs() if post is not None else 0)
            out["dgate"] = dg.sum(0), sums64(big, eg + 4 * E32 * big, parts)[1]
    dn, en = t * gate, et * gate.abs() + 3 * E32 * (t * gate).abs()
    if post is not None:
        out["dpost_w"] = sums64(dn * xh, en * (xh.abs() + exh) + dn.abs() * exh + 3 * E32 * (dn * xh).abs(), parts)
        out["dpost_b"] = sums64(dn, en + 3 * E32 * dn.abs(), parts)
        dn, en = norm_back64(dn, en, post[0], xh, exh, rstd1, kind)
    out["dy"] = dn, en
    return out


def rounded(value, error, dtype, tiny):
    """The bound of a value stored in dtype."""
    return U[dtype] * value.abs() + error * 1.01 + tiny
