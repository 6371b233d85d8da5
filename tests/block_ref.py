"""64-bit definitions of the norms of heads with the rotation and of dropout, and how far their outputs may be off by rounding alone (packed_ref: HALF, F32)."""
import math

import numpy
import torch

from packed_ref import F32, HALF


def _pairs(rot, adjacent):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)


def _turn(x, rot, adjacent, c, s, factor):
    """(values, sum of the absolute values that each is made of)."""
    first, second = _pairs(rot, adjacent)
    out, size = x.clone(), x.abs()
    u, v = x[..., first], x[..., second]
    out[..., first], out[..., second] = factor * (u * c - v * s), factor * (u * s + v * c)
    size[..., first] = size[..., second] = factor * (u.abs() + v.abs())
    return out, size


def norm(qkv, nq, nkv, dh, rot, adjacent, positions, freq, factor, gamma_q, gamma_k, per_head, eps, dqkv=None):
    """(values, bounds) by name: out, and with dqkv dout, dgamma_q, dgamma_k."""
    t, M, heads = qkv.dtype, qkv.shape[0], nq + nkv
    rows = qkv.double().cpu().view(M, nq + 2 * nkv, dh)
    x = rows[:, :heads]
    wide = lambda w, n: w.double().cpu().view(-1, dh).expand(n, dh)      # noqa: E731
    gamma = torch.cat([wide(gamma_q, nq), wide(gamma_k, nkv)])
    a = positions.double().cpu()[:, None] * torch.tensor(freq, dtype=torch.float64)
    c, s = a.cos()[:, None], a.sin()[:, None]
    # an angle of 64 bits, position (31 bits) times frequency and its whole turns, and sine and cosine to 4 roundings of 32 bits
    far = 8 * F32 + positions.abs().max().item() * 2.0 ** -50
    rstd = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    xh = x * rstd
    ex = (dh / 2 + 8) * F32                                              # of xh: half of the sum's, root and quotient, product
    y, size = _turn(xh * gamma, rot, adjacent, c, s, factor)
    out, tol = rows.clone(), torch.zeros_like(rows)
    out[:, :heads] = y
    e = (ex + 2 * F32 + far) * size
    tol[:, :heads] = e + HALF[t] * (y.abs() + e)
    val, off = {"out": out.reshape(M, -1)}, {"out": tol.reshape(M, -1)}
    if dqkv is None:
        return val, off
    up = dqkv.double().cpu().view(M, nq + 2 * nkv, dh)
    g, size = _turn(up[:, :heads], rot, adjacent, c, -s, factor)
    eg = far * size
    w = g * gamma
    mean = (w * xh).mean(-1, keepdim=True)
    e_mean = (eg * (gamma * xh).abs()).mean(-1, keepdim=True) + (dh + 8 + ex / F32) * F32 * (w * xh).abs().mean(-1, keepdim=True)
    dx = rstd * (w - xh * mean)
    e = rstd * (eg * gamma.abs() + (ex + 4 * F32) * w.abs() + xh.abs() * e_mean + (2 * ex + 4 * F32) * (xh * mean).abs())
    dout, tol = up.clone(), torch.zeros_like(up)
    dout[:, :heads], tol[:, :heads] = dx, e + HALF[t] * (dx.abs() + e)
    val["dout"], off["dout"] = dout.reshape(M, -1), tol.reshape(M, -1)
    terms, size = (g * xh), eg * xh.abs() + (ex + 2 * F32) * (g * xh).abs()
    for name, h in (("dgamma_q", slice(0, nq)), ("dgamma_k", slice(nq, heads))):
        dims = (0,) if per_head else (0, 1)
        n = M * (1 if per_head else h.stop - h.start)
        d, e = terms[:, h].sum(dims), size[:, h].sum(dims) + (n + 8) * F32 * terms[:, h].abs().sum(dims)
        val[name], off[name] = d.reshape(-1), (e + HALF[t] * (d.abs() + e)).reshape(-1)
    return val, off


def philox(counter, key):
    """Philox4x32-10 (Salmon et al., SC 2011) in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(M, N, p, seed, step, site, first_row, first_col, width):
    """(mask [M, N], scale)."""
    t = min(65535, math.floor(65536 * p + 0.5))
    keep = numpy.zeros((M, N), dtype=bool)
    for r in range(M):
        for c in range(0, N, 8):
            g = ((first_row + r) * width + first_col + c) // 8
            w = philox([g & 0xFFFFFFFF, (g >> 32) + 4096 * site, step & 0xFFFFFFFF, step >> 32], [seed & 0xFFFFFFFF, seed >> 32])
            keep[r, c:c + 8] = [(w[e // 2] >> 16 * (e % 2) & 0xFFFF) >= t for e in range(8)]
    return torch.from_numpy(keep), 65536.0 / (65536 - t)


def dropout(x, bias, resid, keep, scale):
    """(out, bound): a sum, a product, a sum, each rounded to 32 bits, and the output."""
    v = x.double().cpu()
    size = v.abs()
    if bias is not None:
        v, size = v + bias.double().cpu(), size + bias.double().cpu().abs()
    out, size = torch.where(keep, v * scale, 0.0), torch.where(keep, size * scale, 0.0)
    if resid is not None:
        out, size = out + resid.double().cpu(), size + resid.double().cpu().abs()
    e = 4 * F32 * size
    return out, e + HALF[x.dtype] * (out.abs() + e)


def dropout_bwd(dout, keep, scale):
    """(din, bound, dbias, bound)."""
    d = torch.where(keep, dout.double().cpu() * scale, 0.0)
    e = 2 * F32 * d.abs()
    s, es = d.sum(0), e.sum(0) + (d.shape[0] + 8) * F32 * d.abs().sum(0)
    h = HALF[dout.dtype]
    return d, e + h * (d.abs() + e), s, es + h * (s.abs() + es)
