"""64-bit definitions of the packed-batch operators, and how far their outputs may be off by rounding alone.

HALF[t] is half a step of the type, relative to the value.  Bounds are sums of absolute values in 64 bits times the roundings that the kernels
make: stored outputs, weights as bf16 operands, and float sums of n terms (n + a few roundings of 2^-24)."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -24


def attention(qkv, offsets, nq, nkv, dh, causal, d_o=None):
    """(values, bounds) by name: o, lse, and with d_o dqkv.  Rows of no sequence: NaN."""
    M, t = qkv.shape[0], qkv.dtype
    bf = t == torch.bfloat16
    rows = qkv.double().cpu().view(M, nq + 2 * nkv, dh)
    G, c = nq // nkv, 1.0 / math.sqrt(dh)
    new = lambda *s: torch.full(s, math.nan, dtype=torch.float64)     # noqa: E731
    val = {"o": new(M, nq, dh), "lse": new(M, nq)}
    tol = {"o": new(M, nq, dh), "lse": new(M, nq)}
    if d_o is not None:
        up = d_o.double().cpu().view(M, nq, dh)
        val["dqkv"], tol["dqkv"] = new(M, nq + 2 * nkv, dh), new(M, nq + 2 * nkv, dh)
    for a, z in zip(offsets[:-1], offsets[1:]):
        n = z - a
        if n <= 0:
            continue
        b = slice(a, z)
        if d_o is not None:
            val["dqkv"][b] = 0.0
            tol["dqkv"][b] = 0.0
        hide = torch.ones(n, n, dtype=torch.bool).triu(1) if causal else torch.zeros(n, n, dtype=torch.bool)
        for h in range(nq):
            kh, vh = nq + h // G, nq + nkv + h // G
            q, k, v = rows[b, h], rows[b, kh], rows[b, vh]
            s = (q @ k.t() * c).masked_fill(hide, -math.inf)
            lse = s.logsumexp(-1)
            p = (s - lse[:, None]).exp()
            # error of a score (products summed in float, scale, exponent) and with it the relative error of a weight
            es = ((dh + 8) * F32 * (q.abs() @ k.abs().t()) * c + 8 * F32 * (s.abs().masked_fill(hide, 0.0) + lse.abs()[:, None])).masked_fill(hide, 0.0)
            ep = es + es.amax(-1, keepdim=True) + (n + 16) * F32
            rw = HALF[t] if bf else 0.0
            val["o"][b, h] = p @ v
            eo = (p * (ep + rw)) @ v.abs() + (n + 8) * F32 * (p @ v.abs())
            tol["o"][b, h] = eo + HALF[t] * (val["o"][b, h].abs() + eo)
            val["lse"][b, h] = lse
            tol["lse"][b, h] = es.amax(-1) + (n + 16) * F32 * (1.0 + lse.abs())
            if d_o is None:
                continue
            g = up[b, h]
            dp = g @ v.t()
            D = (g * val["o"][b, h]).sum(-1, keepdim=True)
            ds = p * (dp - D)
            e_dp = (dh + 8) * F32 * (g.abs() @ v.abs().t())
            e_D = (g.abs() * (tol["o"][b, h] + (dh + 8) * F32 * val["o"][b, h].abs())).sum(-1, keepdim=True)
            e_lse = tol["lse"][b, h][:, None]
            e_ds = ds.abs() * (ep + e_lse + rw) + p * (e_dp + e_D + 2 * F32 * (dp.abs() + D.abs()))
            e_p = p * (ep + e_lse + rw)
            add = lambda at, x, e: (val["dqkv"][b, at].add_(x), tol["dqkv"][b, at].add_(e))     # noqa: E731
            nr = (n * G + 8) * F32
            add(h, ds @ k * c, (e_ds @ k.abs() + nr * (ds.abs() @ k.abs())) * c)
            add(kh, ds.t() @ q * c, (e_ds.t() @ q.abs() + nr * (ds.abs().t() @ q.abs())) * c)
            add(vh, p.t() @ g, e_p.t() @ g.abs() + nr * (p.t() @ g.abs()))
        if d_o is not None:
            tol["dqkv"][b] += HALF[t] * (val["dqkv"][b].abs() + tol["dqkv"][b])
    flat = lambda x: x.reshape(M, -1)     # noqa: E731
    return {k: flat(x) for k, x in val.items()}, {k: flat(x) for k, x in tol.items()}


def check(got, val, tol, what):
    """Every value within its bound; rows without a value (NaN) are not looked at."""
    got = got.double().cpu().reshape(val.shape)
    have = ~torch.isnan(val)
    assert torch.isfinite(got[have]).all(), what
    off = (got - val).abs()[have]
    worst = (off / (tol[have] + 1e-300)).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound"
    return worst


def loss(x, w, labels, first, vocab, lse, dloss):
    """(values, bounds) of one shard for a given lse over the whole vocabulary: own lse, target, dx, dw."""
    t = x.dtype
    X, W, y = x.double().cpu(), w.double().cpu(), labels.long().cpu()
    M, H, V = X.shape[0], X.shape[1], W.shape[0]
    z = X @ W.t()
    ez = (H + 8) * F32 * (X.abs() @ W.abs().t()) + 8 * F32 * z.abs()
    own = z.logsumexp(1)
    top = ez.amax(1)
    here = (y >= first) & (y < first + V)
    at = (y - first).clamp(0, V - 1)
    val = {"lse": own, "target": torch.where(here, z.gather(1, at[:, None])[:, 0], torch.full_like(own, -math.inf))}
    tol = {"lse": top + (V + 32) * F32 * (1 + own.abs()), "target": top}
    L, d = lse.double().cpu(), dloss.double().cpu()
    known = (y >= 0) & (y < vocab)
    d = torch.where(known, d, torch.zeros_like(d))
    p = (z - L[:, None]).exp()
    one = torch.zeros_like(p)
    one[here.nonzero()[:, 0], at[here]] = 1.0
    dz = (p - one) * d[:, None]
    rw = HALF[t] if t == torch.bfloat16 else 0.0
    e = p * (ez + 8 * F32 * (1 + L.abs()[:, None])) * d.abs()[:, None] + dz.abs() * (4 * F32) + one * d.abs()[:, None] * F32
    e = e + rw * (dz.abs() + e)
    # a probability, or a product with it, below the least normal float (2^-126) may become zero: off by that much at most
    e = e + 2.0 ** -126 * (1 + d.abs()[:, None])
    val["dx"], val["dw"] = dz @ W, dz.t() @ X
    tol["dx"] = e @ W.abs() + (V + 32) * F32 * (dz.abs() @ W.abs())
    tol["dw"] = e.t() @ X.abs() + (M + 32) * F32 * (dz.abs().t() @ X.abs())
    for k in ("dx", "dw"):
        tol[k] = tol[k] + HALF[t] * (val[k].abs() + tol[k]) + 2.0 ** -126
    return val, tol


def rotary(rows, nq, nkv, dh, rot, adjacent, positions, freq, factor, back):
    t, M = rows.dtype, rows.shape[0]
    x = rows.double().cpu().view(M, nq + 2 * nkv, dh)
    a = positions.double().cpu()[:, None] * torch.tensor(freq, dtype=torch.float64)
    c, s = (a.cos() * factor)[:, None], (a.sin() * (-factor if back else factor))[:, None]
    i = torch.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
    out, tol = x.clone(), torch.zeros_like(x)
    u, v = x[:, :nq + nkv, first], x[:, :nq + nkv, second]
    out[:, :nq + nkv, first], out[:, :nq + nkv, second] = u * c - v * s, u * s + v * c
    # sine and cosine to 4 roundings, two products and a sum; the angle of 64 bits at most 2^-20 of a float step off
    e = 8 * F32 * factor * (u.abs() + v.abs())
    tol[:, :nq + nkv, first], tol[:, :nq + nkv, second] = e, e
    tol[:, :nq + nkv, :rot] += HALF[t] * (out[:, :nq + nkv, :rot].abs() + tol[:, :nq + nkv, :rot])
    return out.reshape(M, -1), tol.reshape(M, -1)
