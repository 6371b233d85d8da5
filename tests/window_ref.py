"""64-bit definition of attention with a sliding window and first tokens that stay visible, and how far its outputs may be off by rounding alone:
the roundings that the kernels make as in packed_ref."""
import math

import torch

from packed_ref import F32, HALF


def sees(n, window, sinks):
    """[query, key] of a sequence of n tokens."""
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    return (j <= i) & ((i - j < window) | (j < sinks))


def attention(qkv, offsets, nq, nkv, dh, window, sinks, d_o=None):
    """(values, bounds) by name: o, lse, and with d_o dqkv.  Rows of no sequence: NaN."""
    M, t = qkv.shape[0], qkv.dtype
    rw = HALF[t] if t == torch.bfloat16 else 0.0                      # weights and dS as operands
    rows = qkv.double().cpu().view(M, nq + 2 * nkv, dh)
    G, c = nq // nkv, 1.0 / math.sqrt(dh)
    widths = {"o": (nq, dh), "lse": (nq,)}
    if d_o is not None:
        widths["dqkv"] = (nq + 2 * nkv, dh)
        up = d_o.double().cpu().view(M, nq, dh)
    val = {k: torch.full((M, *w), math.nan, dtype=torch.float64) for k, w in widths.items()}
    tol = {k: x.clone() for k, x in val.items()}
    for a, z in zip(offsets[:-1], offsets[1:]):
        n, b = z - a, slice(a, z)
        if n <= 0:
            continue
        if d_o is not None:
            val["dqkv"][b] = tol["dqkv"][b] = 0.0
        hide = ~sees(n, window, sinks)
        for h in range(nq):
            kh, vh = nq + h // G, nq + nkv + h // G
            q, k, v = rows[b, h], rows[b, kh], rows[b, vh]
            s = (q @ k.t() * c).masked_fill(hide, -math.inf)
            lse = s.logsumexp(-1)
            p = (s - lse[:, None]).exp()
            es = (dh + 8) * F32 * (q.abs() @ k.abs().t()) * c + 8 * F32 * (s.abs() + lse.abs()[:, None])
            es = es.masked_fill(hide, 0.0)
            ep = es + es.amax(-1, keepdim=True) + (n + 16) * F32
            o = p @ v
            eo = (p * (ep + rw)) @ v.abs() + (n + 8) * F32 * (p @ v.abs())
            val["o"][b, h], tol["o"][b, h] = o, eo + HALF[t] * (o.abs() + eo)
            val["lse"][b, h], tol["lse"][b, h] = lse, es.amax(-1) + (n + 16) * F32 * (1.0 + lse.abs())
            if d_o is None:
                continue
            g = up[b, h]
            dp = g @ v.t()
            D = (g * o).sum(-1, keepdim=True)
            ds = p * (dp - D)
            e_dp = (dh + 8) * F32 * (g.abs() @ v.abs().t())
            e_D = (g.abs() * (tol["o"][b, h] + (dh + 8) * F32 * o.abs())).sum(-1, keepdim=True)
            rel = ep + tol["lse"][b, h][:, None] + rw
            e_ds = ds.abs() * rel + p * (e_dp + e_D + 2 * F32 * (dp.abs() + D.abs()))
            nr = (n * G + 8) * F32
            for at, w, ew, x, f in ((h, ds, e_ds, k, c), (kh, ds.t(), e_ds.t(), q, c), (vh, p.t(), (p * rel).t(), g, 1.0)):
                val["dqkv"][b, at] += w @ x * f
                tol["dqkv"][b, at] += (ew @ x.abs() + nr * (w.abs() @ x.abs())) * f
        if d_o is not None:
            tol["dqkv"][b] += HALF[t] * (val["dqkv"][b].abs() + tol["dqkv"][b])
    return {k: x.reshape(M, -1) for k, x in val.items()}, {k: x.reshape(M, -1) for k, x in tol.items()}
