"""The serving operators in 64 bits, from their definitions, on the CPU.

No code of the library: numpy / torch float64, one sequence, request or head
at a time.
"""
import math

import numpy as np
import torch

#: Significand bits: rounding to nearest moves a value by at most 2^-bits of itself.
BITS_BF16, BITS_F32 = 8, 24


def attend(q, k, v, hidden=None, bias=None):
    """q [n, d], k and v [m, d] float64 -> (out [n, d], lse [n], weights [n, m]).

    hidden [n, m] bool: pairs that do not see each other; bias [m] adds to the
    logits.  A row that sees nothing: out 0, lse -inf, weights 0."""
    x = q @ k.T / math.sqrt(q.shape[1])
    if bias is not None:
        x = x + bias
    if hidden is not None:
        x = x.masked_fill(hidden, -math.inf)
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=q.dtype), x
    m = x.max(dim=1, keepdim=True).values
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = torch.exp(x - m)
    z = p.sum(dim=1, keepdim=True)
    w = torch.where(z > 0, p / torch.where(z > 0, z, torch.ones_like(z)), torch.zeros_like(p))
    return w @ v, (m + torch.log(z))[:, 0], w


def logit_error(q, k, n):
    """Bound of an fp32 logit's error and of its exponential's relative error: the
    dot product (d roundings of sums below sum |q k|) over sqrt(d), and 2^-21 of
    the logit's size for the base-2 exponential and the scaling."""
    d = q.shape[1]
    a = float((q.abs() @ k.abs().T).max()) / math.sqrt(d) if n and q.shape[0] else 0.0
    return d * 2.0 ** -24 * a + 2.0 ** -21 * (1 + a)


def attend_bound(q, k, v, out, w, *, weight_bits, out_bits):
    """Elementwise bound on |computed - out|: weights rounded to `weight_bits`
    significant bits move the mean by 2^-bits sum w |v|; a logit error dx by
    2 dx max |v|; n fp32 sums by n 2^-24 max |v|; the output is rounded once."""
    n = k.shape[0]
    vmax = float(v.abs().max()) if n else 0.0
    dx = logit_error(q, k, n)
    return (2.0 ** -weight_bits * (w @ v.abs() if n else 0.0) + vmax * (2 * dx + 2.0 ** -24 * (n + 64))
            + 2.0 ** -out_bits * out.abs() * 1.01 + 1e-7)


def prompt(q, k, v, cu_q, cu_k, *, bf16):
    """Packed causal attention; returns (out, lse, bound of out, bound of lse);
    rows of no sequence are NaN."""
    q, k, v = (t.double().cpu() for t in (q, k, v))
    Hq, G = q.shape[1], k.shape[1]
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for a, b, c, e in zip(cu_q[:-1], cu_q[1:], cu_k[:-1], cu_k[1:]):
        nq, nk = b - a, e - c
        hidden = torch.arange(nk)[None, :] > (torch.arange(nq) + nk - nq)[:, None]
        for h in range(Hq):
            g = h // (Hq // G)
            o, s, w = attend(q[a:b, h], k[c:e, g], v[c:e, g], hidden)
            out[a:b, h], lse[a:b, h] = o, s
            tol[a:b, h] = attend_bound(q[a:b, h], k[c:e, g], v[c:e, g], o, w, weight_bits=BITS_BF16 if bf16 else BITS_F32,
                                       out_bits=BITS_BF16 if bf16 else BITS_F32)
            fin = torch.where(torch.isinf(s), torch.zeros_like(s), s)
            ltol[a:b, h] = logit_error(q[a:b, h], k[c:e, g], nk) + 2.0 ** -24 * (nk + 64) + 2.0 ** -22 * fin.abs()
    return out, lse, tol, ltol


def rotate(x, pos, base):
    """x [..., n, heads, d] rows of token n rotated to pos [n]."""
    x = x.double().cpu()
    d = x.shape[-1]
    if base == 0:
        return x
    theta = torch.tensor([base ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64)
    ang = pos.double().cpu()[:, None] * theta
    c, s = torch.cos(ang)[:, None, :], torch.sin(ang)[:, None, :]
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([a * c - b * s, a * s + b * c], dim=-1)


def rotate_bound(x, want, bits):
    """Angle 2^-26 turns and sine / cosine 2^-22 off, three fp32 roundings, one to `bits`."""
    x = x.double().cpu()
    d = x.shape[-1]
    a, b = x[..., :d // 2].abs(), x[..., d // 2:].abs()
    s = torch.cat([a + b, a + b], dim=-1)
    return s * 2.0 ** -21 + 2.0 ** -bits * want.abs() * 1.01 + 1e-30


def entries(pool, table_row, n):
    """The n entries of one sequence: rows of its pages in order."""
    ps = pool.shape[1]
    pages = table_row[:-(-n // ps)].long()
    return pool[pages].reshape(-1, *pool.shape[2:])[:n]


def decode(q, K, V, log_m, table, lens, l, *, bf16):
    """Paged attention of layer l: (out, bound)."""
    q, K, V, table, lens = (t.cpu() for t in (q, K, V, table, lens))
    log_m = None if log_m is None else log_m.cpu()
    B, Hq, d = q.shape
    G = table.shape[2]
    gq = Hq // G
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b in range(B):
        for g in range(G):
            n = int(lens[l, b, g])
            k, v = (entries(t, table[l, b, g], n).double() for t in (K, V))
            bias = None if log_m is None else entries(log_m, table[l, b, g], n).double()
            qq = q[b, g * gq:(g + 1) * gq].double()
            o, _, w = attend(qq, k, v, bias=bias)
            out[b, g * gq:(g + 1) * gq] = o
            t = attend_bound(qq, k, v, o, w, weight_bits=2 * BITS_BF16 if bf16 else BITS_F32, out_bits=BITS_BF16 if bf16 else BITS_F32)
            if bias is not None and n:
                # log m joins the logit in fp32: one more rounding of its size
                fin = bias[torch.isfinite(bias) & (bias > -1e30)]
                t = t + 2.0 ** -22 * (float(fin.abs().max()) if fin.numel() else 0.0) * float(v.abs().max())
            tol[b, g * gq:(g + 1) * gq] = t
    return out, tol


def scattered_table(rng, lens, page_size, extra=3):
    """(table [L, B, G, most] int32 with -1 past a sequence, pages) for lens [L, B, G]."""
    lens = np.asarray(lens)
    need = -(-lens // page_size)
    total = int(need.sum()) + extra
    order = rng.permutation(total)[:int(need.sum())].astype(np.int32)
    table = np.full(lens.shape + (max(1, int(need.max())),), -1, np.int32)
    at = 0
    for i in np.ndindex(*lens.shape):
        table[i][:need[i]] = order[at:at + need[i]]
        at += need[i]
    return torch.from_numpy(table), max(1, total)
