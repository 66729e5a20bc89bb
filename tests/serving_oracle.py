"""Plain 64-bit forms of the calls for serving after the prefill, on the CPU,
token after token as include/xattn.h defines them, and the bounds that the
GPU's results are held to (derived here from their rounding steps)."""
from __future__ import annotations

import math

import torch

D = 128
E4M3 = torch.float8_e4m3fn
HALF_BF16 = 2.0 ** -8    # half a step, relative
HALF_E4M3 = 2.0 ** -4
# The hardware's sine and cosine: 2^-21 of absolute error at most over a grid of
# 2^22 turns; the turn itself is rounded to fp32, |turn| <= 1/2: pi 2^-24.
TRIG = 2.0 ** -21 + math.pi * 2.0 ** -24


def freqs(pairs, base=10000.0):
    n = sum(pairs)
    return [base ** (-i / n) for i in range(n)]


def rotate(x, pos, pairs, freq, interleaved, inverse=False):
    """x [batch, heads, tokens, 128] by pos [axes, batch, tokens]; and the bound of each value:
    the trig's error on both values of the pair, three fp32 operations (the products'
    and the sum's roundings), without the last rounding."""
    out, bound = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    for i, f in enumerate(freq):
        m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + 64)
        phi = (pos[axis[i]].double() * f).unsqueeze(1) * (-1 if inverse else 1)
        a, b = x[..., m].double(), x[..., n].double()
        out[..., m] = a * phi.cos() - b * phi.sin()
        out[..., n] = a * phi.sin() + b * phi.cos()
        # angles in 64 bits: turns * 2^-52 of the definition's own product
        far = phi.abs() * 2.0 ** -51
        both = (a.abs() + b.abs()) * (TRIG + 3 * 2.0 ** -24 + far)
        bound[..., m] = bound[..., n] = both
    return out, bound


def bf16_bound(want, before):
    """Half a step of the value that is rounded, which may be off by `before`; the least step is
    2^-133."""
    return (want.abs() + before) * HALF_BF16 + before + 2.0 ** -134


def e4m3(x, given, pairs_of=None):
    """(values, bytes) of vectors x whose scale follows from `given`, the values before the
    rotation; pairs_of: None, or whether the rotated pairs are interleaved."""
    g = given.double()
    g = torch.where(torch.isfinite(g), g, 0.0)
    if pairs_of is not None:
        g = torch.hypot(g[..., 0::2], g[..., 1::2]) if pairs_of else \
            torch.hypot(g[..., :64], g[..., 64:])
    most = g.abs().amax(-1, keepdim=True)
    e = torch.where(most > 0, torch.ceil(torch.log2(most / 448)), 0.0).clamp(-126, 127)
    y = (x.double() / torch.exp2(e)).clamp(-448, 448)  # keeps NaN
    return y.float().to(E4M3), (e.squeeze(-1) + 127).to(torch.uint8), torch.exp2(e)


def cached(k, v, table_row, k_scale, v_scale, page, tokens):
    """Keys and values (fp64 [hkv, tokens, 128]) of one sequence and which exist."""
    pages, hkv = k.shape[:2]
    kk = torch.zeros(hkv, tokens, D, dtype=torch.float64)
    vv, there = torch.zeros_like(kk), torch.zeros(tokens, dtype=torch.bool)
    for t in range(tokens):
        p = int(table_row[t // page])
        if 0 <= p < pages:
            there[t] = True
            kk[:, t], vv[:, t] = k[p, :, t % page].double(), v[p, :, t % page].double()
            if k_scale is not None:
                kk[:, t] *= torch.exp2(k_scale[p, :, t % page].double() - 127).unsqueeze(-1)
                vv[:, t] *= torch.exp2(v_scale[p, :, t % page].double() - 127).unsqueeze(-1)
    return kk, vv, there


def decode(q, k, v, table, lens, k_scale=None, v_scale=None):
    """o, lse, weight increments and their bounds, for q [batch, hq, 128]."""
    batch, hq = q.shape[:2]
    hkv, page = k.shape[1], k.shape[2]
    group, capacity = hq // hkv, table.shape[1] * page
    o = torch.zeros(batch, hq, D, dtype=torch.float64)
    lse = torch.full((batch, hq), -math.inf, dtype=torch.float64)
    w = torch.zeros(batch, hkv, capacity, dtype=torch.float64)
    ob, lb, wb = torch.zeros_like(o), torch.zeros_like(lse), torch.zeros_like(w)
    for b in range(batch):
        n = min(max(int(lens[b]), 0), capacity)
        kk, vv, there = cached(k, v, table[b], k_scale, v_scale, page, n)
        for h in range(hq):
            g = h // group
            x = q[b, h].double()
            z = (kk[g] @ x) / math.sqrt(D)
            z = torch.where(there & (z != -math.inf), z, torch.tensor(-math.inf).double())
            if not (z > -math.inf).any():
                continue
            lse[b, h] = torch.logsumexp(z, 0)
            p = torch.exp(z - lse[b, h])
            use = z > -math.inf
            o[b, h] = p[use] @ vv[g][use]
            w[b, g, :n] += p
            # 128 exact products added in fp32 in any order, each addition off by at
            # most a step (2^-23), then three roundings on the way to the exponent
            dz = float(((kk[g].abs() @ x.abs()) / math.sqrt(D))[use].max()) * 131 * 2.0 ** -23
            dz += float(z[use].abs().max()) * 4 * 2.0 ** -24
            # the exponential's 2^-22 and at most n + 8 roundings of the sums and joins
            rel = 2 * dz + 2.0 ** -20 + (n + 8) * 2.0 ** -24
            # P in the product is two bf16 parts: the upper 8 bits of mantissa leave at
            # most 2^-7 of it, whose rounding to 8 bits is off by at most 2^-8 of that
            ob[b, h] = (p[use] @ vv[g][use].abs()) * (2 * rel + 2.0 ** -15)
            lb[b, h] = dz + 2.0 ** -20 + (n + 8) * 2.0 ** -24 + abs(float(lse[b, h])) * 2.0 ** -22
            wb[b, g, :n] += p * 2 * rel
    return o, lse, w, ob, lb, wb


def keep(weights, n, budget, recent):
    """Tokens kept of one sequence and key head of n tokens, ascending."""
    if n <= budget:
        return list(range(n))
    old = n - recent

    def rank(t):
        x = float(weights[t])
        return (-math.inf, 1) if math.isnan(x) else (x, 0)

    def order(t):
        x, nan = rank(t)
        return (nan, -x, t)

    return sorted(sorted(range(old), key=order)[:budget - recent]) + list(range(old, n))
