"""Inputs, on the CPU, whose results show in how many bits the serving calls
compute, and what fewer bits would give."""
from __future__ import annotations

import math

import torch

from . import serving_oracle as R


def _weights(q, k):
    """softmax weights [batch, hq, keys] in 64 bits of vectors that are one number each."""
    b, hq = q.shape[:2]
    z = q[:, :, :1].double() * k.double().repeat_interleave(hq // k.shape[1], 1) / math.sqrt(R.D)
    return torch.softmax(z, -1)


def cancelling(batch, hq, hkv, page, e4m3, seed):
    """One page a sequence whose first keys' values all but cancel: q and the cache's arrays,
    the outputs in 64 bits and the sums of their terms' magnitudes. Element d of the values is
    made for query head d % group of its key head (the others get what it is for them)."""
    g = torch.Generator().manual_seed(seed)
    n, group = (8 if e4m3 else 4), hq // hkv
    kind = R.E4M3 if e4m3 else torch.bfloat16
    q = torch.zeros(batch, hq, R.D)
    q[:, :, 0] = 6 + 5 * torch.rand(batch, hq, generator=g)
    q = q.bfloat16()
    key = (torch.rand(batch, hkv, n, generator=g) * 2 - 1).to(kind)
    p = _weights(q, key.float())
    values = torch.zeros(batch, hkv, n, R.D, dtype=torch.float64)
    made = p.view(batch, hkv, group, n).transpose(2, 3)[..., torch.arange(R.D) % group]
    values[:, :, 0] = 224.0 if e4m3 else 1.0
    rest = made[:, :, 0] * values[:, :, 0]
    for j in range(1, n):
        values[:, :, j] = (-rest / made[:, :, j]).clamp(-448, 448).float().to(kind).double()
        rest = rest + made[:, :, j] * values[:, :, j]
    per_head = values.repeat_interleave(group, 1)
    want = (p.unsqueeze(-1) * per_head).sum(2)
    total = (p.unsqueeze(-1) * per_head.abs()).sum(2)
    k = torch.zeros(batch, hkv, page, R.D)
    v = torch.zeros(batch, hkv, page, R.D)
    k[:, :, :n, 0], v[:, :, :n] = key.float(), values.float()
    scales = ()
    if e4m3:
        scales = tuple(torch.full((batch, hkv, page), 127, dtype=torch.uint8) for _ in "kv")
    return q, k.to(kind), v.to(kind), scales, want, total


def in_two_parts(q, k, v, scales, n):
    """The outputs, else in 64 bits, with every weight as the sum of two bf16 values: its upper
    half, and the rest of weight * (1 + 2^-17), which goes out with the sum."""
    p = _weights(q, k[:, :, :n, 0].float())
    p = (p / p.amax(-1, keepdim=True)).float()
    upper = (p.view(torch.int32) & -65536).view(torch.float32)
    more = 1 + 2.0 ** -17
    rest = (p.double() * more - upper.double()).float().bfloat16()
    parts = upper.double() + rest.double()
    per_head = v[:, :, :n].double().repeat_interleave(q.shape[1] // k.shape[1], 1)
    return (parts.unsqueeze(-1) * per_head).sum(2) / (more * p.double().sum(-1, keepdim=True))


def rotated_in_8_bits(k, pos, pairs, freq, interleaved):
    """(least, most, bytes): the e4m3 values that keys k [batch, heads, tokens, 128], rotated and
    scaled, may round to if their angles are good to 2^-50 of themselves and their sines to
    1e-12, and the scales' bytes. Nearly everywhere least and most are the same."""
    out, _ = R.rotate(k, pos, pairs, freq, interleaved)
    off = torch.zeros_like(out)
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    for i, f in enumerate(freq):
        m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + 64)
        phi = (pos[axis[i]].double() * f).abs().unsqueeze(1)
        both = k[..., m].double().abs() + k[..., n].double().abs()
        off[..., m] = off[..., n] = both * (phi * 2.0 ** -50 + 1e-12)
    least, scale, _ = R.e4m3(out - off, k, interleaved)
    most, _, _ = R.e4m3(out + off, k, interleaved)
    return least, most, scale


def rotated_in_fp32(k, pos, pairs, freq, interleaved):
    """The same values if the keys are turned in 32 bits: the turn in 64, all behind it not."""
    out = k.float().clone()
    axis = [a for a, n in enumerate(pairs) for _ in range(n)]
    for i, f in enumerate(freq):
        m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + 64)
        turn = pos[axis[i]].double() * (f / (2 * math.pi))
        phi = ((turn - turn.round()).float() * (2 * math.pi)).unsqueeze(1)
        a, b = k[..., m].float(), k[..., n].float()
        out[..., m], out[..., n] = a * phi.cos() - b * phi.sin(), a * phi.sin() + b * phi.cos()
    return R.e4m3(out, k, interleaved)[0]
