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
