"""The operators of a server that answers after the prefill, in their plain form
and as calls of this library: rotary positions with several axes, the append of
keys and values to a paged cache, the attention of one new token over that
cache, and the eviction of its lightest tokens.

A case is a dict of plain values. `op` names the call:

  rotary  rotation of the heads of q or k by their positions, from the
          projections' token-major order to the heads' order that attention takes
  append  keys (rotated on the way where `rotate`) and values of new tokens
          into their pages, `type` bf16 or e4m3 with a power-of-two scale per vector
  decode  one new token per sequence over its pages; `weights`: the cache's
          accumulated attention weights are updated too
  evict   the `budget` tokens of each sequence and key head that are worth most
          (the last `recent` and the heaviest) moved to other pages

Lengths of a ragged batch follow from the case alone (`_lens`), values from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DIM = 128
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # The queries of one new token in a batch of 8: the smallest call, latency alone.
        dict(name="rotary_token", op="rotary", batch=8, heads=32, tokens=1, axes=1,
             interleaved=False, restart=False, inverse=False, far=100000),
        # The queries of a 32K-token prompt with images (time, height, width).
        dict(name="rotary_prompt_32k", op="rotary", batch=1, heads=32, tokens=32768, axes=3,
             interleaved=False, restart=False, inverse=False, far=33000),
        # A 115,200-token video layer (30 x 60 x 64), each axis with its own frequencies.
        dict(name="rotary_video_115200", op="rotary", batch=1, heads=24, tokens=115200, axes=3,
             interleaved=True, restart=True, inverse=False, far=64),
        # Odd sizes, back: as for keys that are to be given other positions.
        dict(name="rotary_back_1733", op="rotary", batch=3, heads=7, tokens=1733, axes=2,
             interleaved=False, restart=True, inverse=True, far=1000000),
        # The new keys and values of 64 sequences in one decoding step.
        dict(name="append_token_64", op="append", batch=64, hkv=8, tokens=1, page=64, type="bf16",
             rotate=True, ragged=False),
        # Two prompts of up to 30,001 tokens into an 8-bit cache, padded to one length.
        dict(name="append_prompt_e4m3", op="append", batch=2, hkv=8, tokens=30001, page=64,
             type="e4m3", rotate=False, ragged=True),
        # A short chat on one key head: a rank of a split layer.
        dict(name="decode_700_1head", op="decode", batch=1, hq=4, hkv=1, len=700, page=64,
             type="bf16", weights=False, ragged=False),
        # 64 sequences of up to 8000 tokens in one batch.
        dict(name="decode_64_ragged", op="decode", batch=64, hq=32, hkv=8, len=8000, page=64,
             type="bf16", weights=False, ragged=True),
        # One sequence behind a 128K-token prompt.
        dict(name="decode_128k", op="decode", batch=1, hq=32, hkv=8, len=131071, page=128,
             type="bf16", weights=False, ragged=False),
        # 16 sequences of up to 20,011 tokens in an 8-bit cache that will be evicted from.
        dict(name="decode_e4m3_weights", op="decode", batch=16, hq=28, hkv=4, len=20011, page=16,
             type="e4m3", weights=True, ragged=True),
        # Four 16,000-token sequences cut to 4096.
        dict(name="evict_16k_batch4", op="evict", batch=4, hkv=8, len=16000, page=64, type="bf16",
             budget=4096, recent=512, ragged=True),
        # A 128K-token sequence in an 8-bit cache cut to 30,000.
        dict(name="evict_128k_e4m3", op="evict", batch=1, hkv=8, len=131071, page=128,
             type="e4m3", budget=30000, recent=1000, ragged=False),
    ]


HEADS = [(1, 1), (4, 1), (4, 4), (8, 2), (12, 4), (16, 2), (24, 24), (28, 4), (32, 8), (32, 32),
         (40, 2), (64, 8)]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """A case of the same ranges: log-spread lengths and batches, any head layout and page."""
    op = rng.choice(["rotary"] * 2 + ["append"] * 2 + ["decode"] * 4 + ["evict"] * 2)
    hq, hkv = rng.choice(HEADS)
    if op == "rotary":
        case = dict(op=op, batch=_log(rng, 1, 16), heads=rng.choice([1, 7, 8, 24, 32, hkv]),
                    tokens=_log(rng, 1, 115200), axes=rng.choice([1, 2, 3, 3]),
                    interleaved=rng.random() < 0.5, restart=rng.random() < 0.5,
                    inverse=rng.random() < 0.3, far=_log(rng, 2, 1000000))
        while case["batch"] * case["heads"] * case["tokens"] > 2700000:
            case["batch" if case["batch"] > 1 else "tokens"] //= 2
        return case
    case = dict(op=op, batch=_log(rng, 1, 64), hkv=hkv, page=rng.choice([16, 32, 64, 64, 128, 256]),
                type=rng.choice(["bf16", "bf16", "e4m3"]), ragged=rng.random() < 0.7)
    if op == "append":
        case["tokens"] = rng.choice([1, _log(rng, 1, 30001)])
        case["rotate"] = rng.random() < 0.7
        while case["batch"] * hkv * case["tokens"] > 480000:
            case["batch" if case["batch"] > 1 else "tokens"] //= 2
        return case
    case["len"] = _log(rng, 1, 131071)
    while case["batch"] * hkv * case["len"] > 1000000:
        case["batch" if case["batch"] > 1 else "len"] //= 2
    if op == "decode":
        case["hq"] = hq
        case["weights"] = rng.random() < 0.4
    else:
        case["budget"] = max(1, int(case["len"] * rng.uniform(0.1, 0.6)))
        case["recent"] = int(case["budget"] * rng.uniform(0.0, 0.5))
    return case


def _lens(case, most):
    """The sequences' lengths: all alike, or spread over 1 .. most, the longest among them."""
    if not case["ragged"]:
        return [most] * case["batch"]
    return [most if b == 0 else 1 + int((most - 1) * (b * 0.6180339887 % 1.0))
            for b in range(case["batch"])]


def work(case):
    op = case["op"]
    if op == "rotary":
        n = case["batch"] * case["tokens"]
        values = n * case["heads"] * DIM
        return {"bytes": 4 * values + 4 * n * case["axes"], "flops": 3 * values}
    row = 2 * (256 if case["type"] == "bf16" else 129)  # a key and a value in the cache
    if op == "append":
        n = sum(_lens(case, case["tokens"])) * case["hkv"]
        return {"bytes": n * (512 + row), "flops": 3 * n * DIM if case["rotate"] else n * DIM}
    lens = _lens(case, case["len"])
    keys = sum(lens) * case["hkv"]
    if op == "decode":
        heads = case["batch"] * case["hq"]
        flops = 4.0 * DIM * sum(lens) * case["hq"]
        return {"bytes": keys * (row + (8 if case["weights"] else 0)) + heads * 516, "flops": flops}
    kept = sum(min(n, case["budget"]) for n in lens) * case["hkv"]
    cut = case["batch"] * case["hkv"] * case["budget"]
    return {"bytes": 4 * keys + kept * (2 * row + 4) + 4 * cut, "flops": 4 * keys}


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _cuda_ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _sections(axes):
    return {1: [64], 2: [24, 40], 3: [16, 24, 24]}[axes]


def _freqs(sections, restart, base=10000.0):
    """The rotated pairs' frequencies in radians a position: one falling series over all axes,
    or one for each axis."""
    if restart:
        return [base ** (-j / n) for n in sections for j in range(n)]
    return [base ** (-j / sum(sections)) for j in range(sum(sections))]


def _e4m3(x, square):
    """Vectors in 8 bits and the byte of their power-of-two scale: 2^(byte-127), the least with
    square <= (448 * 2^(byte-127))^2; `square` bounds the vector's largest squared value."""
    mantissa, exponent = torch.frexp(square)  # mantissa * 2^exponent, mantissa in [0.5, 1)
    e = (exponent - 18 + (mantissa > 0.765625) + 1) >> 1  # 448^2 = 0.765625 * 2^18
    e = torch.where(square > 0, e, 0).clamp(-126, 127)
    return torch.ldexp(x, -e.unsqueeze(-1)).to(E4M3), (e + 127).to(torch.uint8)


def _squares(x, s, rotate):
    """The largest squared value of each vector, and of one that is to be rotated the largest
    squared length of a rotated pair, which no angle changes."""
    x = x.float().square()
    if not rotate:
        return x.amax(-1)
    x = torch.stack([x[..., 0::2], x[..., 1::2]] if s["interleaved"] else
                    [x[..., :64], x[..., 64:]])
    return x.sum(0).amax(-1)


def _pool(case, pages, gen):
    """Pages as an earlier part of the conversation left them."""
    shape = (pages, case["hkv"], case["page"], DIM)
    k = _normal(shape, gen).mul_(1.5).add_(_normal((1, case["hkv"], 1, DIM), gen))
    v = _normal(shape, gen)
    if case["type"] == "bf16":
        return dict(k=k.bfloat16(), v=v.bfloat16())
    k, k_scale = _e4m3(k, _squares(k, case, False))
    v, v_scale = _e4m3(v, _squares(v, case, False))
    return dict(k=k, v=v, k_scale=k_scale, v_scale=v_scale)


def _tables(case, lens, gen, width):
    """Each sequence's pages, scattered over the pool; -1 behind its last one."""
    used = [-(-n // case["page"]) for n in lens]
    order = torch.randperm(sum(used) + 3, generator=gen, device="cuda").int()
    at = _cuda_ints(used).cumsum(0) - _cuda_ints(used)
    j = torch.arange(width, device="cuda")
    inside = j < _cuda_ints(used).unsqueeze(1)
    return torch.where(inside, order[torch.where(inside, at.unsqueeze(1) + j, 0)], -1), len(order)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] == "rotary":
        b, h, n = case["batch"], case["heads"], case["tokens"]
        # as a projection leaves them: token after token, the heads of a token side by side
        s["x"] = _normal((b, n, h, DIM), gen).bfloat16().transpose(1, 2)
        s["pos"] = torch.randint(0, case["far"], (case["axes"], b, n), generator=gen,
                                 device="cuda", dtype=torch.int32)
        _set_rotary(s, case["axes"], case["interleaved"], case["restart"])
    elif case["op"] == "append":
        b, h, n = case["batch"], case["hkv"], case["tokens"]
        count = _lens(case, n)
        # behind what the sequences hold already, which need not end with a page
        start = [(17 * i) % 61 for i in range(b)]
        last = [x + y for x, y in zip(start, count)]
        s["table"], pages = _tables(case, last, gen, -(-max(last) // case["page"]) + 1)
        s["cache"] = _pool(case, pages, gen)
        s["key"] = _normal((b, n, h, DIM), gen).bfloat16().transpose(1, 2)
        s["value"] = _normal((b, n, h, DIM), gen).bfloat16().transpose(1, 2)
        s["start"], s["count"] = _cuda_ints(start), _cuda_ints(count)
        if case["rotate"]:
            s["pos"] = (s["start"].unsqueeze(1) + torch.arange(n, device="cuda")).int().unsqueeze(0)
            _set_rotary(s, 1, False, False)
    else:
        lens = _lens(case, case["len"])
        width = -(-max(lens) // case["page"]) + 1
        s["lens"] = _cuda_ints(lens)
        if case["op"] == "decode":
            s["table"], pages = _tables(case, lens, gen, width)
            s["cache"] = _pool(case, pages, gen)
            s["q"] = _normal((case["batch"], case["hq"], DIM), gen).bfloat16()
        else:
            # the pages that the kept tokens move to are free ones of the same pool
            kept = [min(n, case["budget"]) for n in lens]
            both, pages = _tables(case, lens + kept, gen, width)
            s["table"] = both[:len(lens)].contiguous()
            s["new_table"] = both[len(lens):, :-(-case["budget"] // case["page"])].contiguous()
            s["cache"] = _pool(case, pages, gen)
        if case.get("weights", True):
            # a few tokens hold most of the weight, many none at all
            w = torch.rand((case["batch"], case["hkv"], width * case["page"]), generator=gen,
                           device="cuda")
            w = (w * 1.2 - 0.2).clamp_(min=0) ** 6 * 10
            s["sums"] = w * (torch.arange(w.shape[2], device="cuda") <
                             s["lens"].view(-1, 1, 1))
    if own:  # the handles that a program makes once, of the same buffers
        import paper_2503_16428_amd as X
        if "cache" in s:
            s["handle"] = X.KVCache(**s["cache"])
        if "freqs" in s:
            s["plan"] = X.Rotary(s["sections"], s["freqs"], s["interleaved"])
    return s


def _set_rotary(s, axes, interleaved, restart):
    s["sections"], s["interleaved"] = _sections(axes), interleaved
    s["freqs"] = _freqs(s["sections"], restart)
    s["freq"] = torch.tensor(s["freqs"], dtype=torch.float64, device="cuda")
    s["axis"] = torch.repeat_interleave(torch.arange(axes, device="cuda"),
                                        torch.tensor(s["sections"], device="cuda"))


def run(s):
    if own:
        return _run_own(s)
    return {"rotary": _rotary, "append": _append, "decode": _decode, "evict": _evict}[s["op"]](s)


def _run_own(s):
    import paper_2503_16428_amd as X
    if s["op"] == "rotary":
        return X.xattn_rotary(s["x"], s["pos"], s["plan"], inverse=s["inverse"])
    if s["op"] == "append":
        X.xattn_cache_append(s["key"], s["value"], s["handle"], s["table"], s["start"], s["count"],
                             pos=s.get("pos"), rotary=s.get("plan"))
        return s["cache"]
    if s["op"] == "decode":
        o, lse = X.xattn_decode(s["q"], s["handle"], s["table"], s["lens"], want_lse=True,
                                weights=s.get("sums"))
        return _answer(s, o, lse)
    kept, lens, weights = X.xattn_cache_evict(s["handle"], s["table"], s["lens"], s["sums"],
                                              s["new_table"], s["budget"], s["recent"])
    return dict(s["cache"], kept=kept, lens=lens, new_weights=weights)


def _answer(s, o, lse):
    return dict(o=o, lse=lse, weights=s["sums"]) if "sums" in s else dict(o=o, lse=lse)


# ---- the plain forms: 32 bits, elementary operations


def _turned(x, s, inverse):
    """x [batch, heads, tokens, 128] rotated by pos [axes, batch, tokens], in 32 bits. The
    angles are products of far positions: in 64 bits."""
    angle = s["pos"][s["axis"]].permute(1, 2, 0).double() * s["freq"]
    c, z = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    if inverse:
        z = -z
    if s["interleaved"]:
        a, b = x[..., 0::2].float(), x[..., 1::2].float()
        return torch.stack([a * c - b * z, a * z + b * c], -1).flatten(-2)
    a, b = x[..., :64].float(), x[..., 64:].float()
    return torch.cat([a * c - b * z, a * z + b * c], -1)


def _rotary(s):
    return _turned(s["x"], s, s["inverse"]).bfloat16()


def _append(s):
    cache, page = s["cache"], s["page"]
    key = _turned(s["key"], s, False) if s["rotate"] else s["key"].float()
    t = torch.arange(s["tokens"], device="cuda")
    b, t = torch.nonzero(t < s["count"].unsqueeze(1), as_tuple=True)
    at = s["start"][b] + t
    pages, slots = s["table"][b, at // page].long(), at % page
    for name, given, x in (("k", s["key"], key), ("v", s["value"], s["value"].float())):
        x = x[b, :, t]
        if s["type"] == "bf16":
            cache[name][pages, :, slots] = x.bfloat16()
        else:
            square = _squares(given, s, s["rotate"] and name == "k")
            x, scale = _e4m3(x, square[b, :, t])
            cache[name].view(torch.uint8)[pages, :, slots] = x.view(torch.uint8)
            cache[name + "_scale"][pages, :, slots] = scale
    return cache


def _rows(s, name, table, dtype):
    """[batch, hkv, len, 128] of a table's pages (page 0 where it has none)."""
    cache = s["cache"]
    at = table.clamp(min=0).long()
    if s["type"] == "bf16":
        x = cache[name][at].to(dtype)
    else:
        x = cache[name].view(torch.uint8)[at].view(E4M3).to(dtype)
        x = x * torch.exp2(cache[name + "_scale"][at].to(dtype) - 127).unsqueeze(-1)
    return x.transpose(1, 2).flatten(2, 3)


def _decode(s):
    b, hq, hkv = s["batch"], s["hq"], s["hkv"]
    k = _rows(s, "k", s["table"], torch.float32)
    v = _rows(s, "v", s["table"], torch.float32)
    qt = (s["q"].float() * DIM ** -0.5).view(b, hkv, hq // hkv, DIM).transpose(2, 3).contiguous()
    x = torch.matmul(k, qt).transpose(2, 3).contiguous()  # [b, hkv, group, len]
    valid = torch.arange(x.shape[3], device="cuda") < s["lens"].view(-1, 1, 1, 1)
    x = x.masked_fill(~valid, -math.inf)
    most = x.amax(-1, keepdim=True)
    p = (x - most).exp()
    total = p.sum(-1, keepdim=True)
    p = p / total
    # the pages' other rows have no weight, whatever they hold
    o = torch.matmul(p, v)
    lse = (most + total.log()).view(b, hq)
    if "sums" in s:
        s["sums"] += p.sum(2)
    return _answer(s, o.view(b, hq, DIM).bfloat16(), lse)


def _kept(s):
    """[batch, hkv, budget] positions in order, -1 behind the last."""
    w, n, budget = s["sums"], s["lens"].view(-1, 1, 1), s["budget"]
    at = torch.arange(w.shape[2], device="cuda")
    rank = torch.where(at >= n, -1.0, torch.where(at >= n - s["recent"], math.inf, w))
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    order = torch.where(torch.arange(order.shape[2], device="cuda") < n, order, w.shape[2])
    order = order.sort(-1).values
    return torch.where(order < w.shape[2], order, -1).int()


def _evict(s):
    cache, page, budget, hkv = s["cache"], s["page"], s["budget"], s["hkv"]
    kept = _kept(s)
    b, h, j = torch.nonzero(kept >= 0, as_tuple=True)
    i = kept[b, h, j].long()
    source, slot = s["table"][b, i // page].long(), i % page
    target, place = s["new_table"][b, j // page].long(), j % page
    for x in cache.values():
        x = x.view(torch.uint8) if x.dtype == E4M3 else x
        x[target, h, place] = x[source, h, slot]
    weights = torch.zeros((s["batch"], hkv, s["new_table"].shape[1] * page), device="cuda")
    weights[b, h, j] = s["sums"][b, h, i]
    return dict(cache, kept=kept, lens=s["lens"].clamp(max=budget), new_weights=weights)


# ---- the definitions in 64 bits, sequence after sequence


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _exact_turned(s, s["x"], s["inverse"])
    if case["op"] == "append":
        return _exact_append(case, s)
    if case["op"] == "decode":
        return _exact_decode(case, s)
    return _exact_evict(case, s)


def _exact_turned(s, x, inverse):
    """Pair after pair as a product of complex numbers."""
    out = x.double().contiguous()
    for i, (f, a) in enumerate(zip(s["freqs"], s["axis"].tolist())):
        phi = s["pos"][a].double().unsqueeze(1) * (-f if inverse else f)
        m, n = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + 64)
        z = torch.complex(x[..., m].double(), x[..., n].double())
        z = z * torch.polar(torch.ones_like(phi), phi)
        out[..., m], out[..., n] = z.real, z.imag
    return out


def _exact_append(case, s):
    """bf16: every value unrounded. e4m3: the rounding is the definition."""
    key = _exact_turned(s, s["key"], False) if case["rotate"] else s["key"].double()
    out = {n: x.double() if x.dtype != torch.uint8 else None for n, x in s["cache"].items()}
    for b, (first, n) in enumerate(zip(s["start"].tolist(), s["count"].tolist())):
        for j in range(first // case["page"], (first + n - 1) // case["page"] + 1):
            low, high = max(first, j * case["page"]), min(first + n, (j + 1) * case["page"])
            p, at = int(s["table"][b, j]), slice(low - j * case["page"], high - j * case["page"])
            new = slice(low - first, high - first)
            for name, x, given in (("k", key, s["key"]), ("v", s["value"].double(), s["value"])):
                x, given = x[b, :, new], given[b, :, new].double()
                if case["type"] != "bf16":
                    if case["rotate"] and name == "k":
                        given = torch.hypot(given[..., :64], given[..., 64:])
                    most = given.abs().amax(-1, keepdim=True)
                    x = (x / torch.exp2(torch.ceil(torch.log2(most / 448)))).float()
                    x = x.to(E4M3).double()
                out[name][p, :, at] = x
    return out


def _exact_decode(case, s):
    b, hq, hkv = case["batch"], case["hq"], case["hkv"]
    group = hq // hkv
    o = torch.empty((b, hq, DIM), dtype=torch.float64, device="cuda")
    lse = torch.empty((b, hq), dtype=torch.float64, device="cuda")
    w = s["sums"].double() if "sums" in s else None
    for i, n in enumerate(s["lens"].tolist()):
        table = s["table"][i:i + 1, :-(-n // case["page"])]
        k = _rows(s, "k", table, torch.float64)[0, :, :n]
        v = _rows(s, "v", table, torch.float64)[0, :, :n]
        for g in range(hkv):
            z = (s["q"][i, g * group:(g + 1) * group].double() @ k[g].T.contiguous()) / DIM ** 0.5
            lse[i, g * group:(g + 1) * group] = torch.logsumexp(z, 1)
            p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
            o[i, g * group:(g + 1) * group] = p @ v[g]
            if w is not None:
                w[i, g, :n] += p.sum(0)
    return dict(o=o, lse=lse) if w is None else dict(o=o, lse=lse, weights=w)


def _exact_evict(case, s):
    page, budget = case["page"], case["budget"]
    out = {n: x.double() if x.dtype != torch.uint8 else None for n, x in s["cache"].items()}
    new = torch.zeros((case["batch"], case["hkv"], s["new_table"].shape[1] * page),
                      dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        for h in range(case["hkv"]):
            keep = torch.arange(n, device="cuda")
            if n > budget:
                old = n - case["recent"]
                w = s["sums"][b, h, :old].double()
                take = budget - case["recent"]
                if take:
                    # the heaviest, and of those that weigh as much as the last one the first
                    least = torch.kthvalue(w, old - take + 1).values
                    same = torch.nonzero(w == least).flatten()
                    above = torch.nonzero(w > least).flatten()
                    picked = torch.cat([above, same[:take - len(above)]])
                    keep = torch.cat([picked.sort().values, keep[old:]])
                else:
                    keep = keep[old:]
            j = torch.arange(len(keep), device="cuda")
            source, target = s["table"][b, keep // page].long(), s["new_table"][b, j // page].long()
            for name in ("k", "v"):
                out[name][target, h, j % page] = out[name][source, h, keep % page]
            new[b, h, :len(keep)] = s["sums"][b, h, keep].double()
    return dict(out, kept=None, lens=None, new_weights=new)
