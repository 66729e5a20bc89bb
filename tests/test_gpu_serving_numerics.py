"""What the serving calls hold in 32 bits, seen where it shows: outputs that are
the small rest of large terms, so that their own rounding to bf16 hides nothing."""
import math

import pytest

from . import serving_oracle as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_16428_amd as X  # noqa: E402

from .serving_numerics import (cancelling, in_two_parts, rotated_in_8_bits,  # noqa: E402
                               rotated_in_fp32)
from .test_gpu_serving import bits, check_decode, decode_case, gen, ints, within  # noqa: E402


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (6, 2), (20, 1)])
@pytest.mark.parametrize("wide", [False, True])
def test_weights_enter_the_product_in_32_bits(hq, hkv, e4m3, wide):
    """Values that all but cancel: the output is their weights' error and little else."""
    batch, page = 24, 16
    q, k, v, scales, want, total = cancelling(batch, hq, hkv, page, e4m3, seed=500 + hq)
    n = 8 if e4m3 else 4
    columns = 70 if wide else 2  # rows that are shared out among workgroups; one workgroup's each
    table = torch.full((batch, columns), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(batch)
    cache = X.KVCache(k.cuda(), v.cuda(), *[s.cuda() for s in scales])
    o, _ = X.xattn_decode(q.cuda(), cache, table.cuda(), ints([n] * batch))
    # The products are exact, |z| <= 1.5 and |z - max| <= 3 in log2: two roundings of z and
    # one of the difference, 6 * 2^-24 at most in the exponent; the exponential's own 2^-22; the
    # weight's parts 2^-22; three parts of n terms, each addition off by at most a step, 2^-23;
    # sum and quotient of the end, 2^-22 of a result that is next to nothing.
    bound = total * (6 * 2.0 ** -24 + 2.0 ** -21 + 3 * n * 2.0 ** -23)
    # that bound tells weights in two bf16 parts from weights in 32 bits
    two = in_two_parts(q, k, v, scales, n)
    assert ((two - want).abs() > R.bf16_bound(want, bound)).any()
    within(o, want, R.bf16_bound(want, bound))
    assert torch.equal(bits(o), bits(X.xattn_decode(q.cuda(), cache, table.cuda(),
                                                    ints([n] * batch))[0]))


@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_of_many_rows_of_wide_groups(e4m3):
    """More than 512 rows of two tiles of heads: 512 workgroups share them."""
    lens = [(11 * i) % 23 for i in range(520)]
    check_decode(*decode_case(520, 17, 1, 16, lens, e4m3, spare=0, columns=66), lens)


@pytest.mark.parametrize("pairs,interleaved", [([64], False), ([16, 24, 24], True), ([20, 30], False)])
def test_keys_that_go_to_8_bits_are_turned_in_64(pairs, interleaved):
    """Every byte, of enough keys that turning them in 32 bits gives other ones."""
    hkv, tokens, page = 4, 6000, 64
    g = torch.Generator().manual_seed(540)
    k = (torch.randn((1, hkv, tokens, 128), generator=g) * 2.5).bfloat16()
    pos = torch.randint(0, 100000, (len(pairs), 1, tokens), generator=g, dtype=torch.int32)
    freq = R.freqs(pairs)
    least, most, scale = rotated_in_8_bits(k, pos, pairs, freq, interleaved)
    assert (bits(least) != bits(most)).double().mean() < 1e-6
    other = bits(rotated_in_fp32(k, pos, pairs, freq, interleaved))
    assert ((other != bits(least)) & (other != bits(most))).any()
    pages = -(-tokens // page)
    cache = X.KVCache.empty(pages, hkv, page, torch.float8_e4m3fn)
    table = torch.randperm(pages, generator=g).int().view(1, pages)
    X.xattn_cache_append(k.cuda(), k.cuda(), cache, table.cuda(), ints([0]), pos=pos.cuda(),
                         rotary=X.Rotary(pairs, freq, interleaved))
    order = table[0].long()
    got = bits(cache.k)[order].transpose(0, 1).reshape(hkv, -1, 128)[:, :tokens]
    byte = cache.k_scale.cpu()[order].transpose(0, 1).reshape(hkv, -1)[:, :tokens]
    assert torch.equal(byte, scale[0])
    assert ((got == bits(least)[0]) | (got == bits(most)[0])).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("power", [127, -77])
def test_values_at_the_ends_of_the_supported_range(power, e4m3, wide):
    """All values near 2^power, every weight alike in one sequence, late large products, which pass
    the first ones by up to 2^8 before they are followed, in the other; and one element the
    largest there is in every value."""
    lens = [700, 700]
    q, k, v, s, table = decode_case(2, 4, 2, 64, lens, e4m3, wide=wide)
    sign = torch.where(torch.rand(v.shape, generator=gen(580)) < 0.5, -1.0, 1.0)
    if e4m3:  # 1 .. 1.75 times 2^power, the values 256 .. 448 times 2^(power - 8)
        v = sign * 256 * (1 + 0.75 * torch.rand(v.shape, generator=gen(581)))
        v[..., 7] = 448.0
        v = v.to(k.dtype)
        s = (s[0], torch.full_like(s[1], 127 + power - 8))
    else:
        v = (sign * (1 + torch.rand(v.shape, generator=gen(581)) * 0.9)).bfloat16()
        v = (v.double() * 2.0 ** power).bfloat16()
        v[..., 7] = torch.finfo(torch.bfloat16).max * 2.0 ** (power - 127)
    k[table[0].long()] = k[table[0, 0].long(), :, :1].clone()
    if e4m3:
        s[0][table[0].long()] = s[0][table[0, 0].long(), :, :1].clone()
    q[1] = q[1].abs()
    for i in range(11):  # page after page a little larger
        k[table[1, i].long()] = (k[table[1, i].long()].float().abs() * (0.05 + 0.04 * i)).to(k.dtype)
    o, _, _ = check_decode(q, k, v, s, table, lens)
    assert torch.isfinite(o.float()).all() and (o.float().abs() > 0).any()
    most = v[0, 0, 0, 7].float() * (2.0 ** (power - 8) if e4m3 else 1)
    assert torch.equal(o[..., 7].float().cpu(), torch.full((2, 4), float(most.bfloat16())))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("at", [1, 1000003])
def test_sine_and_cosine_in_32_bits(at, interleaved):
    """Angles that turn a pair's first value to next to nothing: what is left is their error."""
    g = torch.Generator().manual_seed(590)
    for _ in range(8):
        first, second = (1 + torch.rand((2, 64), generator=g)).bfloat16()
        x = torch.stack([first, second], 1).flatten() if interleaved else torch.cat([first, second])
        turns = torch.randint(0, 4, (64,), generator=g).double() if at > 1 else torch.zeros(64)
        freq = ((torch.atan2(first.double(), second.double()) + 2 * math.pi * turns) / at).tolist()
        x, pos = x.view(1, 1, 1, 128), torch.full((1, 1, 1), at, dtype=torch.int32)
        out = X.xattn_rotary(x.cuda(), pos.cuda(), X.Rotary([64], freq, interleaved))
        want, _ = R.rotate(x, pos, [64], freq, interleaved)
        # the hardware's 1.26e-7, the turn's rounding pi 2^-25, two products and their
        # difference, half a step of 2^-23 each; angles in 64 bits 2^-51 of up to 8 pi
        both = first.double() + second.double()
        both = torch.stack([both, both], 1).flatten() if interleaved else torch.cat([both, both])
        off = both * (1.26e-7 + math.pi * 2.0 ** -25 + 3 * 2.0 ** -24 + 8 * math.pi * 2.0 ** -51)
        within(out, want, R.bf16_bound(want, off.view(want.shape)))
