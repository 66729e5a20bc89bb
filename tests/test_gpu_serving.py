"""The calls for serving after the prefill against their plain 64-bit forms
(tests/serving_oracle.py): rotary positions, the append to the paged cache, one
new token's attention, eviction; and a run of them together behind a prefill."""
import math
import random

import pytest

from . import serving_oracle as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_16428_amd as X  # noqa: E402

E4M3 = torch.float8_e4m3fn
INF, NAN = math.inf, math.nan


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=gen(seed)) * scale).bfloat16()


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def bits(t):
    kind = {2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()]
    return t.contiguous().view(kind).cpu()


def within(got, want, bound):
    err = (got.double().cpu() - want).abs()
    assert not torch.isnan(err).any()
    assert (err <= bound).all(), (err / bound.clamp(min=1e-300)).max()


# ---- rotary

PLANS = [([64], False), ([24, 40], True), ([16, 24, 24], False), ([10, 3], False), ([5, 9, 1], True)]


@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 3, 5), (1, 7, 129), (3, 2, 1000)])
@pytest.mark.parametrize("pairs,interleaved", PLANS)
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(shape, pairs, interleaved, inverse):
    b, h, n = shape
    x = normal((b, n, h, 128), 1).transpose(1, 2)
    pos = torch.randint(-5, 300000, (len(pairs), b, n), generator=gen(2), dtype=torch.int32)
    plan = X.Rotary(pairs, R.freqs(pairs), interleaved)
    xd = x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    out = X.xattn_rotary(xd, pos.cuda(), plan, inverse=inverse)
    want, before = R.rotate(x, pos, pairs, R.freqs(pairs), interleaved, inverse)
    assert out.is_contiguous()
    within(out, want, R.bf16_bound(want, before))
    # into an output of another layout, and in place
    other = torch.full((n, b, h, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    to = other.permute(1, 2, 0, 3)[..., :128]
    assert X.xattn_rotary(xd, pos.cuda(), plan, inverse=inverse, out=to) is to
    assert torch.equal(bits(to), bits(out)) and bool((other[..., 128:] == 7).all())
    X.xattn_rotary(xd, pos.cuda(), plan, inverse=inverse, out=xd)
    assert torch.equal(bits(xd), bits(out))
    if b == 1:  # without the batch dimension
        flat = X.xattn_rotary(x[0].contiguous().cuda(), pos[:, 0].contiguous().cuda(), plan,
                              inverse=inverse)
        assert torch.equal(bits(flat), bits(out[0]))


def test_rotary_at_the_farthest_positions():
    pos = torch.tensor([[[-2**31, -1, 0, 1, 2**31 - 1, 123456789]]], dtype=torch.int32)
    x = normal((1, 2, 6, 128), 3)
    plan = X.Rotary([64], R.freqs([64]))
    want, before = R.rotate(x, pos, [64], R.freqs([64]), False)
    out = X.xattn_rotary(x.cuda(), pos.cuda(), plan)
    within(out, want, R.bf16_bound(want, before))
    assert torch.equal(bits(out[:, :, 2]), bits(x[:, :, 2].cuda()))  # position 0: unturned


@pytest.mark.parametrize("interleaved", [False, True])
def test_pairs_behind_the_plan_are_copied(interleaved):
    x = normal((1, 1, 3, 128), 4)
    first = 20 if interleaved else 10
    x[..., first:64] = NAN if interleaved else INF
    if interleaved:
        x[..., 64:] = -INF
    else:
        x[..., 64 + first:] = NAN
    plan = X.Rotary([10], R.freqs([10]), interleaved)
    out = X.xattn_rotary(x.cuda(), ints([[[5, 6, 7]]]), plan).cpu()
    turned = torch.zeros(128, dtype=torch.bool)
    turned[:20 if interleaved else 10] = True
    if not interleaved:
        turned[64:74] = True
    assert torch.isfinite(out[..., turned].float()).all()
    got, given = out[..., ~turned].float(), x[..., ~turned].float()
    assert torch.equal(torch.isnan(got), torch.isnan(given))
    assert torch.equal(got.nan_to_num(0, 9, -9), given.nan_to_num(0, 9, -9))


def test_rotary_reads_broadcast_inputs():
    x = normal((1, 2, 1, 128), 5).cuda()
    pos = torch.arange(40, dtype=torch.int32).view(1, 1, 40).expand(1, 3, 40).contiguous().cuda()
    plan = X.Rotary([64], R.freqs([64]))
    wide = x.expand(3, 2, 40, 128)
    assert torch.equal(bits(X.xattn_rotary(wide, pos, plan)),
                       bits(X.xattn_rotary(wide.contiguous(), pos, plan)))


@pytest.mark.parametrize("interleaved", [False, True])
def test_inverse_is_the_gradient(interleaved):
    """d <g, R x> / dx = R^T g: the inverse call against differences of the formula."""
    x, g = normal((1, 2, 3, 128), 6), normal((1, 2, 3, 128), 7)
    pos = torch.tensor([[[3, 70, 900]], [[1, 2, 77777]]], dtype=torch.int32)
    plan = X.Rotary([30, 20], R.freqs([30, 20]), interleaved)
    got = X.xattn_rotary(g.cuda(), pos.cuda(), plan, inverse=True).double().cpu()

    def loss(y):
        out = R.rotate(y, pos, [30, 20], R.freqs([30, 20]), interleaved)[0]
        return (out * g.double()).sum((0, 1, 2, 3))

    for at in [(0, 0, 0, 0), (0, 1, 1, 17), (0, 1, 2, 64), (0, 0, 2, 101), (0, 1, 0, 127)]:
        step = torch.zeros(x.shape, dtype=torch.float64)
        step[at] = 0.5
        diff = float(loss(x.double() + step) - loss(x.double() - step))  # linear: exact
        assert abs(float(got[at]) - diff) <= abs(diff) * R.HALF_BF16 + 1e-5


# ---- append


def pool(pages, hkv, page, e4m3, seed=9):
    """A cache whose every byte is set: what a call must not touch is seen to stay."""
    g = gen(seed)
    raw = [torch.randint(0, 100, (pages, hkv, page, 128 if e4m3 else 256), generator=g,
                         dtype=torch.uint8).cuda() for _ in "kv"]
    if not e4m3:
        return X.KVCache(*[t.view(torch.bfloat16) for t in raw])
    scale = [torch.randint(120, 130, (pages, hkv, page), generator=g, dtype=torch.uint8).cuda()
             for _ in "kv"]
    return X.KVCache(*[t.view(E4M3) for t in raw], *scale)


def arrays(cache):
    return [bits(t) for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]


def scattered(pages, rows, columns, seed):
    return torch.randperm(pages, generator=gen(seed))[:rows * columns].view(rows, columns).int()


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("hkv,tokens", [(1, 1), (3, 37), (8, 130)])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("pairs,interleaved", [(None, False), ([64], False), ([20, 30], True)])
def test_append(page, hkv, tokens, e4m3, pairs, interleaved):
    batch = 4
    start, count = [0, page - 1, 5, 3], [tokens, max(0, tokens - 3), 0, tokens]
    columns = -(-(page + tokens) // page) + 1
    cache = pool(batch * columns + 2, hkv, page, e4m3)
    before = arrays(cache)
    table = scattered(batch * columns + 2, batch, columns, 11)
    k, v = (normal((batch, tokens, hkv, 128), s, 2.5).transpose(1, 2) for s in (12, 13))
    kd, vd = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (k, v))
    pos = plan = None
    if pairs:
        pos = torch.randint(0, 100000, (len(pairs), batch, tokens), generator=gen(14),
                            dtype=torch.int32)
        plan = X.Rotary(pairs, R.freqs(pairs), interleaved)
    X.xattn_cache_append(kd, vd, cache, table.cuda(), ints(start), ints(count),
                         None if pos is None else pos.cuda(), plan)
    rot, rb = (k.double(), None) if pos is None else R.rotate(k, pos, pairs, R.freqs(pairs),
                                                              interleaved)
    after = arrays(cache)
    touched = torch.zeros(before[0].shape[:3], dtype=torch.bool)
    for b in range(batch):
        for t in range(count[b]):
            p, s = int(table[b, (start[b] + t) // page]), (start[b] + t) % page
            touched[p, :, s] = True
            key, value = cache.k[p, :, s].cpu(), cache.v[p, :, s].cpu()
            if not e4m3:
                assert torch.equal(bits(value), bits(v[b, :, t]))
                if pos is None:
                    assert torch.equal(bits(key), bits(k[b, :, t]))
                else:
                    within(key, rot[b, :, t], R.bf16_bound(rot[b, :, t], rb[b, :, t]))
                continue
            want, scale, _ = R.e4m3(v[b, :, t], v[b, :, t])
            assert torch.equal(bits(value), bits(want))
            assert torch.equal(cache.v_scale[p, :, s].cpu(), scale)
            want, scale, unit = R.e4m3(rot[b, :, t], k[b, :, t], interleaved if pairs else None)
            assert torch.equal(cache.k_scale[p, :, s].cpu(), scale)
            if pos is None:
                assert torch.equal(bits(key), bits(want))
            else:  # half a step of the value, or of the least step 2^-9
                got = key.double() * unit
                bound = (rot[b, :, t].abs() * R.HALF_E4M3).clamp(min=2.0 ** -10 * unit)
                within(got, rot[b, :, t], bound + 2 * rb[b, :, t])
    for x, y in zip(before, after):
        assert torch.equal(x[~touched], y[~touched])


def test_append_without_counts_and_in_three_dimensions():
    cache, other = pool(4, 2, 16, False), pool(4, 2, 16, False)
    k, v = normal((2, 20, 128), 20).cuda(), normal((2, 20, 128), 21).cuda()
    table, start = ints([[2, 0]]), ints([7])
    X.xattn_cache_append(k, v, cache, table, start)
    X.xattn_cache_append(k[None], v[None], other, table, start, ints([1000]))  # more than there are
    assert all(torch.equal(a, b) for a, b in zip(arrays(cache), arrays(other)))
    assert torch.equal(bits(cache.k[2, :, 7:]), bits(k[:, :9]))
    assert torch.equal(bits(cache.v[0, :, :11]), bits(v[:, 9:]))


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_stores_nothing_outside_the_pages(e4m3):
    """No page, pages past the pool, places before and behind the table's row."""
    cache = pool(3, 2, 16, e4m3)
    before = arrays(cache)
    table = ints([[-1, 3], [2**31 - 1, -2**31], [1, 1], [0, 2]])
    k, v = normal((4, 2, 20, 128), 22).cuda(), normal((4, 2, 20, 128), 23).cuda()
    X.xattn_cache_append(k, v, cache, table, ints([0, 3, 32, 30]), ints([20, 20, 20, -4]))
    X.xattn_cache_append(k, v, cache, table, ints([0, 3, 2**31 - 1, -20]))
    assert all(torch.equal(a, b) for a, b in zip(before, arrays(cache)))
    X.xattn_cache_append(k, v, cache, table, ints([0, 0, 2**31 - 1, -19]))  # its last token alone
    for x, y, new in zip(arrays(cache), before, (k, v)):
        if not e4m3:
            assert torch.equal(x[0, :, 0], bits(new[3, :, 19]))
        assert not torch.equal(x[0, :, 0], y[0, :, 0])
        x[0, :, 0] = y[0, :, 0]
        assert torch.equal(x, y)


@pytest.mark.parametrize("rotated", [False, True])
def test_append_in_8_bits_at_the_ends_of_the_range(rotated):
    """Zeros, the least and the largest bf16, borders of the scale, infinities and NaN."""
    rows = torch.zeros(11, 128, dtype=torch.bfloat16)
    rows[1, 3] = 2.0 ** -133
    rows[2] = 3.0e38
    rows[3, 5], rows[3, 70] = 448.0, -1.0
    rows[4, 5] = 450.0
    rows[5, 5], rows[5, 6] = INF, 2.0
    rows[6, 5], rows[6, 6] = NAN, -3.0
    rows[7, 0], rows[7, 1], rows[7, 64] = 336.0, 296.0, 296.0  # a pair of 447.8
    rows[8] = -INF
    rows[9] = torch.arange(128).bfloat16() * 2.0 ** -130
    rows[10, 5], rows[10, 69] = 336.0, -300.0  # a pair of 450.4
    cache = pool(1, 1, 16, True)
    plan = X.Rotary([64], [0.0] * 64) if rotated else None  # rotates by nothing, by the pairs' rule
    pos = torch.zeros((1, 11), dtype=torch.int32).cuda() if rotated else None
    X.xattn_cache_append(rows[None].cuda(), rows[None].cuda(), cache, ints([[0]]), ints([0]),
                         pos=pos, rotary=plan)
    finite = [0, 1, 2, 3, 4, 7, 9, 10]
    for x, scale, rule in ((cache.k, cache.k_scale, False if rotated else None),
                           (cache.v, cache.v_scale, None)):
        want, byte, _ = R.e4m3(rows, rows, rule)
        assert torch.equal(scale[0, 0, :11].cpu(), byte)
        got = x[0, 0, :11].cpu()
        assert torch.equal(got[finite].float(), want[finite].float())
        if rule is None:
            assert torch.equal(got.float().nan_to_num(999), want.float().nan_to_num(999))


# ---- decode


def decode_case(batch, hq, hkv, page, lens, e4m3, seed=30, columns=None, spare=2, wide=False):
    """wide: a table of more than 1024 tokens, whose rows are shared out among workgroups; short
    ones are one workgroup's each."""
    columns = columns or max(1, -(-max(lens) // page)) + 1
    if wide:
        columns = max(columns, 1040 // page + 1)
    pages = batch * columns + spare
    g = gen(seed)
    k = torch.randn((pages, hkv, page, 128), generator=g) * 1.3
    v = torch.randn((pages, hkv, page, 128), generator=g) + 0.3
    scales = ()
    if e4m3:
        k, ks, _ = R.e4m3(k, k)
        v, vs, _ = R.e4m3(v, v)
        scales = (ks, vs)
    else:
        k, v = k.bfloat16(), v.bfloat16()
    q = normal((batch, hq, 128), seed + 1, 1.5)
    table = scattered(pages, batch, columns, seed + 2)
    return q, k, v, scales, table


def on_gpu(k, v, scales):
    return X.KVCache(k.cuda(), v.cuda(), *[s.cuda() for s in scales])


def check_decode(q, k, v, scales, table, lens, weights=True):
    cache = on_gpu(k, v, scales)
    hkv, capacity = k.shape[1], table.shape[1] * k.shape[2]
    w0 = torch.rand((q.shape[0], hkv, capacity), generator=gen(77))
    w = w0.cuda() if weights else None
    o, lse = X.xattn_decode(q.cuda(), cache, table.cuda(), ints(lens), weights=w, want_lse=True)
    wo, wl, ww, ob, lb, wb = R.decode(q, k, v, table, lens, *scales)
    within(o, wo, R.bf16_bound(wo, ob))
    empty = wl == -INF
    assert torch.equal(lse.cpu() == -INF, empty)
    assert (bits(o)[empty] == 0).all()
    within(lse.cpu()[~empty], wl[~empty], lb[~empty])
    if weights:
        total = w0.double() + ww
        within(w, total, wb + total * 2.0 ** -24 + 1e-30)
        for b, n in enumerate(lens):
            n = min(max(n, 0), capacity)
            assert torch.equal(w[b, :, n:].cpu(), w0[b, :, n:])
    # without weights and lse, into given outputs, on a workspace full of NaN
    need = X.decode_workspace_size(cache, q.shape[0], q.shape[1], table.shape[1])
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    to = torch.full_like(q.cuda(), NAN)
    o2, none = X.xattn_decode(q.cuda(), cache, table.cuda(), ints(lens), o=to, workspace=ws)
    assert o2 is to and none is None and torch.equal(bits(to), bits(o))
    return o, lse, w


WIDE = pytest.mark.parametrize("wide", [False, True])


@WIDE
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1), (7, 1), (16, 1), (17, 1), (40, 1), (6, 3), (8, 8)])
def test_decode_heads(hq, hkv, e4m3, wide):
    lens = [77, 1, 300]
    check_decode(*decode_case(3, hq, hkv, 16, lens, e4m3, wide=wide), lens)


@WIDE
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_decode_lengths(page, e4m3, wide):
    lens = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, page, page + 1, 2 * page - 1]
    check_decode(*decode_case(len(lens), 4, 2, page, lens, e4m3, wide=wide), lens)


@WIDE
def test_decode_without_keys(wide):
    for lens in ([0], [0, 0, 0]):
        check_decode(*decode_case(len(lens), 40, 2, 16, lens, False, wide=wide), lens)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv,lens,page", [(4, 2, [5000], 64), (8, 1, [1, 2999, 777], 32),
                                              (4, 4, [4096, 4095, 0], 128), (24, 1, [2049], 16)])
def test_decode_long(hq, hkv, lens, page, e4m3):
    check_decode(*decode_case(len(lens), hq, hkv, page, lens, e4m3), lens)


@WIDE
def test_decode_of_many_short_sequences(wide):
    lens = [(37 * i) % 90 for i in range(150)]
    check_decode(*decode_case(150, 4, 1, 16, lens, False, wide=wide), lens)


@pytest.mark.parametrize("columns", [32, 33, 48, 49, 64, 65])
@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_around_the_lengths_of_whole_rows(columns, e4m3):
    """Tables of 512, 768, 1024 and a page more tokens, few rows and many."""
    for batch in (2, 64):
        lens = [columns * 16 - (13 * i) % (columns * 16) for i in range(batch)]
        check_decode(*decode_case(batch, 4, 2, 16, lens, e4m3, columns=columns), lens)


@pytest.mark.parametrize("columns", [13, 66])
def test_decode_of_more_sequences_than_lanes(columns):
    lens = [(7 * i) % 5 if i % 97 else 200 for i in range(1000)]
    check_decode(*decode_case(1000, 1, 1, 16, lens, False, spare=0, columns=columns), lens)


@pytest.mark.parametrize("seed", range(24))
def test_decode_of_random_shapes(seed):
    rng = random.Random(seed)
    hkv = rng.choice([1, 1, 2, 3, 5, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 7, 8, 15, 16, 18, 32, 33, 65])
    page, batch = rng.choice([16, 32, 64, 128, 256]), rng.choice([1, 2, 3, 7, 20, 70])
    most = int(math.exp(rng.uniform(0, math.log(40000 / batch / max(1, hq // 16)))))
    lens = [rng.choice([0, 1, most, rng.randint(0, most)]) for _ in range(batch)]
    lens[rng.randrange(batch)] = most
    print(f"{batch=} {hq=} {hkv=} {page=} {most=}", flush=True)
    q, k, v, s, table = decode_case(batch, hq, hkv, page, lens, rng.random() < 0.5, seed=300 + seed)
    if rng.random() < 0.3:
        table[torch.rand(table.shape, generator=gen(400 + seed)) < 0.1] = -1
    check_decode(q, k, v, s, table, lens)


def test_decode_of_lengths_past_the_table():
    """Lengths outside 0 .. capacity count as its ends."""
    q, k, v, s, table = decode_case(3, 4, 2, 16, [48], False, columns=3)
    a = check_decode(q, k, v, s, table, [49, -7, 2**31 - 1])
    b = check_decode(q, k, v, s, table, [48, 0, 48])
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(a, b))


@WIDE
@pytest.mark.parametrize("e4m3", [False, True])
def test_what_lies_behind_a_length_has_no_effect(e4m3, wide):
    lens = [5, 0, 83, 64]
    q, k, v, s, table = decode_case(4, 4, 2, 32, lens, e4m3, wide=wide)
    clean = check_decode(q, k, v, s, table, lens)
    used = torch.zeros(k.shape[0], k.shape[2], dtype=torch.bool)
    for b, n in enumerate(lens):
        for t in range(n):
            used[int(table[b, t // 32]), t % 32] = True
    free = ~used.unsqueeze(1).expand(k.shape[:3])
    for bad in ((NAN, NAN) if e4m3 else (INF, NAN)), (NAN, 448.0):
        k2, v2, s2 = k.clone(), v.clone(), [x.clone() for x in s]
        for x, y in zip((k2, v2), bad):
            f = x.float()
            f[free] = y
            x.copy_(f.to(x.dtype))
        for x in s2:
            x[free] = 255
        t2 = table.clone()  # and columns behind the last page hold nonsense
        for b, n in enumerate(lens):
            t2[b, -(-n // 32):] = 2**31 - 1
        dirty = X.xattn_decode(q.cuda(), on_gpu(k2, v2, s2), t2.cuda(), ints(lens), want_lse=True)
        assert torch.equal(bits(dirty[0]), bits(clean[0]))
        assert torch.equal(bits(dirty[1]), bits(clean[1]))


@WIDE
@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_skips_missing_pages(e4m3, wide):
    lens = [100, 64, 40]
    q, k, v, s, table = decode_case(3, 4, 2, 16, lens, e4m3, wide=wide)
    table[0, 1], table[0, 5] = -1, k.shape[0]
    table[1, :] = -2**31          # a row without a key
    table[2, 0] = 2**31 - 1
    check_decode(q, k, v, s, table, lens)


@WIDE
def test_products_of_minus_infinity_have_no_weight(wide):
    lens = [40, 20]
    q, k, v, s, table = decode_case(2, 4, 1, 16, lens, False, wide=wide)
    q = q.abs() + 0.5
    k[table[0, 0], :, :] = -INF                  # the first sequence's first page
    v[table[0, 0], 0, 3] = 7.0
    k[table[1, 0]], k[table[1, 1]] = -INF, -INF  # every key of the second
    check_decode(q, k, v, s, table, lens)


@WIDE
def test_infinite_and_nan_products_reach_their_own_row_only(wide):
    lens = [40, 40, 40]
    q, k, v, s, table = decode_case(3, 4, 1, 16, lens, False, wide=wide)
    clean = X.xattn_decode(q.cuda(), on_gpu(k, v, s), table.cuda(), ints(lens), want_lse=True)
    k[table[1, 1], 0, 4] = NAN
    v[table[2, 0], 0, 5, 9] = INF
    o, lse = X.xattn_decode(q.cuda(), on_gpu(k, v, s), table.cuda(), ints(lens), want_lse=True)
    assert torch.isnan(o[1].float()).all() and torch.isnan(lse[1]).all()
    assert torch.equal(bits(o[0]), bits(clean[0][0])) and torch.equal(bits(lse[0]), bits(clean[1][0]))
    assert torch.isinf(o[2, :, 9].float()).all() and torch.equal(bits(lse[2]), bits(clean[1][2]))
    rest = torch.arange(128) != 9
    assert torch.equal(bits(o[2].cpu()[:, rest]), bits(clean[0][2].cpu()[:, rest]))


@WIDE
def test_large_products_and_weights_of_one_key(wide):
    """One key far above the rest, late and early, and keys alike."""
    lens = [300, 300, 33]
    q, k, v, s, table = decode_case(3, 4, 2, 64, lens, False, wide=wide)
    q[0], q[1] = q[0].abs() * 4, q[1].abs() * 4
    k[table[0, 4], :, 20] = 30.0
    k[table[1, 0], :, 0] = 30.0
    k[table[2, 0]] = k[table[2, 0], :, :1]
    check_decode(q, k, v, s, table, lens)


def test_several_new_tokens_are_rows_that_share_pages():
    q, k, v, s, table = decode_case(1, 8, 2, 32, [400], False)
    rows = 5
    many = normal((rows, 8, 128), 50, 1.5)
    o, lse, _ = check_decode(many, k, v, s, table.expand(rows, -1).contiguous(),
                             [400 - rows + 1 + i for i in range(rows)])
    one = X.xattn_decode(many[2:3].cuda(), on_gpu(k, v, s), table.cuda(), ints([398]))[0]
    assert (one.float() - o[2:3].float()).abs().max() <= 2.0 ** -6


def test_decode_is_deterministic_and_follows_its_stream():
    lens = [3000, 1500]
    q, k, v, s, table = decode_case(2, 8, 2, 64, lens, False)
    cache, qd, td, ld = on_gpu(k, v, s), q.cuda(), table.cuda(), ints(lens)
    w = torch.zeros((2, 2, table.shape[1] * 64), device="cuda")
    ref = X.xattn_decode(qd, cache, td, ld, weights=w, want_lse=True)
    torch.cuda.synchronize()
    for _ in range(3):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        w2 = torch.zeros_like(w)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            q2 = qd.clone()
        o, lse = X.xattn_decode(q2, cache, td, ld, weights=w2, want_lse=True, stream=side)
        with torch.cuda.stream(side):
            q2.zero_()  # behind the call
        # what the call allocated is not handed out on the current stream meanwhile
        torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
        side.synchronize()
        assert torch.equal(bits(o), bits(ref[0])) and torch.equal(bits(lse), bits(ref[1]))
        assert torch.equal(w2, w)


def test_two_calls_at_once():
    """Different batches on two streams, each with its own workspace: the results of each alone."""
    cases = []
    for i, (lens, e4m3) in enumerate((([3000, 10, 777], False), ([2500, 2500], True))):
        q, k, v, s, table = decode_case(len(lens), 8, 2, 64, lens, e4m3, seed=200 + i)
        w = torch.rand((len(lens), 2, table.shape[1] * 64), generator=gen(210 + i))
        cases.append((q.cuda(), on_gpu(k, v, s), table.cuda(), ints(lens), w))
    alone = []
    for q, cache, table, lens, w in cases:
        u = w.cuda()
        alone.append((*X.xattn_decode(q, cache, table, lens, weights=u, want_lse=True), u))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    held = [w.cuda() for *_, w in cases]
    torch.cuda.synchronize()
    outs = [X.xattn_decode(q, cache, table, lens, weights=u, want_lse=True, stream=st)
            for (q, cache, table, lens, _), u, st in zip(cases, held, streams)]
    torch.cuda.synchronize()
    for (o, lse, w), (o2, lse2), w2 in zip(alone, outs, held):
        assert torch.equal(bits(o), bits(o2)) and torch.equal(lse, lse2) and torch.equal(w, w2)


def test_scales_far_apart():
    """Values of one vector are alike in size, those of different tokens 2^60 apart."""
    lens = [130, 33]
    q, k, v, s, table = decode_case(2, 6, 2, 16, lens, True)
    g = gen(220)
    ks = s[0].clone()
    ks[torch.rand(ks.shape, generator=g) < 0.5] -= 40  # products of next to nothing
    vs = (s[1].int() + torch.randint(-30, 31, s[1].shape, generator=g)).to(torch.uint8)
    check_decode(q, k, v, (ks, vs), table, lens)


def test_workspaces_may_hold_anything():
    lens = [900, 0, 77, 2000]
    q, k, v, s, table = decode_case(4, 20, 1, 32, lens, False, columns=520)
    cache, qd, td, ld = on_gpu(k, v, s), q.cuda(), table.cuda(), ints(lens)
    w0 = torch.rand((4, 1, table.shape[1] * 32), generator=gen(230)).cuda()
    new_table = torch.zeros((4, 8), dtype=torch.int32, device="cuda") - 1  # nothing is moved
    want = None
    for fill in (0, 255, 127, 1):
        ws = torch.full((X.decode_workspace_size(cache, 4, 20, table.shape[1], True),), fill,
                        dtype=torch.uint8, device="cuda")
        es = torch.full((X.evict_workspace_size(cache, 4, table.shape[1]),), fill,
                        dtype=torch.uint8, device="cuda")
        w = w0.clone()
        got = (*X.xattn_decode(qd, cache, td, ld, weights=w, want_lse=True, workspace=ws), w,
               *X.xattn_cache_evict(cache, td, ld, w0, new_table, 200, 7, workspace=es))
        want = want or got
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want)), fill


def test_projections_are_read_where_they_are():
    """q, k and v as slices of one projection's output [batch, tokens, heads, 128]."""
    qkv = normal((2, 9, 8 + 2 + 2, 128), 240).cuda()
    q, k, v = (t.transpose(1, 2) for t in qkv.split([8, 2, 2], dim=2))
    pos = torch.arange(9, dtype=torch.int32).expand(1, 2, 9).contiguous().cuda()
    plan = X.Rotary([64], R.freqs([64]))
    assert torch.equal(bits(X.xattn_rotary(q, pos, plan)),
                       bits(X.xattn_rotary(q.contiguous(), pos, plan)))
    one, two = pool(3, 2, 16, False), pool(3, 2, 16, False)
    table, start = ints([[0], [2]]), ints([0, 7])
    X.xattn_cache_append(k, v, one, table, start, pos=pos, rotary=plan)
    X.xattn_cache_append(k.contiguous(), v.contiguous(), two, table, start, pos=pos, rotary=plan)
    assert all(torch.equal(a, b) for a, b in zip(arrays(one), arrays(two)))
    before = qkv.clone()
    X.xattn_rotary(q, pos, plan, out=q)  # in place, the keys and values beside it untouched
    assert torch.equal(bits(qkv[:, :, 8:]), bits(before[:, :, 8:]))
    with pytest.raises(X.XAttnError):
        X.xattn_rotary(q, pos, plan, out=qkv.view(-1)[:q.numel()].view(q.shape))


def test_decode_offsets_past_32_bits():
    """A pool of more than 2^31 values: its last pages hold the sequence."""
    page, hkv = 256, 8
    pages = (1 << 31) // (page * hkv * 128) + 40
    q, k, v, _, table = decode_case(1, 8, hkv, page, [600], False, spare=0)
    big = X.KVCache.empty(pages, hkv, page)
    n = k.shape[0]
    big.k[-n:], big.v[-n:] = k.cuda(), v.cuda()
    o, lse = X.xattn_decode(q.cuda(), big, (table + pages - n).cuda(), ints([600]), want_lse=True)
    want, wl, _, ob, lb, _ = R.decode(q, k, v, table, [600])
    within(o, want, R.bf16_bound(want, ob))
    within(lse, wl, lb)
    # and the append writes there
    new = normal((1, hkv, 3, 128), 60).cuda()
    X.xattn_cache_append(new, new, big, (table + pages - n).cuda(), ints([10]))
    at = int(table[0, 0]) + pages - n
    assert torch.equal(bits(big.k[at, :, 10:13]), bits(new[0]))
    assert torch.equal(bits(big.v[at, :, 10:13]), bits(new[0]))


# ---- eviction


def check_evict(weights, lens, page, hkv, budget, recent, e4m3, hole=None, seed=70):
    batch, columns = len(lens), weights.shape[2] // page
    new_columns = -(-budget // page) + 1
    pages = batch * (columns + new_columns) + 3
    cache = pool(pages, hkv, page, e4m3, seed)
    order = torch.randperm(pages, generator=gen(seed)).int()
    table = order[:batch * columns].view(batch, columns).clone()
    new_table = order[batch * columns:batch * (columns + new_columns)].view(batch, new_columns).clone()
    if hole:
        table[0, hole[0]], new_table[0, hole[1]] = -1, 2**31 - 1
    before = arrays(cache)
    given = weights.cuda()
    kept, new_lens, new_w = X.xattn_cache_evict(cache, table.cuda(), ints(lens), given,
                                                new_table.cuda(), budget, recent)
    want = [x.clone() for x in before]
    for b, n in enumerate(lens):
        n = min(max(n, 0), columns * page)
        assert int(new_lens[b]) == min(n, budget)
        for h in range(hkv):
            at = R.keep(weights[b, h], n, budget, recent)
            assert kept[b, h].tolist() == at + [-1] * (budget - len(at))
            w = torch.zeros(new_columns * page)
            w[:len(at)] = weights[b, h, at]
            assert torch.equal(bits(new_w[b, h]), bits(w))
            for j, t in enumerate(at):
                p, r = int(table[b, t // page]), int(new_table[b, j // page])
                if 0 <= p < pages and 0 <= r < pages:
                    for x, y in zip(want, before):
                        x[r, h, j % page] = y[p, h, t % page]
    assert all(torch.equal(x, y) for x, y in zip(want, arrays(cache)))
    assert torch.equal(bits(given), bits(weights))
    return kept


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page,lens,budget,recent", [
    (16, [0, 1, 5, 47], 5, 2), (16, [48], 48, 3), (16, [48], 1, 0), (16, [48], 1, 1),
    (32, [90, 64, 17], 33, 0), (32, [96, 50], 20, 20), (64, [1000, 3], 100, 37),
    (256, [2500], 1100, 30), (16, [80, -3, 2**31 - 1], 7, 3)])
def test_evict(page, lens, budget, recent, e4m3):
    columns = max(-(-min(n, 3000) // page) for n in lens) + (lens[0] != 80)
    w = torch.rand((len(lens), 3, columns * page), generator=gen(71)).clamp(min=0.3)  # many alike
    check_evict(w, lens, page, 3, budget, recent, e4m3)


def test_evict_orders_every_float():
    """Zeros of both signs alike, infinities, subnormals, negatives, NaN below all."""
    special = [0.0, -0.0, INF, -INF, NAN, 1e-45, -1e-45, 3e38, -3e38, 1.0, 1.0 + 2**-23, -1.0]
    w = torch.tensor((special * 12)[:144]).view(1, 1, 144)[..., torch.randperm(144, generator=gen(72))]
    for budget in (1, 11, 12, 13, 40, 60, 61, 120, 131, 132, 133, 143):
        check_evict(w.contiguous(), [144], 16, 1, budget, 0, False)
        check_evict(w.contiguous(), [141], 16, 1, budget, min(budget, 9), False)


def test_evict_of_weights_alike():
    for value in (0.0, 0.25, NAN):
        kept = check_evict(torch.full((1, 2, 4096), value), [4001], 64, 2, 1500, 100, False)
        assert kept[0, 0].tolist() == list(range(1400)) + list(range(3901, 4001))


@pytest.mark.parametrize("kind", ["spread", "alike", "one digit"])
def test_evict_of_long_rows(kind):
    """Rows of several workgroups: lengths around their borders, the last place in any of them."""
    lens = [20001, 8193, 8192, 5001, 16384, 100]
    g = gen(74)
    w = torch.rand((6, 1, 20032), generator=g)
    if kind == "alike":
        w = (w * 8).floor()
    elif kind == "one digit":  # weights whose upper 11 bits are the same
        w = 1.0 + w * 2.0 ** -4
    for columns in (313, 257, 256, 129, 128):  # by three launches from 257 on, else by one
        x, n = w[..., :64 * columns].contiguous(), [min(n, 64 * columns) for n in lens]
        check_evict(x, n, 64, 1, 5000, 37, kind == "alike")
    check_evict(w, lens, 64, 1, 90, 0, False)
    check_evict(w[:1, :, :16000].contiguous(), [15990], 64, 1, 15989, 0, False)


@pytest.mark.parametrize("columns", [24, 300])
@pytest.mark.parametrize("unit", [None, 2.0 ** -13, 2.0 ** -23])
def test_evict_of_whole_groups(unit, columns):
    """Weights in groups of seven that differ in their upper 11, 22 or 32 bits only, the last place
    at a group's end, before and behind it; and the same with some of every group a little more."""
    n = columns * 64 - 5
    at = torch.randperm(columns * 64, generator=gen(76))
    group = (at // 7).float().view(1, 1, -1)
    w = 1 + group * unit if unit else torch.exp2(-group.clamp(max=100))
    more = w * (1 + 2.0 ** -22 * (at % 3).float().view(1, 1, -1))
    for x in (w, more):
        ranked = x[0, 0, :n].sort(descending=True).values
        ends = (torch.nonzero(ranked[1:] != ranked[:-1]).flatten() + 1).tolist()
        for end in (ends[0], ends[40]):
            for budget in (end - 1, end, end + 1):
                check_evict(x, [n], 64, 1, max(budget, 1), 0, False)
    check_evict(-w, [n], 64, 1, 777, 0, True)


@pytest.mark.parametrize("seed", range(12))
def test_evict_of_random_shapes(seed):
    rng = random.Random(500 + seed)
    page, batch, hkv = rng.choice([16, 64, 256]), rng.choice([1, 2, 5]), rng.choice([1, 2, 3])
    most = int(math.exp(rng.uniform(math.log(2), math.log(24000 / batch / hkv))))
    lens = [most] + [rng.randint(0, most) for _ in range(batch - 1)]
    budget = rng.randint(1, min(most, 3000))
    print(f"{batch=} {hkv=} {page=} {lens=} {budget=}", flush=True)
    columns = -(-most // page) + rng.randint(0, 2)
    w = torch.randn((batch, hkv, columns * page), generator=gen(600 + seed))
    if rng.random() < 0.5:
        w = w.clamp(min=0)  # half of them alike
    check_evict(w, lens, page, hkv, budget, rng.randint(0, budget), rng.random() < 0.5)


def test_evict_with_missing_pages():
    w = torch.rand((2, 2, 128), generator=gen(73))
    check_evict(w, [120, 100], 16, 2, 50, 10, False, hole=(2, 1))
    check_evict(w, [120, 100], 16, 2, 50, 10, True, hole=(0, 2))


# ---- together


@pytest.mark.parametrize("columns", [8, 66])
def test_graph_of_a_decoding_step_replays_like_eager(columns):
    """Rotation, append, attention with weights and eviction in one captured step, on new inputs
    and lengths at every replay; two graphs share a workspace. Rows of one workgroup, and shared
    ones."""
    batch, hq, hkv, page = 3, 8, 2, 16
    lens = [60, 33, 0]
    q, k, v, s, table = decode_case(batch, hq, hkv, page, lens, False, columns=columns, spare=40)
    plan = X.Rotary([64], R.freqs([64]))
    free = [p for p in range(k.shape[0]) if p not in table.flatten().tolist()]
    new_table = torch.tensor(free[:batch * 2]).view(batch, 2).int().cuda()
    td = table.cuda()

    def fresh():
        return on_gpu(k, v, s), torch.zeros((batch, hkv, columns * page), device="cuda")

    def step(cache, w, x, key, value, pos, start, ln, ws):
        X.xattn_rotary(x, pos, plan, out=x)
        X.xattn_cache_append(key, value, cache, td, start, pos=pos, rotary=plan)
        o, lse = X.xattn_decode(x[:, :, 0], cache, td, ln, weights=w, want_lse=True, workspace=ws)
        return (o, lse, *X.xattn_cache_evict(cache, td, ln, w, new_table, 20, 5))

    def inputs(i):
        return dict(x=normal((batch, hq, 1, 128), 80 + i).cuda(),
                    key=normal((batch, hkv, 1, 128), 90 + i).cuda(),
                    value=normal((batch, hkv, 1, 128), 100 + i).cuda(),
                    pos=ints([[[n + i] for n in lens]]), start=ints([n + i for n in lens]),
                    ln=ints([n + i + 1 for n in lens]))

    probe, _ = fresh()
    ws = torch.empty(X.decode_workspace_size(probe, batch, hq, columns, True), dtype=torch.uint8,
                     device="cuda")
    eager_cache, eager_w = fresh()
    graphs = []
    for _ in range(2):
        cache, w = fresh()
        held = inputs(0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            warm_cache, warm_w = fresh()
            step(warm_cache, warm_w, **{n: t.clone() for n, t in held.items()}, ws=ws)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(cache, w, **held, ws=ws)
        torch.cuda.synchronize()
        graphs.append((g, held, out, cache, w))
    for i in range(4):
        new = inputs(i)
        want = step(eager_cache, eager_w, **{n: t.clone() for n, t in new.items()}, ws=None)
        torch.cuda.synchronize()
        for g, held, out, cache, w in graphs:
            for n, t in new.items():
                held[n].copy_(t)
            g.replay()
        torch.cuda.synchronize()
        for g, held, out, cache, w in graphs:
            for a, b in zip(out, want):
                assert torch.equal(bits(a), bits(b)), i
            assert torch.equal(w, eager_w), i
            assert all(torch.equal(a, b) for a, b in zip(arrays(cache), arrays(eager_cache))), i


@pytest.mark.parametrize("e4m3", [False, True])
def test_prefill_then_answer(e4m3):
    """A prompt of 256 tokens through the dense prefill on rotated heads, its last token again
    through the cache; three more tokens; eviction; two more. Lengths, positions and pages as a
    server keeps them, every step against the plain forms on the call's own cache."""
    hq, hkv, page, L = 8, 2, 64, 256
    plan, pairs = X.Rotary([64], R.freqs([64])), [64]
    q, k, v = (normal((1, L, h, 128), s).cuda().transpose(1, 2)
               for h, s in ((hq, 110), (hkv, 111), (hkv, 112)))
    pos = torch.arange(L, dtype=torch.int32).view(1, 1, L).cuda()
    qr, kr = X.xattn_rotary(q, pos, plan), X.xattn_rotary(k, pos, plan)
    prefill, _ = X.xattn_dense_attn(qr, kr, v.contiguous())
    cache = X.KVCache.empty(24, hkv, page, torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    table = scattered(16, 1, 8, 113).cuda()
    X.xattn_cache_append(k, v, cache, table, ints([0]), pos=pos, rotary=plan)
    w = torch.zeros((1, hkv, 8 * page), device="cuda")

    def host():
        s = () if not e4m3 else (cache.k_scale.cpu(), cache.v_scale.cpu())
        return (cache.k.cpu(), cache.v.cpu()), s

    def attend(x, table, length, w):
        before = w.cpu().double()
        o, lse = X.xattn_decode(x, cache, table, ints([length]), weights=w, want_lse=True)
        (kk, vv), s = host()
        wo, wl, ww, ob, lb, wb = R.decode(x.cpu(), kk, vv, table.cpu(), [length], *s)
        within(o, wo, R.bf16_bound(wo, ob))
        within(lse, wl, lb)
        within(w, before + ww, wb + (before + ww) * 2.0 ** -24)
        return o

    o = attend(qr[:, :, -1].contiguous(), table, L, w)
    # the prefill rounds P to bf16 (half a step of it), its output once, as o is
    if not e4m3:
        gap = (o.float() - prefill[:, :, -1].float()).abs().max()
        assert gap <= 3 * R.HALF_BF16 * v.float().abs().max()
    length, where = L, L
    for i in range(5):
        if i == 3:
            new_table = torch.tensor([[20, 21, 22, 23]], dtype=torch.int32).cuda()
            kept, lens, w = X.xattn_cache_evict(cache, table, ints([length]), w, new_table, 150, 32)
            assert int(lens[0]) == 150 and kept[0, 0, -32:].tolist() == list(range(length - 32, length))
            table, length = new_table, 150
        x, key, value = (normal((1, h, 1, 128), 120 + 3 * i + j).cuda()
                         for j, h in enumerate((hq, hkv, hkv)))
        at = ints([[[where]]])
        x = X.xattn_rotary(x, at, plan)
        X.xattn_cache_append(key, value, cache, table, ints([length]), pos=at, rotary=plan)
        length, where = length + 1, where + 1
        attend(x[:, :, 0].contiguous(), table, length, w)
