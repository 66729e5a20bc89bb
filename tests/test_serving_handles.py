"""Handles of the serving calls and the numbers and tensors that go to C as they are,
on the CPU: what would reach a kernel as something else than was given is refused."""
import ctypes

import pytest
import torch

import paper_2503_16428_amd as X
from paper_2503_16428_amd import binding as B

from .test_serving_checks import HostCache, bf, c_cache, expect, i32


def test_a_cache_keeps_its_arrays():
    """Its C struct holds their addresses: another tensor in their place would not be used, and
    the memory that is used could belong to someone else by then."""
    c = HostCache()
    k, ref = c.k, c._ref
    for name, value in (("k", bf(8, 2, 16, 128)), ("v", bf(8, 2, 16, 128)), ("k_scale", None),
                        ("pages", 8), ("hkv", 1), ("page", 32), ("e4m3", True), ("device", None),
                        ("_ref", None)):
        expect("is fixed", setattr, c, name, value)
    expect("is fixed", delattr, c, "k")
    c.owner = "a program's own attribute"
    del c.owner
    assert c.k is k and c._ref is ref and c.pages == 4


def test_a_plan_keeps_its_pairs():
    plan = X.Rotary([16, 24, 24], X.rotary_freqs([16, 24, 24]))
    for name in ("axes", "pairs", "interleaved", "_freq", "_plan"):
        expect("is fixed", setattr, plan, name, 1)
    assert plan.axes == 3 and plan.pairs == (16, 24, 24) and not plan.interleaved


@pytest.mark.parametrize("recent", [2**32, 2**32 + 1, -1, 5, -2**32 + 1])
def test_recent_is_checked_before_it_is_32_bits(recent):
    expect("recent must be", X.xattn_cache_evict, HostCache(), i32(3, 2), i32(3),
           torch.zeros(3, 2, 32), i32(3, 1), 4, recent)


def test_sizes_are_checked_before_they_are_32_bits():
    c = HostCache()
    assert X.decode_workspace_size(c, 1, 4, 100) > 0 and X.evict_workspace_size(c, 1, 2000) > 0
    for n in (2**32 + 1, 2**31, -2**32 + 1):
        for sizes in ((n, 4, 100), (1, n, 100), (1, 4, n)):
            expect("must fit 32 bits", X.decode_workspace_size, c, *sizes)
        for sizes in ((n, 2000), (1, n)):
            expect("must fit 32 bits", X.evict_workspace_size, c, *sizes)


def test_tensors_that_a_call_needs_are_missed():
    c, table, k = HostCache(), i32(3, 2), bf(3, 2, 5, 128)
    plan = X.Rotary([64], X.rotary_freqs([64]))
    expect("pos must be given", X.xattn_rotary, k, None, plan)
    expect("start must be given", X.xattn_cache_append, k, k, c, table, None)
    expect("lens must be given", X.xattn_decode, bf(3, 4, 128), c, table, None)
    w, new = torch.zeros(3, 2, 32), i32(3, 1)
    expect("lens must be given", X.xattn_cache_evict, c, table, None, w, new, 4, 1)
    expect("weights must be given", X.xattn_cache_evict, c, table, i32(3), None, new, 4, 1)


# ---- arrays that share memory (addresses that are never used: every call is refused)

POOL = ("k", "v", "k_scale", "v_scale")
on_the_cpu = pytest.mark.skipif(torch.cuda.is_available(), reason="calls with made-up addresses")


def _laid_out(sizes):
    """An address for each array, more between them than the largest has."""
    return {name: (i + 1) << 32 for i, name in enumerate(sizes)}


def _decode(cache, at, sizes):
    return X.lib().xattn_decode(at["q"], cache, 2, 4, at["table"], 100, at["lens"], at["o"],
                                at["lse"], at["weights"], at["workspace"], sizes["workspace"], None)


def _evict(cache, at, sizes):
    return X.lib().xattn_cache_evict(cache, 2, at["table"], 1100, at["lens"], at["weights"], 20, 3,
                                     at["new_table"], 2, at["kept"], at["new_lens"],
                                     at["new_weights"], at["workspace"], sizes["workspace"], None)


def _cases():
    """(call, sizes, written): two sequences, 4 / 2 heads, pages of 16, an 8-bit cache of 300."""
    pool = dict(k=300 * 2 * 16 * 128, v=300 * 2 * 16 * 128, k_scale=300 * 2 * 16,
                v_scale=300 * 2 * 16)
    n = ctypes.c_size_t(0)
    cache = c_cache(pages=300, type=1)
    assert X.lib().xattn_decode_workspace_size(cache, 2, 4, 100, 1, ctypes.byref(n)) == 0
    yield _decode, dict(pool, q=2048, table=800, lens=8, o=2048, lse=32, weights=2 * 2 * 1600 * 4,
                        workspace=n.value), ("o", "lse", "weights", "workspace")
    assert X.lib().xattn_evict_workspace_size(cache, 2, 1100, ctypes.byref(n)) == 0
    yield _evict, dict(pool, table=8800, lens=8, weights=2 * 2 * 17600 * 4, new_table=16,
                       kept=2 * 2 * 20 * 4, new_lens=8, new_weights=2 * 2 * 32 * 4,
                       workspace=n.value), ("kept", "new_lens", "new_weights", "workspace")


@on_the_cpu
@pytest.mark.parametrize("which", [0, 1])
def test_written_arrays_share_no_memory(which):
    """Every written array against every other, at its first and its last 16 bytes."""
    call, sizes, written = list(_cases())[which]
    for a in written:
        for b in sizes:
            for first in ((True, False) if a != b else ()):
                at = _laid_out(sizes)
                # the 16 aligned bytes with b's first or last one
                at[a] = at[b] if first else at[b] + (sizes[b] - 1) // 16 * 16
                if (a, b) == ("o", "q") and first:
                    continue  # in place
                cache = c_cache(pages=300, type=1, **{n: at[n] for n in sizes if n in POOL})
                assert call(cache, at, sizes) == B.XATTN_ERR_ARG, (a, b, first)
                message = X.lib().xattn_last_error().decode()
                assert "share memory" in message and a in message and b in message


@on_the_cpu
def test_a_rotation_over_its_input_is_refused():
    """Slices of 4 heads of a projection's 12, in bytes from the first one."""
    s = (ctypes.c_int64 * 3)(9 * 12 * 128, 128, 12 * 128)
    plan = X.Rotary([64], X.rotary_freqs([64]))
    for heads in (-3, -1, 1, 2, 3, 12, -12, 11 * 9):
        rc = X.lib().xattn_rotary(1 << 32, s, 2, 4, 9, 128, 1 << 20, plan._ref, 0,
                                  (1 << 32) + heads * 256, s, None)
        assert rc == B.XATTN_ERR_ARG and b"apart" in X.lib().xattn_last_error(), heads


def test_a_rotation_does_not_lose_a_gradient_in_silence():
    plan, pos = X.Rotary([64], X.rotary_freqs([64])), i32(1, 2, 5)
    x = bf(2, 3, 5, 128).requires_grad_()
    expect("requires a gradient", X.xattn_rotary, x, pos, plan)
    expect("requires a gradient", X.xattn_rotary, x * 2, pos, plan, out=bf(2, 3, 5, 128))
    with torch.no_grad():
        expect("device tensor", X.xattn_rotary, x, pos, plan)
    expect("device tensor", X.xattn_rotary, x.detach(), pos, plan)


@pytest.mark.parametrize("batch,hq,hkv,page,pages", [(1, 4, 2, 16, 100), (64, 32, 8, 64, 2048),
                                                     (3, 80, 2, 16, 70), (5, 17, 1, 256, 33)])
def test_workspaces_are_as_large_as_the_header_says(batch, hq, hkv, page, pages):
    c = c_cache(hkv=hkv, page=page)
    n = ctypes.c_size_t(0)
    group = min(hq // hkv, 32)
    parts = 1536 * 520 * group
    for weights in (0, 1):
        assert X.lib().xattn_decode_workspace_size(c, batch, hq, pages, weights, ctypes.byref(n)) == 0
        most = parts + weights * batch * hq * (4 * pages * page + 8)
        assert most <= n.value < most + 4 * 256
    assert X.lib().xattn_evict_workspace_size(c, batch, pages, ctypes.byref(n)) == 0
    chunks = -(-pages * page // 8192) * batch * hkv if pages * page > 16384 else 0
    assert 49160 * chunks <= n.value <= 49160 * chunks + (batch * hkv * 8 + 512 if chunks else 0)
