"""Handles of the serving calls and the numbers and tensors that go to C as they are,
on the CPU: what would reach a kernel as something else than was given is refused."""
import pytest
import torch

import paper_2503_16428_amd as X

from .test_serving_checks import HostCache, bf, expect, i32


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
