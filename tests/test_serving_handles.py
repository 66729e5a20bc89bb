"""Handles of the serving calls and the numbers and tensors that go to C as they are,
on the CPU: what would reach a kernel as something else than was given is refused."""
import paper_2503_16428_amd as X

from .test_serving_checks import HostCache, bf, expect


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
