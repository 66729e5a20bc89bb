"""Refusals of the calls for serving after the prefill, without a GPU: the C ABI
before any HIP call, the binding before any C call (its tensors live on the
host; a call that passed every other check stops at the device check)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2503_16428_amd as X
from paper_2503_16428_amd import binding as B

E4M3 = torch.float8_e4m3fn
FAKE = 0x1000  # never dereferenced: every case fails validation


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def strides(*v):
    return (ctypes.c_int64 * 3)(*v)


def c_plan(**kw):
    freq = kw.pop("freq", [1.0] * 64)
    keep = None if freq is None else (ctypes.c_double * len(freq))(*freq)
    d = dict(axes=1, pairs=(64, 0, 0), interleaved=0)
    d.update(kw)
    p = B.RotaryPlan(d["axes"], (ctypes.c_int32 * 3)(*d["pairs"]), d["interleaved"],
                     ctypes.cast(keep, ctypes.c_void_p) if keep is not None else None)
    p.keep = keep
    return p


def c_cache(**kw):
    d = dict(pages=4, page=16, hkv=2, head_dim=128, type=0, k=FAKE, v=FAKE, k_scale=None,
             v_scale=None)
    d.update(kw)
    return B.Cache(*[d[n] for n, _ in B.Cache._fields_])


def refused(rc, code=B.XATTN_ERR_ARG):
    assert rc == code, X.lib().xattn_last_error()
    assert X.lib().xattn_last_error()


def rotary(**kw):
    d = dict(x=FAKE, xs=strides(0, 128, 256), batch=1, heads=2, tokens=3, dim=128, pos=FAKE,
             plan=c_plan(), inverse=0, out=FAKE, os=strides(0, 384, 128))
    d.update(kw)
    return X.lib().xattn_rotary(d["x"], d["xs"], d["batch"], d["heads"], d["tokens"], d["dim"],
                                d["pos"], d["plan"], d["inverse"], d["out"], d["os"], None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(x=FAKE + 8), dict(pos=None), dict(pos=FAKE + 2), dict(out=None),
    dict(out=FAKE + 2), dict(xs=None), dict(os=None), dict(plan=None), dict(batch=0),
    dict(heads=0), dict(tokens=-1), dict(dim=0), dict(inverse=2),
    dict(xs=strides(0, 4, 256)), dict(xs=strides(0, -128, 256)), dict(xs=strides(0, 128, 2**41)),
    dict(os=strides(0, 384, 0)), dict(os=strides(0, 0, 128)), dict(os=strides(0, 384, 64)),
    dict(os=strides(0, 128, 128)), dict(os=strides(0, 256, 128)), dict(os=strides(0, 128, 248)),
    dict(batch=2, os=strides(128, 384, 128)), dict(batch=2, os=strides(640, 384, 128)),
    dict(plan=c_plan(axes=0)), dict(plan=c_plan(axes=4)), dict(plan=c_plan(pairs=(0, 0, 0))),
    dict(plan=c_plan(pairs=(60, 4, 0))), dict(plan=c_plan(axes=2, pairs=(60, 5, 0))),
    dict(plan=c_plan(axes=2, pairs=(60, 0, 0))), dict(plan=c_plan(pairs=(65, 0, 0))),
    dict(plan=c_plan(pairs=(-1, 0, 0))), dict(plan=c_plan(interleaved=2)),
    dict(plan=c_plan(freq=None)), dict(plan=c_plan(freq=[1.0] * 63 + [float("nan")])),
    dict(plan=c_plan(freq=[float("inf")] + [1.0] * 63))])
def test_rotary_refuses(kw):
    refused(rotary(**kw))


def test_rotary_refuses_what_it_does_not_support():
    refused(rotary(dim=64), B.XATTN_ERR_UNSUPPORTED)
    refused(rotary(batch=2**15, tokens=2**14), B.XATTN_ERR_UNSUPPORTED)
    refused(rotary(heads=65536), B.XATTN_ERR_UNSUPPORTED)


def append(**kw):
    d = dict(k=FAKE, ks=strides(0, 128, 256), v=FAKE, vs=strides(0, 128, 256), batch=1, tokens=3,
             count=None, start=FAKE, table=FAKE, pages=2, pos=None, plan=None, cache=c_cache())
    d.update(kw)
    return X.lib().xattn_cache_append(d["k"], d["ks"], d["v"], d["vs"], d["batch"], d["tokens"],
                                      d["count"], d["start"], d["table"], d["pages"], d["pos"],
                                      d["plan"], d["cache"], None)


BAD_CACHES = [dict(page=0), dict(page=8), dict(page=48), dict(page=512), dict(pages=0), dict(hkv=0),
              dict(head_dim=0), dict(type=2), dict(k=None), dict(v=None), dict(k=FAKE + 8),
              dict(type=1), dict(type=1, k_scale=FAKE), dict(type=1, k_scale=FAKE, v_scale=FAKE + 1)]


@pytest.mark.parametrize("kw", [
    dict(k=None), dict(v=None), dict(v=FAKE + 4), dict(ks=None), dict(vs=strides(0, 128, 12)),
    dict(batch=0), dict(tokens=0), dict(start=None), dict(table=None), dict(pages=0),
    dict(count=FAKE + 2), dict(pos=FAKE + 1, plan=c_plan()),
    dict(pos=FAKE), dict(plan=c_plan()), dict(pos=FAKE, plan=c_plan(axes=5)), dict(cache=None),
    *[dict(cache=c_cache(**c)) for c in BAD_CACHES]])
def test_append_refuses(kw):
    refused(append(**kw))


def decode(**kw):
    d = dict(q=FAKE, cache=c_cache(), batch=1, hq=4, table=FAKE, pages=2, lens=FAKE, o=FAKE,
             weights=None, lse=None, ws=FAKE, bytes=1 << 40)
    d.update(kw)
    return X.lib().xattn_decode(d["q"], d["cache"], d["batch"], d["hq"], d["table"], d["pages"],
                                d["lens"], d["o"], d["lse"], d["weights"], d["ws"], d["bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(q=FAKE + 8), dict(o=None), dict(lens=None), dict(table=None), dict(batch=0),
    dict(hq=0), dict(hq=3), dict(pages=0), dict(pages=-1), dict(cache=None),
    dict(weights=FAKE + 4), dict(lse=FAKE + 2),
    *[dict(cache=c_cache(**c)) for c in BAD_CACHES]])
def test_decode_refuses(kw):
    refused(decode(**kw))


def test_decode_refuses_workspaces_and_sizes():
    n = ctypes.c_size_t(0)
    c = c_cache()
    assert X.lib().xattn_decode_workspace_size(c, 1, 4, 200, 0, ctypes.byref(n)) == 0
    assert n.value > 0
    for kw in (dict(ws=None), dict(bytes=n.value - 1), dict(ws=FAKE + 8)):
        refused(decode(pages=200, **kw), B.XATTN_ERR_WORKSPACE)
    assert X.lib().xattn_decode_workspace_size(c, 1, 4, 2, 0, ctypes.byref(n)) == 0
    assert n.value == 0  # a row is one workgroup's; with weights its products are kept
    refused(decode(weights=FAKE, ws=None), B.XATTN_ERR_WORKSPACE)
    refused(X.lib().xattn_decode_workspace_size(c, 1, 4, 2, 0, None))
    refused(X.lib().xattn_decode_workspace_size(c, 1, 3, 2, 0, ctypes.byref(n)))
    U = B.XATTN_ERR_UNSUPPORTED
    refused(decode(cache=c_cache(head_dim=64)), U)
    refused(decode(pages=2**27), U)
    refused(decode(batch=2**19), U)
    refused(decode(batch=2**16, hq=32), U)
    refused(decode(batch=2**12, pages=2**20), U)


def test_decode_workspaces_grow_with_the_call():
    def size(batch, hq, pages, weights, **kw):
        n = ctypes.c_size_t(0)
        rc = X.lib().xattn_decode_workspace_size(c_cache(**kw), batch, hq, pages, weights,
                                                 ctypes.byref(n))
        assert rc == 0
        return n.value

    for batch, hq, pages in ((1, 2, 1), (3, 34, 7), (64, 32, 1000), (1, 64, 8192)):
        plain = size(batch, hq, pages, 0)
        assert (0 < plain < 1 << 34) if pages > 64 else plain == 0
        # the products of every head and token, for the weights
        assert size(batch, hq, pages, 1) >= plain + batch * hq * pages * 16 * 4
        assert size(batch, hq, pages, 0, type=1, k_scale=FAKE, v_scale=FAKE) == plain


def evict(**kw):
    d = dict(cache=c_cache(), batch=1, table=FAKE, pages=2, lens=FAKE, weights=FAKE, budget=8,
             recent=2, new_table=FAKE + 64, new_pages=1, kept=FAKE, new_lens=FAKE + 64,
             new_weights=FAKE + 64, ws=FAKE, bytes=1 << 40)
    d.update(kw)
    return X.lib().xattn_cache_evict(d["cache"], d["batch"], d["table"], d["pages"], d["lens"],
                                     d["weights"], d["budget"], d["recent"], d["new_table"],
                                     d["new_pages"], d["kept"], d["new_lens"], d["new_weights"],
                                     d["ws"], d["bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(lens=None), dict(weights=None), dict(new_table=None), dict(kept=None),
    dict(new_lens=None), dict(new_weights=None), dict(budget=0), dict(recent=-1), dict(recent=9),
    dict(budget=17), dict(new_pages=0), dict(new_lens=FAKE), dict(new_weights=FAKE),
    dict(new_table=FAKE), dict(batch=0), dict(weights=FAKE + 68), dict(cache=None),
    *[dict(cache=c_cache(**c)) for c in BAD_CACHES]])
def test_evict_refuses(kw):
    refused(evict(**kw))


def test_evict_refuses_workspaces():
    n, size = ctypes.c_size_t(0), X.lib().xattn_evict_workspace_size
    assert size(c_cache(), 1, 1024, ctypes.byref(n)) == 0 and n.value == 0  # 16384 tokens
    assert size(c_cache(), 1, 1025, ctypes.byref(n)) == 0 and n.value > 16400 * 2 * 4
    for kw in (dict(ws=None), dict(bytes=n.value - 1), dict(ws=FAKE + 8)):
        refused(evict(pages=1025, **kw), B.XATTN_ERR_WORKSPACE)
    refused(size(c_cache(), 1, 2, None))
    refused(size(c_cache(), 0, 2, ctypes.byref(n)))
    expect("workspace must be", X.xattn_cache_evict, HostCache(), i32(3, 2), i32(3),
           torch.zeros(3, 2, 32), i32(3, 1), 4, 1, workspace=torch.zeros(8))


def test_evict_refuses_what_it_does_not_support():
    U = B.XATTN_ERR_UNSUPPORTED
    refused(evict(pages=2**27), U)
    refused(evict(new_pages=2**27), U)
    refused(evict(batch=2**12, budget=2**20, new_pages=2**16), U)


# ---- the binding


def expect(msg, fn, *a, **kw):
    with pytest.raises(B.XAttnError) as e:
        fn(*a, **kw)
    assert msg in str(e.value), str(e.value)
    assert e.value.status == B.XATTN_ERR_ARG


class HostCache(X.KVCache):
    """A cache of host tensors, past the constructor's own device check."""

    def __init__(self, pages=4, hkv=2, page=16):
        self.k = self.v = bf(pages, hkv, page, 128)
        self.k_scale = self.v_scale = None
        self.pages, self.hkv, self.page, self.e4m3 = pages, hkv, page, False
        self.device = self.k.device
        self._ref = ctypes.byref(c_cache(pages=pages, hkv=hkv, page=page))


PLAN = X.Rotary([64], X.rotary_freqs([64]))


def test_plans_are_checked():
    for pairs, n in (([], 0), ([0], 0), ([40, 25], 65), ([1, 1, 1, 1], 4), ([64], 63), ([-1, 3], 2)):
        with pytest.raises(B.XAttnError):
            X.Rotary(pairs, np.ones(n))
    with pytest.raises(B.XAttnError):
        X.Rotary([2], [1.0, float("nan")])
    assert np.allclose(X.rotary_freqs([2, 2], 16.0), [1, 0.5, 0.25, 0.125])
    assert np.allclose(X.rotary_freqs([2, 1], 16.0, restart=True), [1, 0.25, 1])
    freq = np.ones(64)
    plan = X.Rotary([64], freq)
    freq[:] = float("nan")  # the plan has its own copy
    assert np.isfinite(plan._freq).all()


def test_rotary_tensors_are_checked():
    f, pos = X.xattn_rotary, i32(1, 2, 5)
    x = bf(2, 3, 5, 128)
    expect("must be torch.bfloat16", f, x.float(), pos, PLAN)
    expect("x must be", f, x[..., :64], pos, PLAN)
    expect("x must be", f, x[0, 0], pos, PLAN)
    expect("x must be", f, bf(2, 0, 5, 128), i32(1, 2, 5), PLAN)
    expect("must be contiguous", f, bf(2, 3, 5, 256)[..., ::2], pos, PLAN)
    expect("pos must have shape", f, x, i32(2, 5), PLAN)
    expect("pos must have shape", f, x[0], pos, PLAN)
    expect("pos must be", f, x, pos.long(), PLAN)
    expect("rotary must be", f, x, pos, [64])
    expect("out must have shape", f, x, pos, PLAN, out=bf(2, 3, 4, 128))
    expect("out must be", f, x, pos, PLAN, out=x.float())
    expect("device tensor", f, x, pos, PLAN)


def test_append_tensors_are_checked():
    f, c = X.xattn_cache_append, HostCache()
    k, table, start = bf(3, 2, 5, 128), i32(3, 2), i32(3)
    expect("cache must be", f, k, k, None, table, start)
    expect("v must have shape", f, k, bf(3, 2, 4, 128), c, table, start)
    expect("has 3 heads", f, bf(3, 3, 5, 128), bf(3, 3, 5, 128), c, table, start)
    expect("table must be", f, k, k, c, i32(2, 2), start)
    expect("table must be", f, k, k, c, i32(3), start)
    expect("table must be", f, k, k, c, table.long(), start)
    expect("start must have shape", f, k, k, c, table, i32(2))
    expect("count must be", f, k, k, c, table, start, start.long())
    expect("go together", f, k, k, c, table, start, pos=i32(1, 3, 5))
    expect("go together", f, k, k, c, table, start, rotary=PLAN)
    expect("pos must have shape", f, k, k, c, table, start, pos=i32(1, 3, 4), rotary=PLAN)
    expect("device tensor", f, k, k, c, table, start)


def test_decode_tensors_are_checked():
    f, c = X.xattn_decode, HostCache()
    q, table, lens = bf(3, 4, 128), i32(3, 2), i32(3)
    expect("cache must be", f, q, c.k, table, lens)
    expect("q must be", f, q[0], c, table, lens)
    expect("q must be", f, q.float(), c, table, lens)
    expect("table must be", f, q, c, i32(4, 2), lens)
    expect("lens must have shape", f, q, c, table, i32(4))
    expect("lens must be", f, q, c, table, lens.float())
    expect("o must have shape", f, q, c, table, lens, o=bf(3, 5, 128))
    expect("lse must be", f, q, c, table, lens, lse=torch.zeros(3, 4).double())
    expect("weights must have shape", f, q, c, table, lens, weights=torch.zeros(3, 2, 31))
    expect("workspace must be", f, q, c, table, lens, workspace=torch.zeros(8))
    expect("device tensor", f, q, c, table, lens)


def test_evict_tensors_are_checked():
    f, c = X.xattn_cache_evict, HostCache()
    table, lens, w, new = i32(3, 2), i32(3), torch.zeros(3, 2, 32), i32(3, 1)
    expect("table must be", f, c, table[0], lens, w, new, 4, 1)
    expect("new_table must be", f, c, table, lens, w, i32(2, 1), 4, 1)
    expect("weights must have shape", f, c, table, lens, w[:, :, :16], new, 4, 1)
    expect("weights must be", f, c, table, lens, w.double(), new, 4, 1)
    expect("budget must be", f, c, table, lens, w, new, 17, 1)
    expect("budget must be", f, c, table, lens, w, new, 0, 0)
    expect("kept must have shape", f, c, table, lens, w, new, 4, 1, kept=i32(3, 2, 5))
    expect("new_lens must have shape", f, c, table, lens, w, new, 4, 1, new_lens=i32(2))
    expect("new_weights must have", f, c, table, lens, w, new, 4, 1, new_weights=w)
    expect("device tensor", f, c, table, lens, w, new, 4, 1)


def test_caches_are_checked():
    k, s = bf(4, 2, 16, 128), torch.zeros(4, 2, 16, dtype=torch.uint8)
    k8 = torch.zeros(4, 2, 16, 128, dtype=torch.uint8).view(E4M3)
    expect("k must be", X.KVCache, bf(4, 2, 24, 128), bf(4, 2, 24, 128))
    expect("k must be", X.KVCache, bf(4, 2, 16, 64), bf(4, 2, 16, 64))
    expect("k must be", X.KVCache, k[0], k[0])
    expect("k must be", X.KVCache, k.float(), k.float())
    expect("v must have shape", X.KVCache, k, k[:3])
    expect("v must be", X.KVCache, k, k.float())
    expect("needs k_scale", X.KVCache, k8, k8)
    expect("k_scale must have shape", X.KVCache, k8, k8, s[:3], s)
    expect("v_scale must be", X.KVCache, k8, k8, s, s.float())
    expect("no scales", X.KVCache, k, k, s, s)
    expect("device tensor", X.KVCache, k, k)
    expect("dtype must be", X.KVCache.empty, 4, 2, 16, torch.float16, "cpu")
