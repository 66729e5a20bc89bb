"""Where the serving calls may write: in place, beside their inputs in one buffer."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_16428_amd as X  # noqa: E402

from . import serving_oracle as R  # noqa: E402
from .test_gpu_serving import bits, decode_case, ints, on_gpu, within  # noqa: E402


@pytest.mark.parametrize("hq,hkv,columns", [(4, 2, 4), (4, 2, 80), (40, 1, 4), (40, 1, 80)])
def test_decode_in_place(hq, hkv, columns):
    """o is q: whole rows and shared ones, one tile of heads and two, a row without keys."""
    lens = [60, 0, 1, 33]
    if columns > 4:
        lens[0] = 1200
    q, k, v, s, table = decode_case(4, hq, hkv, 16, lens, False, columns=columns)
    cache, td, ld = on_gpu(k, v, s), table.cuda(), ints(lens)
    want, lse = X.xattn_decode(q.cuda(), cache, td, ld, want_lse=True)
    x = q.cuda()
    o, lse2 = X.xattn_decode(x, cache, td, ld, o=x, want_lse=True)
    assert o is x and torch.equal(bits(x), bits(want)) and torch.equal(bits(lse), bits(lse2))


def test_outputs_may_lie_side_by_side():
    """Outputs and workspace cut from one buffer, one behind the other."""
    lens = [700, 1300]
    q, k, v, s, table = decode_case(2, 4, 2, 16, lens, False, columns=90)
    cache, qd, td, ld = on_gpu(k, v, s), q.cuda(), table.cuda(), ints(lens)
    n = X.decode_workspace_size(cache, 2, 4, 90, True)
    w0 = torch.rand((2, 2, 1440), device="cuda")
    w = w0.clone()
    want = (*X.xattn_decode(qd, cache, td, ld, weights=w, want_lse=True), w)
    parts = [2 * 4 * 128 * 2, 2 * 4 * 4, 2 * 2 * 1440 * 4, n]
    buffer = torch.zeros(sum(parts) + 64, dtype=torch.uint8, device="cuda")
    at = [sum(parts[:i]) for i in range(4)]
    o, lse, w2, ws = (buffer[a:a + m] for a, m in zip(at, parts))
    o, lse = o.view(torch.bfloat16).view(2, 4, 128), lse.view(torch.float32).view(2, 4)
    w2 = w2.view(torch.float32).view(2, 2, 1440).copy_(w0)
    got = (*X.xattn_decode(qd, cache, td, ld, o=o, lse=lse, weights=w2, workspace=ws), w2)
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(want, got))
    assert bool((buffer[sum(parts):] == 0).all())
    with pytest.raises(X.XAttnError, match="share memory"):
        X.xattn_decode(qd, cache, td, ld, o=o, weights=w2, workspace=buffer[at[2]:])


def test_rotary_into_another_slice_of_the_buffer():
    """The heads of a projection's output to those beside them, which are not over them; in
    place whatever the strides of dimensions of size 1 say."""
    plan = X.Rotary([64], X.rotary_freqs([64]))
    buffer = torch.randn((2, 9, 12, 128), device="cuda").bfloat16()
    x, out, over = (buffer[:, :, a:a + 4].transpose(1, 2) for a in (0, 4, 2))
    pos = torch.arange(18, dtype=torch.int32, device="cuda").view(1, 2, 9)
    want, before = X.xattn_rotary(x, pos, plan), buffer.clone()
    assert X.xattn_rotary(x, pos, plan, out=out) is out
    assert torch.equal(bits(out), bits(want))
    assert torch.equal(bits(buffer[:, :, :4]), bits(before[:, :, :4]))
    assert torch.equal(bits(buffer[:, :, 8:]), bits(before[:, :, 8:]))
    with pytest.raises(X.XAttnError, match="apart"):
        X.xattn_rotary(x, pos, plan, out=over)
    one = x[:1]  # another batch stride, of one sequence
    same = one.as_strided(one.shape, (12345 * 8, *one.stride()[1:]))
    X.xattn_rotary(one, pos[:, :1].contiguous(), plan, out=same)
    assert torch.equal(bits(one), bits(want[:1]))


@pytest.mark.parametrize("inverse", [False, True])
def test_rotary_in_an_autograd_function(inverse):
    """As a program that wants gradients has it: forward and backward are the two calls."""
    plan = X.Rotary([30, 20], X.rotary_freqs([30, 20]), True)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos):
            ctx.save_for_backward(pos)
            return X.xattn_rotary(x, pos, plan, inverse=inverse)

        @staticmethod
        def backward(ctx, g):
            return X.xattn_rotary(g.contiguous(), ctx.saved_tensors[0], plan,
                                  inverse=not inverse), None

    g = torch.Generator().manual_seed(570)
    x = torch.randn((2, 3, 5, 128), generator=g).bfloat16()
    to = torch.randn((2, 3, 5, 128), generator=g).bfloat16()
    pos = torch.randint(0, 5000, (2, 2, 5), generator=g, dtype=torch.int32)
    xd = x.cuda().requires_grad_()
    Turn.apply(xd, pos.cuda()).backward(to.cuda())
    want, off = R.rotate(to, pos, [30, 20], list(X.rotary_freqs([30, 20])), True, not inverse)
    within(xd.grad, want, R.bf16_bound(want, off))


def test_graphs_of_long_evictions():
    """The eviction of three launches, captured twice on one workspace, replayed on new lengths
    and weights with eager calls on the same workspace between."""
    batch, hkv, page, columns, budget = 2, 2, 64, 300, 700
    pages = batch * (columns + 12)
    g = torch.Generator().manual_seed(620)
    k, v = (torch.randn((pages, hkv, page, 128), generator=g).bfloat16() for _ in "kv")
    order = torch.randperm(pages, generator=g).int()
    table = order[:batch * columns].view(batch, columns).contiguous().cuda()
    new_table = order[batch * columns:].view(batch, 12).contiguous().cuda()
    ws = torch.empty(X.evict_workspace_size(on_gpu(k, v, ()), batch, columns), dtype=torch.uint8,
                     device="cuda")

    def inputs(i):
        h = torch.Generator().manual_seed(630 + i)
        w = torch.rand((batch, hkv, columns * page), generator=h)
        return ints([19000 - 700 * i, [8193, 600, 17000, 0][i]]), (w * 4).floor().cuda()

    def step(cache, lens, w):
        return X.xattn_cache_evict(cache, table, lens, w, new_table, budget, 40, workspace=ws)

    graphs = []
    for _ in range(2):
        cache, (lens, w) = on_gpu(k, v, ()), inputs(0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(on_gpu(k, v, ()), lens, w)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(cache, lens, w)
        torch.cuda.synchronize()
        graphs.append((graph, cache, lens, w, out))
    eager = on_gpu(k, v, ())
    for i in (1, 2, 3, 0):
        new_lens, new_w = inputs(i)
        want = [t.clone() for t in step(eager, new_lens, new_w)]
        for graph, cache, lens, w, out in graphs:
            lens.copy_(new_lens)
            w.copy_(new_w)
            graph.replay()
        torch.cuda.synchronize()
        for graph, cache, lens, w, out in graphs:
            assert all(torch.equal(bits(a), bits(b)) for a, b in zip(out, want)), i
            assert torch.equal(bits(cache.k), bits(eager.k)), i
            assert torch.equal(bits(cache.v), bits(eager.v)), i
