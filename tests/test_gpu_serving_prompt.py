"""A prompt that is evicted from before its first answer: its last queries give its
tokens their weights."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_16428_amd as X  # noqa: E402

from . import serving_oracle as R  # noqa: E402
from .test_gpu_serving import ints, normal, scattered, within  # noqa: E402


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_prompts_last_queries_weigh_its_tokens(e4m3):
    hq, hkv, page, L, n, budget, recent = 8, 2, 64, 384, 16, 100, 20
    plan = X.Rotary([64], X.rotary_freqs([64]))
    q, k, v = (normal((1, L, h, 128), s).cuda().transpose(1, 2)
               for h, s in ((hq, 600), (hkv, 601), (hkv, 602)))
    pos = torch.arange(L, dtype=torch.int32, device="cuda").view(1, 1, L)
    qr = X.xattn_rotary(q, pos, plan)
    cache = X.KVCache.empty(12, hkv, page, torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    pages = scattered(12, 1, 9, 603)
    table, new_table = pages[:, :7].contiguous().cuda(), pages[:, 7:].contiguous().cuda()
    X.xattn_cache_append(k, v, cache, table, ints([0]), pos=pos, rotary=plan)
    rows = torch.zeros((n, hkv, 7 * page), device="cuda")
    last = qr[0, :, L - n:].transpose(0, 1).contiguous()
    lens = torch.arange(L - n + 1, L + 1, dtype=torch.int32, device="cuda")
    X.xattn_decode(last, cache, table.expand(n, -1).contiguous(), lens, weights=rows)
    w = rows.sum(0, keepdim=True)
    scales = (cache.k_scale.cpu(), cache.v_scale.cpu()) if e4m3 else ()
    _, _, want, _, _, bound = R.decode(last.cpu(), cache.k.cpu(), cache.v.cpu(),
                                       table.cpu().expand(n, -1), lens.tolist(), *scales)
    # sixteen additions in fp32, each half a step of the sum
    within(w[0], want.sum(0), bound.sum(0) + want.sum(0) * n * 2.0 ** -24)
    assert abs(float(w.sum()) - n * hq) < 1e-3 * n * hq
    kept, new_lens, new_w = X.xattn_cache_evict(cache, table, ints([L]), w, new_table, budget, recent)
    assert int(new_lens[0]) == budget
    for h in range(hkv):
        at = R.keep(w[0, h].cpu(), L, budget, recent)
        assert kept[0, h].tolist() == at and at[-recent:] == list(range(L - recent, L))
        assert at[:budget - recent] != list(range(budget - recent))
        assert torch.equal(new_w[0, h, :budget], w[0, h, at])
