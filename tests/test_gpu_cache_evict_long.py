"""fdllm_cache_evict on rows of millions of slots: more keys of one digit in a thread block than
16 bits count.  Pages repeat in the table, so that the cache itself is small."""
import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,heads", [(2200001, 64), (8500003, 1)])
@pytest.mark.parametrize("form", ["spread", "ties"])
def test_rows_of_millions_of_slots(fd, n, heads, form):
    D, page, pool, budget, first, last = 64, 256, 9, 1000, 4, 60
    g = torch.Generator(device="cuda").manual_seed(n)
    per = -(-n // page)
    held, _ = ref.make_cache(fd, [pool * page], heads, D, page, seed=heads, spare=0, poison=False)
    need = -(-budget // page)
    cache = fd.KvCache.empty(pool + need, heads, page, D)
    for a, b in ((cache.k_codes, held.k_codes), (cache.v_codes, held.v_codes),
                 (cache.k_affine, held.k_affine), (cache.v_affine, held.v_affine)):
        a[:pool] = b
    table = torch.randint(0, pool, (1, per), generator=g, device="cuda", dtype=torch.int32)
    dst = (pool + torch.arange(need, dtype=torch.int32)).view(1, -1).cuda()
    # weights of one leading digit but for a few zeros, as accumulated attention has them
    w = torch.rand(1, heads, n, generator=g, device="cuda") + 1e-3
    if form == "ties":
        w = torch.floor(w * 64) / 64 + 1e-3
    w[:, :, ::1000] = 0.0
    lens, kept_w, index = fd.fdllm_cache_evict(cache, table, ints([n]), w, budget, dst,
                                               keep_first=first, keep_last=last)
    k, v = fd.fdllm_cache_read(cache, dst, None, budget, torch.float32)
    kd, vd = ref.unpack_cache(held)
    assert lens.tolist() == [budget]
    for h in range(heads):
        order = torch.sort(w[0, h, first:n - last], descending=True, stable=True)[1]
        middle = first + order[:budget - first - last]
        want = torch.cat((torch.arange(first, device="cuda"), middle.sort()[0],
                          torch.arange(n - last, n, device="cuda")))
        assert torch.equal(index[0, h].long(), want)
        assert torch.equal(kept_w[0, h], w[0, h, want])
        at, slot = table[0, want // page].long().cpu(), (want % page).cpu()
        assert torch.equal(k[0, :, h].cpu(), kd[at, h, slot].float())
        assert torch.equal(v[0, :, h].cpu(), vd[at, h, slot].float())
