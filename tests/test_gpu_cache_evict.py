"""fdllm_cache_evict: kept slots, their weights and their held rows, exactly."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def expected(weights, n, budget, first, last):
    """Kept slots of one head: weights a list of n numbers."""
    if n <= budget:
        return list(range(n))
    rank = lambda j: (1, 0.0, j) if math.isnan(weights[j]) else (0, -weights[j], j)
    middle = sorted(range(first, n - last), key=rank)[:budget - first - last]
    return sorted(list(range(first)) + middle + list(range(n - last, n)))


def check(fd, lens, heads, D, page, budget, first, last, weights, seed=0):
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed, poison=False)
    B = len(lens)
    need = -(-budget // page)
    P = cache.pages
    grown = fd.KvCache.empty(P + B * need, heads, page, D)
    for a, b in ((grown.k_codes, cache.k_codes), (grown.v_codes, cache.v_codes),
                 (grown.k_affine, cache.k_affine), (grown.v_affine, cache.v_affine)):
        a[:P] = b
    dst = (P + torch.randperm(B * need).view(B, need)).int().cuda()
    out_lens, out_w, out_i = fd.fdllm_cache_evict(grown, table, ints(lens), weights, budget, dst,
                                                  keep_first=first, keep_last=last)
    k, v = fd.fdllm_cache_read(grown, dst, None, budget, torch.float32, count=out_lens)
    kd, vd = ref.unpack_cache(cache)
    for b, n in enumerate(lens):
        assert int(out_lens[b]) == min(n, budget)
        kb, vb = ref.sequence(kd, table[b], page, n), ref.sequence(vd, table[b], page, n)
        for h in range(heads):
            w = weights[b, h, :n].cpu().tolist()
            kept = expected(w, n, budget, first, last)
            m = len(kept)
            assert out_i[b, h, :m].cpu().tolist() == kept
            assert bool((out_i[b, h, m:] == -1).all()) and bool((out_w[b, h, m:] == 0).all())
            assert torch.equal(torch.nan_to_num(out_w[b, h, :m].cpu(), nan=-7.0),
                               torch.nan_to_num(torch.tensor([w[j] for j in kept], dtype=torch.float32), nan=-7.0))
            assert torch.equal(k[b, :m, h].cpu(), kb[h, kept].float())
            assert torch.equal(v[b, :m, h].cpu(), vb[h, kept].float())
    # the source pages are as they were
    assert torch.equal(grown.k_codes[:P], cache.k_codes)
    assert torch.equal(grown.v_codes[:P], cache.v_codes)
    return out_lens


@pytest.mark.parametrize("lens,heads,D,page,budget,first,last", [
    ([100, 0, 33], 2, 128, 32, 32, 4, 8), ([5, 64, 65], 1, 64, 64, 64, 0, 0),
    ([700, 699], 3, 128, 64, 333, 1, 16), ([300], 2, 64, 128, 17, 9, 8),
    ([40, 41], 1, 128, 32, 1, 0, 0), ([1300], 1, 128, 256, 1299, 0, 1), ([64], 1, 64, 32, 50, 50, 0),
])
def test_kept_slots_weights_and_rows(fd, lens, heads, D, page, budget, first, last):
    g = torch.Generator().manual_seed(budget)
    width = max(-(-max(lens) // page) * page, 1)
    w = torch.rand(len(lens), heads, width, generator=g).cuda()
    check(fd, lens, heads, D, page, budget, first, last, w, seed=budget)


def test_equal_weights_keep_the_lower_slot(fd):
    g = torch.Generator().manual_seed(3)
    w = torch.randint(0, 4, (2, 2, 640), generator=g).float()
    w[1] = 0.0
    w[0, 1, ::3] = -0.0
    check(fd, [640, 601], 2, 64, 64, 200, 3, 11, w.cuda())


def test_negative_infinite_and_nan_weights(fd):
    g = torch.Generator().manual_seed(4)
    w = torch.randn(1, 3, 256, generator=g)
    w[0, 0, ::5] = math.inf
    w[0, 1, ::2] = math.nan
    w[0, 2] = math.nan
    check(fd, [250], 3, 64, 64, 180, 0, 4, w.cuda())


def test_wrong_lengths(fd):
    cache, table = ref.make_cache(fd, [64, 64, 64], 1, 64, 32, seed=1)
    w = torch.rand(3, 1, 60, device="cuda")
    dst = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    dst[:] = torch.tensor([[cache.pages], [-1], [cache.pages]])  # no such pages: nothing moves
    saved = [t.clone() for t in (cache.k_codes, cache.v_codes)]
    lens, out_w, out_i = fd.fdllm_cache_evict(cache, table, ints([61, -2, 50]), w, 32, dst)
    assert lens.cpu().tolist() == [-1, -1, 32]
    assert bool((out_i[:2] == -1).all()) and bool((out_i[2] >= 0).all())
    assert torch.equal(saved[0], cache.k_codes) and torch.equal(saved[1], cache.v_codes)


def test_refusals(fd):
    cache, table = ref.make_cache(fd, [64], 1, 64, 32, seed=1)
    w = torch.rand(1, 1, 64, device="cuda")
    dst = table[:, :1].contiguous()
    n = ints([64])
    for kw in (dict(budget=0), dict(budget=33), dict(budget=8, keep_first=5, keep_last=4),
               dict(budget=8, keep_first=-1), dict(budget=8, keep_last=-1)):
        with pytest.raises(fd.FdllmError):
            fd.fdllm_cache_evict(cache, table, n, w, dst_table=dst, **kw)
    with pytest.raises(ValueError):
        fd.fdllm_cache_evict(cache, table, n, w[:, :, ::2], 8, dst)
    with pytest.raises(TypeError):
        fd.fdllm_cache_evict(cache, table, n, w.half(), 8, dst)
