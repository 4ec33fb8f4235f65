"""Pools whose rows of all pages and heads pass 31 bits."""
import pytest
import torch

from test_gpu_cache_attention import gaussian, ints

pytestmark = pytest.mark.gpu


def test_the_last_pages_of_a_pool_of_73_gb(fd):
    """2^24 and some page-heads of 32 slots and 128 channels: written, attended to, weighed,
    evicted and read at its ends, as in a pool of a few pages."""
    pages, heads, page, D, n = (1 << 20) + 9, 16, 32, 128, 150
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("not enough free device memory")
    big, small = fd.KvCache.empty(pages, heads, page, D), fd.KvCache.empty(9, heads, page, D)
    assert pages * heads * D > 2 ** 31
    here = torch.tensor([[3, 0, 7, 5, 1], [8, 6, 4, 2, 2]], dtype=torch.int32).cuda()
    there = torch.where(here == 0, 0, here + pages - 9).int()
    k, v = gaussian((1, n, heads, D), 1, torch.bfloat16), gaussian((1, n, heads, D), 2, torch.bfloat16)
    q, lens = gaussian((1, 33, heads, D), 3, torch.bfloat16), ints([n])
    results = []
    for cache, table in ((big, there), (small, here)):
        source, dst = table[:1].contiguous(), table[1:].contiguous()
        fd.fdllm_cache_append(cache, source, None, k, v)
        out, lse = fd.fdllm_cache_attention(q, cache, source, lens, return_lse=True)
        w = fd.fdllm_cache_key_weights(q, lse, cache, source, lens)
        kept = fd.fdllm_cache_evict(cache, source, lens, w, 100, dst, keep_first=2, keep_last=9)
        results.append((out, lse, w, *kept, *fd.fdllm_cache_read(cache, source, None, n),
                        *fd.fdllm_cache_read(cache, dst, None, 100)))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    del big, cache, results
    torch.cuda.empty_cache()
