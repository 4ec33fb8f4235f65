"""fdllm_cache_append and fdllm_cache_read where a sequence starts outside its slots."""
import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import gaussian, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 5, 8, 9, 40])  # both forms of the kernel
@pytest.mark.parametrize("start", [-2 ** 31, -33, -3, -1, 64, 65, 2 ** 31 - 1])
def test_sequences_that_start_outside_are_not_written(fd, n, start):
    cache = fd.KvCache.empty(4, 2, 32, 64)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32).cuda()
    k, v = gaussian((2, 64, 2, 64), 1, torch.bfloat16), gaussian((2, 64, 2, 64), 2, torch.bfloat16)
    fd.fdllm_cache_append(cache, table, None, k, v)
    k2, v2 = gaussian((2, n, 2, 64), 3, torch.bfloat16), gaussian((2, n, 2, 64), 4, torch.bfloat16)
    at = ints([start, 7])
    fd.fdllm_cache_append(cache, table, at, k2, v2)
    got_k, got_v = fd.fdllm_cache_read(cache, table, None, 64, torch.float32)
    for got, old, new in ((got_k, k, k2), (got_v, v, v2)):
        assert torch.equal(got[0].cpu(), ref.values(old[0]).float())
        assert torch.equal(got[1, 7:7 + n].cpu(), ref.values(new[1]).float())
        assert torch.equal(got[1, :7].cpu(), ref.values(old[1, :7]).float())
        assert torch.equal(got[1, 7 + n:].cpu(), ref.values(old[1, 7 + n:]).float())
    # reading takes each slot for itself
    got_k, _ = fd.fdllm_cache_read(cache, table, at, n, torch.float32)
    want = ref.values(k[0]).float()
    for i in range(n):
        slot = start + i
        if 0 <= slot < 64:
            assert torch.equal(got_k[0, i].cpu(), want[slot])
        else:
            assert bool(torch.isnan(got_k[0, i]).all())
