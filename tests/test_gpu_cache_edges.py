"""The prefix cache's operators where their kernels change form, and rows that repeat."""
import math

import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import check, check_weights, gaussian, ints
from test_gpu_cache_evict import check as check_evict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("D,Lq", [(128, 9), (64, 40)])
def test_own_rows_that_repeat(fd, axis, D, Lq):
    """Keys and values of one sequence, token or head for all (an axis of stride 0)."""
    lens = [70, 3]
    cache, table = ref.make_cache(fd, lens, 2, D, 64, seed=axis)
    shape = [2, Lq, 2, D]
    one = list(shape)
    one[axis] = 1
    k = gaussian(one, 20 + axis, torch.bfloat16).expand(shape)
    v = gaussian(one, 30 + axis, torch.bfloat16).expand(shape)
    q = gaussian((2, Lq, 4, D), 40, torch.bfloat16)
    for causal in (False, True):
        check(fd, q, cache, table, lens, k, v, [Lq, Lq - 2], causal)


@pytest.mark.parametrize("new", [1, 31, 32, 33, 127, 128, 129])
@pytest.mark.parametrize("Lq,Hq", [(1, 2), (9, 4), (33, 4)])
def test_own_counts_around_a_load(fd, new, Lq, Hq):
    """Own keys end inside, at and behind the 32 of a load and the 128 of a tile; what lies
    behind the count is not finite."""
    lens = [5, 0]
    cache, table = ref.make_cache(fd, lens, 2, 64, 32, seed=new)
    k = gaussian((2, 140, 2, 64), new, torch.float16)
    v = gaussian((2, 140, 2, 64), new + 1, torch.float16)
    k[:, new:], v[:, new:] = math.nan, math.inf
    check(fd, gaussian((2, Lq, Hq, 64), Lq, torch.float16), cache, table, lens, k, v, [new, new])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_own_keys_that_outweigh_the_prefix(fd, dtype):
    """The references move between cached and own keys, and among the own."""
    lens = [130, 64]
    cache, table = ref.make_cache(fd, lens, 1, 128, 64, seed=2)
    k = gaussian((2, 70, 1, 128), 3, dtype)
    k *= torch.linspace(1, 12, 70, device="cuda").to(dtype)[None, :, None, None]
    v = gaussian((2, 70, 1, 128), 4, dtype)
    for causal in (False, True):
        check(fd, gaussian((2, 70, 1, 128), 5, dtype, 2.0), cache, table, lens, k, v, [70, 69], causal)


def test_key_weights_of_many_queries(fd):
    """More rows a head than the kernel holds at once, over several tiles of keys."""
    lens = [513, 130, 0]
    cache, table = ref.make_cache(fd, lens, 2, 128, 64, seed=11)
    q = gaussian((3, 150, 8, 128), 12, torch.bfloat16, 1.5)
    _, lse = fd.fdllm_cache_attention(q, cache, table, ints(lens), return_lse=True)
    w = torch.rand(3, 2, table.shape[1] * 64, generator=torch.Generator().manual_seed(2)).cuda()
    check_weights(fd, q, lse, cache, table, lens, w)


@pytest.mark.parametrize("n,budget", [(2047, 700), (2048, 700), (2049, 700), (5000, 4999),
                                      (32769, 1000), (66000, 33000)])
def test_evict_around_the_forms_of_the_selection(fd, n, budget):
    g = torch.Generator().manual_seed(n)
    width = -(-n // 256) * 256
    w = torch.rand(1, 1, width, generator=g)
    w[0, 0, ::7] = w[0, 0, 3]  # a group of equals at the cut or near it
    check_evict(fd, [n], 1, 64, 256, budget, 4, 64, w.cuda(), seed=n)


@pytest.mark.parametrize("n,heads", [(3000, 5), (4097, 3), (8193, 65), (9000, 66)])
def test_evict_of_many_long_rows(fd, n, heads):
    g = torch.Generator().manual_seed(n)
    w = torch.rand(1, heads, n, generator=g)
    w[0, 1] = torch.floor(8 * w[0, 1])
    check_evict(fd, [n], heads, 64, 256, 129, 4, 5, w.cuda(), seed=n)


@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 32, 33])
@pytest.mark.parametrize("start", [0, 1, 31])
def test_append_around_the_few_token_form(fd, n, start):
    cache = fd.KvCache.empty(6, 3, 32, 128)
    table = torch.tensor([[4, 1, 2], [0, 5, 3]], dtype=torch.int32).cuda()
    k, v = gaussian((2, n, 3, 128), n, torch.bfloat16), gaussian((2, n, 3, 128), n + 1, torch.bfloat16)
    at = ints([start, 0])
    fd.fdllm_cache_append(cache, table, at, k, v)
    rk, rv = fd.fdllm_cache_read(cache, table, at, n, torch.float32)
    assert torch.equal(rk.cpu(), ref.values(k).float()) and torch.equal(rv.cpu(), ref.values(v).float())


def test_status_after_the_kernels(fd):
    lens = [300]
    cache, table = ref.make_cache(fd, lens, 1, 64, 32, seed=1)
    q = gaussian((1, 4, 1, 64), 1, torch.bfloat16)
    _, lse = fd.fdllm_cache_attention(q, cache, table, ints(lens), return_lse=True)
    fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens))
    assert fd.fdllm_cache_status() == 0
