"""The bounded waits of the cache's kernels: one that runs out is reported, once, and leaves the
device usable.  No kernel is made to fail: a warp waits on a barrier that nobody completes."""
import time

import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import gaussian, ints

pytestmark = pytest.mark.gpu
ERR_ARG, ERR_DEVICE = 1, 6


def test_a_wait_that_runs_out_is_reported_once(fd):
    cache, table = ref.make_cache(fd, [300], 1, 64, 32, seed=1)
    q, n = gaussian((1, 4, 1, 64), 1, torch.bfloat16), ints([300])
    want = fd.fdllm_cache_attention(q, cache, table, n)
    assert fd.fdllm_cache_status() == 0
    for tries in (1, 100):
        assert fd.fdllm_cache_check_wait(tries) == 0
        assert torch.equal(fd.fdllm_cache_attention(q, cache, table, n), want)
        assert fd.fdllm_cache_status() == ERR_DEVICE  # sticky through the call after it
        assert fd.fdllm_cache_status() == 0


def test_the_kernels_own_limit_is_about_a_second(fd):
    """A host that waits for a call that gives up gets its answer: the limit, counted in tries, is
    neither within reach of an ordinary wait nor many seconds."""
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    assert fd.fdllm_cache_check_wait() == 0
    assert fd.fdllm_cache_status() == ERR_DEVICE
    assert 0.05 <= time.perf_counter() - t0 <= 5.0
    assert fd.fdllm_cache_status() == 0


def test_limits_out_of_range(fd):
    assert fd.fdllm_cache_check_wait(-1) == ERR_ARG
    assert fd.fdllm_cache_check_wait((1 << 18) + 1) == ERR_ARG
    assert fd.fdllm_cache_status() == 0
