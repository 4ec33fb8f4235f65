"""fdllm_cache_key_weights of queries that count nothing."""
import math

import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import gaussian, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Lq", [1, 9, 150])
def test_key_weights_of_rows_that_count_nothing(fd, dtype, Lq):
    """Queries of a log-sum-exp of -inf (padding) may hold anything."""
    lens = [200, 63]
    cache, table = ref.make_cache(fd, lens, 2, 128, 64, seed=Lq)
    q = gaussian((2, Lq, 4, 128), Lq, dtype)
    _, lse = fd.fdllm_cache_attention(q, cache, table, ints(lens), return_lse=True)
    lse[:, ::3, 1:3] = -math.inf
    want = fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens))
    for value in (math.nan, math.inf, -math.inf, 6e4):
        q[:, ::3, 1:3] = value
        got = fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens))
        assert torch.equal(got, want)
