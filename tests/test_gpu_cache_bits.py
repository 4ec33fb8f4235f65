"""What fdllm_cache_attention keeps of its weights: the error that its own arithmetic adds to
the rounding of the result's type.

A weight is held to 2^-20 of itself (fp16's 22 bits in two numbers, and the score's own fp32
roundings) and to 2^-34 of the row's largest; the fp32 sums of a tensor core lose up to a unit
of their last place, 2^-23, at each step of 16 keys."""
import math

import pytest
import torch

import cache_ref as ref
from test_gpu_cache_attention import check, gaussian, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Lq", [1, 20, 40])
@pytest.mark.parametrize("nats", [8.0, 11.3, math.log(2.0 ** 24 / 2.49), math.log(2.0 ** 24 / 0.45)])
def test_a_first_key_that_outweighs_a_long_tail(fd, dtype, Lq, nats):
    """Key 0 lies `nats` above 30000 equal keys.  The values are 0 in all channels but one, where
    they are 15 (scale 1, offset 0): any error of the small weights stays in the zeros.  608 sequences
read the same pages, so that the keys of most are summed in one place."""
    B, D, page, n = 608, 64, 256, 30001
    cache = fd.KvCache.empty(-(-n // page), 1, page, D)
    table = torch.arange(cache.pages, dtype=torch.int32).view(1, -1).cuda()
    k, v = torch.zeros(1, n, 1, D, device="cuda"), torch.zeros(1, n, 1, D, device="cuda")
    k[0, 0, 0, 0] = 15.0  # code 15 of scale 1: exactly 15
    v[..., 5] = 15.0
    fd.fdllm_cache_append(cache, table, None, k, v)
    q = torch.zeros(B, Lq, 1, D, dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    out = fd.fdllm_cache_attention(q, cache, table.expand(B, -1).contiguous(), ints([n] * B),
                                   scale=nats / 15.0).cpu().double().view(-1, D)
    total = 1.0 + (n - 1) * math.exp(-nats)
    tol = 15.0 * (2.0 ** -20 + n / 16 * 2.0 ** -23 * (1 - 1 / total) + n * 2.0 ** -34 / total)
    want = torch.zeros(D, dtype=torch.float64)
    want[5] = 15.0
    err = (out - want).abs()
    assert float(err[:, 5].max()) <= 15.0 * ref.EPS[dtype] + tol
    err[:, 5] = 0.0
    assert float(err.max()) <= tol, float(err.max()) / tol


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Lq,Hq,heads,D,lens,new", [
    (32, 4, 4, 128, [640, 300, 511], 32), (64, 8, 2, 128, [3000], 64), (90, 4, 4, 64, [130, 0], 90),
    (1, 8, 2, 128, [1021] * 6, 1),
])
def test_the_error_is_the_rounding_of_the_result(fd, dtype, Lq, Hq, heads, D, lens, new):
    """The root mean square of the error against that of the exact result's own rounding.  bf16
    rounds at up to 2^-8; own weights in bf16 (2^-17) and everything else add less than 2^-15 of
    it, which in squares is below 1 %; fp16 rounds at up to 2^-11, the rest adds less than 2^-18."""
    B = len(lens)
    cache, table = ref.make_cache(fd, lens, heads, D, 64, seed=D + Lq)
    q = gaussian((B, Lq, Hq, D), 1, dtype, 1.5)
    k, v = gaussian((B, new, heads, D), 2, dtype), gaussian((B, new, heads, D), 3, dtype)
    out = fd.fdllm_cache_attention(q, cache, table, ints(lens), k, v).cpu().double()
    want = ref.attention(q, cache, table, lens, k, v)[0]
    rounding = float((want.to(dtype).double() - want).square().mean().sqrt())
    error = float((out - want).square().mean().sqrt())
    assert error <= 1.01 * rounding, error / rounding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Lq", [1, 20, 40])
@pytest.mark.parametrize("power", [16, 28, 40])
def test_scores_beyond_the_bits_of_fp32(fd, dtype, Lq, power):
    """Scores 2^power times 0 to 15: all weight is on the keys of the largest, equally, although a
    score of this size is rounded to a multiple of many units."""
    D, n = 64, 300
    cache, table = ref.make_cache(fd, [n], 1, D, 64, seed=power)
    code = torch.arange(n) * 7 % 16
    code[:40] = 3
    k = torch.zeros(1, n, 1, D)
    k[0, :, 0, 0], k[..., 1] = code.float(), 15.0  # scale 1, offset 0: held exactly
    v = gaussian((1, n, 1, D), 1, torch.float32)
    fd.fdllm_cache_append(cache, table, None, k.cuda(), v)
    q = torch.zeros(1, Lq, 1, D, dtype=dtype, device="cuda")
    q[..., 0] = 16.0
    out, lse = fd.fdllm_cache_attention(q, cache, table, ints([n]), scale=2.0 ** (power - 4), return_lse=True)
    most = code == 15
    want, want_lse = ref.values(v)[0, most, 0].mean(0), 15 * 2.0 ** power + math.log(int(most.sum()))
    reach = float(v.abs().max())
    assert bool(((out.cpu().double() - want).abs() <= ref.EPS[dtype] * want.abs() + 2.0 ** -18 * reach).all())
    assert bool(((lse.cpu().double() / want_lse - 1).abs() <= 2.0 ** -20).all())
    # and as own keys, of which the last outweighs all
    own = torch.zeros(1, Lq, 1, D, dtype=dtype, device="cuda")
    own[0, :, 0, 0] = 1.0
    own[0, -1, 0, 0] = 17.0
    v_own = gaussian((1, Lq, 1, D), 2, dtype)
    out = fd.fdllm_cache_attention(q, cache, table, ints([n]), own, v_own, scale=2.0 ** (power - 4))
    assert torch.equal(out[0, :, 0], v_own[0, -1:, 0].expand(Lq, -1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Lq,Hq,heads,D,lens", [
    (1, 8, 1, 128, [300, 65]), (16, 4, 2, 64, [130, 257]), (40, 4, 1, 128, [700]), (150, 4, 2, 128, [513, 130]),
])
def test_rows_of_very_different_sizes_do_not_mix(fd, dtype, Lq, Hq, heads, D, lens):
    """A few queries are 2^24 to 2^26 times as large as the others of their head: the others'
    scores keep the bits that they have alone."""
    B = len(lens)
    cache, table = ref.make_cache(fd, lens, heads, D, 64, seed=D + Lq)
    small = 1.0 if dtype is torch.bfloat16 else 2.0 ** -14
    q = gaussian((B, Lq, Hq, D), 1, torch.float32, 1.5) * small
    q[:, ::13, 1] *= 2.0 ** (24 if dtype is torch.bfloat16 else 26)
    q[:, 0, 2] = 0.0
    q = q.to(dtype)
    scale = D ** -0.5 / small
    k, v = gaussian((B, Lq, heads, D), 2, dtype, 0.2), gaussian((B, Lq, heads, D), 3, dtype)
    for own in (dict(), dict(k_new=k, v_new=v)):
        _, lse = check(fd, q, cache, table, lens, scale=scale, **own)
    # (against the cached keys alone, so that the weights of every query sum to 1)
    _, lse = check(fd, q, cache, table, lens, scale=scale)
    w = torch.zeros(B, heads, table.shape[1] * 64, device="cuda")
    # (a log-sum-exp of 2^24 holds weights to a factor of e: those rows are left out)
    big = q.abs().amax(-1).float() > 1e3 * small
    alone = fd.fdllm_cache_key_weights(q, torch.where(big, -math.inf, lse), cache, table, ints(lens),
                                       weights=w, scale=scale)
    want, tol = ref.key_weights(q, torch.where(big, -math.inf, lse), cache, table, lens, w, scale=scale)
    assert bool(((alone.cpu().double() - want).abs() <= tol).all())
