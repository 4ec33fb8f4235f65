"""fdllm_cache_attention and fdllm_cache_key_weights against 64-bit evaluations of their
formulas; the tolerances are those of cache_ref.py."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu


def gaussian(shape, seed, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn(shape, generator=g)).to(dtype).cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def check(fd, q, cache, table, lens, k_new=None, v_new=None, new_lens=None, causal=False,
          scale=None):
    out, lse = fd.fdllm_cache_attention(q, cache, table, ints(lens), k_new, v_new,
                                        None if new_lens is None else ints(new_lens), causal,
                                        scale, return_lse=True)
    w_out, w_lse, tol, tol_lse = ref.attention(q, cache, table, lens, k_new, v_new, new_lens,
                                               causal, scale)
    err = (out.cpu().double() - w_out).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-30)).max())
    empty = torch.isinf(w_lse)
    assert torch.equal(torch.isneginf(lse.cpu()), empty)
    gap = (lse.cpu().double() - w_lse).abs()[~empty]
    assert bool((gap <= tol_lse[~empty]).all()), float((gap / tol_lse[~empty]).max())
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,Lq,Hq,heads,D,page,lens", [
    (1, 1, 8, 2, 128, 64, [1]),
    (3, 1, 4, 4, 128, 64, [127, 0, 129]),
    (2, 5, 7, 1, 64, 32, [128, 31]),
    (4, 32, 2, 2, 128, 64, [333, 64, 1, 256]),
    (2, 33, 4, 1, 128, 128, [200, 511]),
    (1, 70, 6, 2, 64, 256, [1000]),
    (1, 17, 3, 3, 128, 32, [2049]),
])
def test_cached_keys(fd, dtype, B, Lq, Hq, heads, D, page, lens):
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed=sum(lens) + Lq)
    check(fd, gaussian((B, Lq, Hq, D), Lq, dtype, 1.5), cache, table, lens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Lq,Hq,heads,D,page,lens,new", [
    (1, 4, 2, 128, 64, [65, 0, 3], [1, 1, 0]),
    (32, 2, 2, 128, 64, [100, 0, 0], [32, 32, 0]),
    (19, 6, 2, 64, 32, [0, 33, 128], [19, 1, 7]),
    (150, 2, 1, 128, 64, [40, 0, 200], [150, 129, 0]),
])
def test_own_keys(fd, dtype, causal, Lq, Hq, heads, D, page, lens, new):
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed=Lq + page)
    qkv = gaussian((3, Lq, Hq + 2 * heads, D), Lq, dtype)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + heads], qkv[:, :, Hq + heads:].contiguous()
    k = k.contiguous()
    for b, m in enumerate(new):  # padding behind the counts
        k[b, m:] = math.nan
        v[b, m:] = math.inf
    check(fd, q, cache, table, lens, k, v, new, causal)
    if causal:  # keys behind the bound hold NaN: the rows before them do not see it
        k[0, -1], v[0, -1] = math.nan, math.nan
        out = fd.fdllm_cache_attention(q, cache, table, ints(lens), k, v, ints(new), True)
        assert bool(torch.isfinite(out[0, :-1]).all())


def test_no_cached_key_and_none_at_all(fd):
    cache, table = ref.make_cache(fd, [0, 0], 2, 64, 32, seed=1)
    q = gaussian((2, 3, 2, 64), 1, torch.bfloat16)
    out, lse = check(fd, q, cache, table, [0, 0])
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("std,scale", [(40.0, None), (1.0, 0.0), (1.0, -0.2), (1e-3, 1.0)])
def test_peaked_flat_and_negative_scores(fd, std, scale):
    lens = [700, 130]
    cache, table = ref.make_cache(fd, lens, 2, 128, 64, seed=4)
    check(fd, gaussian((2, 8, 4, 128), 3, torch.bfloat16, std), cache, table, lens, scale=scale)


def test_scores_that_grow_along_the_keys(fd):
    """Every later key scores higher by more than any fixed margin: the running maximum moves
    at every step; and the values' scales span many binary orders."""
    heads, D, page, n = 1, 128, 64, 640
    cache, table = ref.make_cache(fd, [n], heads, D, page, seed=5)
    k = torch.zeros(1, n, heads, D, device="cuda")
    k[0, :, 0, 0] = torch.arange(n, device="cuda") * 0.25
    v = gaussian((1, n, heads, D), 6, torch.float32)
    v *= torch.exp2(torch.arange(n, device="cuda") % 41 - 20.0)[None, :, None, None]
    fd.fdllm_cache_append(cache, table, None, k, v)
    q = gaussian((1, 4, 1, D), 7, torch.bfloat16, 0.01)
    q[..., 0] = 16.0
    check(fd, q, cache, table, [n], scale=1.0)
    q[..., 0] = -16.0
    check(fd, q, cache, table, [n], scale=1.0)


def test_wrong_lengths_and_pages_report_nan(fd):
    lens = [40, 40, 40, 40]
    cache, table = ref.make_cache(fd, lens, 2, 64, 32, seed=6, min_pages=2)
    q = gaussian((4, 2, 2, 64), 8, torch.bfloat16)
    k = gaussian((4, 3, 2, 64), 9, torch.bfloat16)
    good = fd.fdllm_cache_attention(q, cache, table, ints(lens), k, k)
    table = table.clone()
    table[3, 1] = cache.pages
    out, lse = fd.fdllm_cache_attention(q, cache, table, ints([40, -1, 65, 40]), k, k,
                                        return_lse=True)
    assert torch.equal(out[0], good[0])
    assert bool(torch.isnan(out[1:]).all()) and bool(torch.isnan(lse[1:]).all())
    out = fd.fdllm_cache_attention(q, cache, table, ints(lens), k, k, ints([3, 4, -1, 0]))
    assert torch.equal(out[0], good[0]) and bool(torch.isnan(out[1:]).all())


def test_held_nan_rows_reach_only_their_sequence(fd):
    lens = [60, 60]
    cache, table = ref.make_cache(fd, lens, 1, 64, 32, seed=7)
    q = gaussian((2, 2, 1, 64), 10, torch.bfloat16)
    good = fd.fdllm_cache_attention(q, cache, table, ints(lens))
    x = gaussian((2, 1, 1, 64), 11, torch.bfloat16)
    x[1, 0, 0, 3] = math.nan
    x[0] = 0
    fd.fdllm_cache_append(cache, table[1:], ints([50]), x[1:], x[1:])
    out = fd.fdllm_cache_attention(q, cache, table, ints(lens))
    assert torch.equal(out[0], good[0]) and bool(torch.isnan(out[1]).all())


def test_one_call_is_deterministic_and_rows_do_not_mix(fd):
    """The same call twice gives the same bits, and a sequence alone gives what it gives in a
    batch up to the tolerance of both (the work is split by the whole batch's lengths)."""
    lens = [900, 17, 400]
    cache, table = ref.make_cache(fd, lens, 4, 128, 64, seed=8)
    q = gaussian((3, 32, 8, 128), 12, torch.bfloat16)
    a = fd.fdllm_cache_attention(q, cache, table, ints(lens))
    assert torch.equal(a, fd.fdllm_cache_attention(q, cache, table, ints(lens)))
    for b in range(3):
        check(fd, q[b:b + 1], cache, table[b:b + 1], lens[b:b + 1])


def test_another_stream_and_a_graph(fd):
    lens = [300, 45]
    cache, table = ref.make_cache(fd, lens, 2, 128, 64, seed=9)
    q = gaussian((2, 32, 2, 128), 13, torch.bfloat16)
    n = ints(lens)
    want = fd.fdllm_cache_attention(q, cache, table, n)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = fd.fdllm_cache_attention(q, cache, table, n, stream=other)
    other.synchronize()
    assert torch.equal(got, want)
    need = fd.fdllm_cache_attention_workspace_bytes(2, 32, 2, 2, 128)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fdllm_cache_attention(q, cache, table, n, out=out, workspace=ws)
    for shift in (0.0, 1.0):
        q.add_(shift)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fd.fdllm_cache_attention(q, cache, table, n))


def test_long_prefix(fd):
    """A prefix long enough that many CTAs share a head, against the reference."""
    lens = [20011]
    cache, table = ref.make_cache(fd, lens, 1, 128, 256, seed=10)
    check(fd, gaussian((1, 2, 4, 128), 14, torch.bfloat16, 1.5), cache, table, lens)


@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(fd, seed):
    r = torch.Generator().manual_seed(100 + seed)
    pick = lambda low, high: int(torch.randint(low, high + 1, (1,), generator=r))
    heads, group = pick(1, 4), pick(1, 5)
    D, page = (64, 128)[pick(0, 1)], (32, 64, 128, 256)[pick(0, 3)]
    B, Lq, Ln = pick(1, 5), pick(1, 90), pick(0, 90)
    lens = [pick(0, 700) * pick(0, 1) for _ in range(B)]
    new = [pick(0, Ln) for _ in range(B)]
    dtype = (torch.bfloat16, torch.float16)[pick(0, 1)]
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed=seed)
    q = gaussian((B, Lq, heads * group, D), seed, dtype, 1.5)
    k = gaussian((B, Ln, heads, D), seed + 1, dtype) if Ln else None
    v = gaussian((B, Ln, heads, D), seed + 2, dtype) if Ln else None
    check(fd, q, cache, table, lens, k, v, new if Ln else None, causal=bool(Ln) and bool(pick(0, 1)))


def check_weights(fd, q, lse, cache, table, lens, weights):
    got = fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens), weights=weights)
    want, tol = ref.key_weights(q, lse, cache, table, lens, weights)
    err = (got.cpu().double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-30)).max())
    for b, n in enumerate(lens):
        assert bool((got[b, :, n:] == 0).all())
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,Lq,Hq,heads,D,page,lens", [
    (1, 1, 2, 2, 128, 64, [1]), (3, 4, 6, 2, 64, 32, [0, 129, 77]),
    (2, 32, 4, 4, 128, 64, [400, 128]), (1, 75, 8, 2, 128, 128, [1000]),
])
def test_key_weights(fd, dtype, B, Lq, Hq, heads, D, page, lens):
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed=Lq)
    q = gaussian((B, Lq, Hq, D), Lq, dtype, 1.5)
    _, lse = fd.fdllm_cache_attention(q, cache, table, ints(lens), return_lse=True)
    width = table.shape[1] * page
    w = torch.rand(B, heads, width, generator=torch.Generator().manual_seed(1)).cuda()
    got = check_weights(fd, q, lse, cache, table, lens, w)
    zero = fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens))
    for b, n in enumerate(lens):  # every query's weights sum to 1
        total = zero[b].double().sum(-1).cpu()
        want = float(Lq * Hq // heads) if n else 0.0
        assert bool(((total - want).abs() <= 1e-4 * max(want, 1.0)).all())
    same = w.clone()
    fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens), weights=same, out=same)
    assert torch.equal(same, got)
    assert torch.equal(got, fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens), weights=w))


def test_key_weights_of_empty_rows_wrong_lengths_and_pages(fd):
    lens = [40, 40, 40]
    cache, table = ref.make_cache(fd, lens, 1, 64, 32, seed=3, min_pages=2)
    q = gaussian((3, 2, 1, 64), 5, torch.bfloat16)
    lse = torch.full((3, 2, 1), -math.inf, device="cuda")
    w = fd.fdllm_cache_key_weights(q, lse, cache, table, ints(lens))
    assert bool((w == 0).all())
    table = table.clone()
    table[2, 1] = -1
    lse[:] = 3.0
    w = fd.fdllm_cache_key_weights(q, lse, cache, table, ints([40, 65, 40]))
    assert bool(torch.isfinite(w[0]).all()) and bool(torch.isnan(w[1]).all())
    assert bool(torch.isfinite(w[2, :, :32]).all()) and bool(torch.isnan(w[2, :, 32:40]).all())
    assert bool((w[2, :, 40:] == 0).all())
    short = fd.fdllm_cache_key_weights(q, lse, cache, table, ints([40, 40, 30]), max_len=39)
    assert bool(torch.isnan(short[:2]).all()) and bool(torch.isfinite(short[2, :, :30]).all())


def test_refusals(fd):
    cache, table = ref.make_cache(fd, [40], 2, 64, 32, seed=3)
    q = gaussian((1, 2, 4, 64), 5, torch.bfloat16)
    n = ints([40])
    call = lambda **kw: fd.fdllm_cache_attention(**{**dict(q=q, cache=cache, block_table=table,
                                                           cache_lens=n), **kw})
    call()
    with pytest.raises(TypeError):
        call(q=q.float())
    with pytest.raises(TypeError):
        call(cache_lens=n.long())
    for bad in (dict(q=q[..., :32]), dict(cache_lens=ints([40, 1])), dict(k_new=q[:, :, :2]),
                dict(block_table=table.cpu()), dict(q=q.cpu()),
                dict(k_new=q[:, :, :1], v_new=q[:, :, :1])):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    for bad in (dict(q=q[:, :, :3]), dict(scale=math.nan),
                dict(workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(fd.FdllmError):
            call(**bad)
