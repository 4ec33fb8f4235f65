"""fdllm_tree_mask against walks up the parents, and fdllm_cache_tree_attention against a 64-bit
evaluation of its formula, with cache_ref.py's tolerances."""
import math

import pytest
import torch

import cache_ref as ref
import draft_ref
from test_gpu_cache_attention import gaussian, ints

pytestmark = pytest.mark.gpu


def trees(B, M, seed, reach=6):
    g = torch.Generator().manual_seed(seed)
    parents = torch.arange(M) - 1 - (torch.rand(B, M, generator=g) ** 2 * reach).long()
    parents = parents.clamp_min(0).int()
    parents[:, 0] = -1
    return parents


@pytest.mark.parametrize("B,M", [(1, 1), (3, 2), (2, 31), (2, 32), (5, 33), (2, 64), (1, 100), (3, 257),
                                 (2, 1000), (2, 1024)])
def test_tree_mask(fd, B, M):
    for parents in (trees(B, M, M), trees(B, M, M, 1e9), (torch.arange(M) - 1).int().expand(B, M).contiguous()):
        if M > 5:
            parents = parents.clone()
            parents[0, 4], parents[0, 5] = 4, -3  # detached
        for lens in (None, [(7 * b + 3) % (M + 3) - 1 for b in range(B)]):
            mask, depth = fd.fdllm_tree_mask(parents.cuda(), None if lens is None else ints(lens))
            sees, want = draft_ref.tree_mask(parents, lens)
            assert torch.equal(mask.cpu(), draft_ref.bits(sees)) and torch.equal(depth.cpu().long(), want)


def reference(q, cache, table, lens, k, v, new, sees, scale=None):
    """The formula in fp64: (out, lse) and their tolerances."""
    B, Lq, Hq, D = q.shape
    group = Hq // cache.heads
    scale = D ** -0.5 if scale is None else scale
    kd, vd = ref.unpack_cache(cache)
    k_reach = ref.row_reach(cache.k_affine, D)
    v_reach = (15 * cache.v_affine[..., :1].cpu().double()).expand(-1, -1, -1, D)
    out = torch.zeros(B, Lq, Hq, D, dtype=torch.float64)
    lse = torch.full((B, Lq, Hq), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n, m = int(lens[b]), k.shape[1] if new is None else int(new[b])
        ck, cv, ckr, cvr = (ref.sequence(x, table[b], cache.page_size, n) for x in (kd, vd, k_reach, v_reach))
        cvr = torch.maximum(cv.abs(), cvr)
        ok, ov = (x[b, :m].cpu().double().transpose(0, 1) for x in (k, v))
        for i in range(Lq):
            on = sees[b, i, :m]
            for h in range(Hq):
                g = h // group
                kh, vh = torch.cat((ck[g], ok[g][on])), torch.cat((cv[g], ov[g][on]))
                if not len(kh):
                    continue
                krh, vrh = torch.cat((ckr[g], ok[g][on].abs())), torch.cat((cvr[g], ov[g][on].abs()))
                x64 = q[b, i, h].cpu().double()
                x = kh @ x64 * scale
                d = 2.0 ** -21 * abs(scale) * float((krh @ x64.abs()).max())
                lse[b, i, h] = torch.logsumexp(x, 0)
                p = torch.softmax(x, 0)
                out[b, i, h] = p @ vh
                tol[b, i, h] = ref.EPS[q.dtype] * out[b, i, h].abs() + (2.0 ** -11 + 2 * d) * (p @ vrh) + 1e-30
                tol_lse[b, i, h] = d + 4 * 2.0 ** -24 * max(1.0, abs(float(lse[b, i, h]))) + 1e-6
    return out, lse, tol, tol_lse


def check(fd, q, cache, table, lens, k, v, sees, new=None, scale=None):
    out, lse = fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, v, draft_ref.bits(sees).cuda(),
                                             None if new is None else ints(new), scale, return_lse=True)
    w_out, w_lse, tol, tol_lse = reference(q, cache, table, lens, k, v, new, sees, scale)
    err = (out.cpu().double() - w_out).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp_min(1e-30)).max())
    empty = torch.isinf(w_lse)
    assert torch.equal(torch.isneginf(lse.cpu()), empty)
    gap = (lse.cpu().double() - w_lse).abs()[~empty]
    assert bool((gap <= tol_lse[~empty]).all())
    assert fd.fdllm_cache_status() == 0
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,Hq,heads,D,page,lens", [
    (1, 4, 2, 128, 64, [65, 0, 3]),
    (7, 8, 2, 128, 32, [0, 130]),
    (16, 2, 2, 128, 64, [333]),
    (17, 7, 1, 64, 128, [128, 0, 31]),
    (31, 3, 3, 64, 256, [500]),
    (33, 6, 2, 128, 64, [100, 1]),
    (64, 2, 1, 128, 64, [129]),
    (129, 2, 2, 64, 32, [40, 0]),
    (200, 3, 1, 128, 64, [0]),
])
def test_trees(fd, dtype, M, Hq, heads, D, page, lens):
    B = len(lens)
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed=M + page)
    qkv = gaussian((B, M, Hq + 2 * heads, D), M, dtype)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + heads], qkv[:, :, Hq + heads:].contiguous()
    parents = trees(B, M, M)
    sees, _ = draft_ref.tree_mask(parents)
    check(fd, q, cache, table, lens, k, v, sees)
    new = [max(0, M - 5 * (b + 1)) for b in range(B)]
    mask, _ = fd.fdllm_tree_mask(parents.cuda(), ints(new))
    short, _ = draft_ref.tree_mask(parents, new)
    k, v = k.clone(), v.clone()
    for b, m in enumerate(new):  # padding
        k[b, m:], v[b, m:] = math.nan, math.inf
    out, _ = check(fd, q, cache, table, lens, k, v, short, new)
    got = fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, v, mask, ints(new))
    assert torch.equal(got, out)
    # bits behind the count are not read as set
    wild = mask.clone()
    for b, m in enumerate(new):
        full = torch.ones(M, M, dtype=torch.bool)
        full[:, :m] = short[b, :, :m]
        wild[b] = draft_ref.bits(full).cuda()
    assert torch.equal(got, fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, v, wild, ints(new)))


@pytest.mark.parametrize("seed", range(14))
def test_any_pattern(fd, seed):
    """Patterns that are no trees: rows that see nothing, rows that see one late key, other counts of
    queries than of keys."""
    r = torch.Generator().manual_seed(200 + seed)
    pick = lambda low, high: int(torch.randint(low, high + 1, (1,), generator=r))
    heads, group = pick(1, 3), pick(1, 5)
    D, page = (64, 128)[pick(0, 1)], (32, 64, 128, 256)[pick(0, 3)]
    B, Lq, Ln = pick(1, 4), pick(1, 90), pick(1, 290)
    lens = [pick(0, 400) * pick(0, 1) for _ in range(B)]
    new = [pick(0, Ln) for _ in range(B)]
    dtype = (torch.bfloat16, torch.float16)[pick(0, 1)]
    cache, table = ref.make_cache(fd, lens, heads, D, page, seed=seed)
    q = gaussian((B, Lq, heads * group, D), seed, dtype, 1.5)
    k, v = gaussian((B, Ln, heads, D), seed + 1, dtype), gaussian((B, Ln, heads, D), seed + 2, dtype)
    sees = torch.rand(B, Lq, Ln, generator=r) < (0.5, 0.05, 0.002)[seed % 3]
    sees[:, ::4] = False
    sees[0, 0, :] = False
    sees[0, 0, Ln - 1] = True
    check(fd, q, cache, table, lens, k, v, sees, new, scale=(None, -0.3, 2.0)[seed % 3])


def test_scores_that_grow_behind_unseen_keys(fd):
    """A row's first key comes late and scores far from those that others see: its reference starts
    where it first sees a key."""
    cache, table = ref.make_cache(fd, [0], 1, 128, 64, seed=3)
    M = 150
    k = gaussian((1, M, 1, 128), 4, torch.float16, 0.05)
    k[0, :, 0, 0] = torch.arange(M, device="cuda", dtype=torch.float16) - 75
    v = gaussian((1, M, 1, 128), 5, torch.float16)
    for lead in (12.0, -12.0):
        q = gaussian((1, M, 1, 128), 6, torch.float16, 0.05)
        q[..., 0] = lead
        sees = torch.tril(torch.ones(M, M, dtype=torch.bool))[None] & (torch.rand(1, M, M, generator=torch.Generator().manual_seed(7)) < 0.3)
        check(fd, q, cache, table, [0], k, v, sees, scale=1.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,group", [(20, 1), (60, 3), (140, 1)])
def test_non_finite_values_reach_those_who_see_them(fd, dtype, M, group):
    lens = [37, 0]
    cache, table = ref.make_cache(fd, lens, 2, 64, 32, seed=9)
    q = gaussian((2, M, 2 * group, 64), 1, dtype)
    k, v = gaussian((2, M, 2, 64), 2, dtype), gaussian((2, M, 2, 64), 3, dtype)
    parents = trees(2, M, 11)
    sees, _ = draft_ref.tree_mask(parents)
    clean, _ = check(fd, q, cache, table, lens, k, v, sees)
    v[0, 3, 1, 5], v[0, 9, 1, 6], v[1, M - 1, 0, 7] = math.nan, math.inf, -math.inf
    k[1, 6, 1, 0] = math.nan
    out = fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, v, draft_ref.bits(sees).cuda())
    want = torch.zeros(2, M, 2 * group, 64, dtype=torch.bool)
    want[0, sees[0, :, 3], group:, 5] = True
    want[0, sees[0, :, 9], group:, 6] = True
    want[1, sees[1, :, M - 1], :group, 7] = True
    want[1, sees[1, :, 6], group:] = True
    assert torch.equal(torch.isnan(out).cpu(), want)
    assert torch.equal(out.cpu()[~want], clean.cpu()[~want])


def test_a_chains_bits_are_the_causal_order(fd):
    for M, group, D in ((5, 1, 128), (40, 4, 64), (300, 1, 128)):
        lens = [90, 0]
        cache, table = ref.make_cache(fd, lens, 2, D, 64, seed=M)
        q, k, v = (gaussian((2, M, h, D), i, torch.bfloat16) for i, h in enumerate((2 * group, 2, 2)))
        parents = (torch.arange(M) - 1).int().expand(2, M).contiguous().cuda()
        mask, depth = fd.fdllm_tree_mask(parents)
        assert torch.equal(depth.cpu(), torch.arange(M).int().expand(2, M))
        out, lse = fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, v, mask, return_lse=True)
        want, want_lse = fd.fdllm_cache_attention(q, cache, table, ints(lens), k, v, causal=True, return_lse=True)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_wrong_lengths_and_pages_report_nan(fd):
    lens = [40, 40, 40, 40]
    cache, table = ref.make_cache(fd, lens, 2, 64, 32, seed=6, min_pages=2)
    q, k = gaussian((4, 3, 2, 64), 8, torch.bfloat16), gaussian((4, 3, 2, 64), 9, torch.bfloat16)
    mask, _ = fd.fdllm_tree_mask(ints([[-1, 0, 0]] * 4))
    good = fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, k, mask)
    table = table.clone()
    table[3, 1] = cache.pages
    out = fd.fdllm_cache_tree_attention(q, cache, table, ints([40, -1, 65, 40]), k, k, mask)
    assert torch.equal(out[0], good[0]) and bool(torch.isnan(out[1:]).all())
    out = fd.fdllm_cache_tree_attention(q, cache, table, ints(lens), k, k, mask, ints([3, 4, -1, 0]))
    assert torch.equal(out[0], good[0]) and bool(torch.isnan(out[1:]).all())


def test_another_stream_and_a_graph(fd):
    lens = [300, 45]
    cache, table = ref.make_cache(fd, lens, 2, 128, 64, seed=9)
    M = 24
    q, k, v = (gaussian((2, M, 2, 128), i, torch.bfloat16) for i in range(3))
    parents, n = trees(2, M, 1).cuda(), ints(lens)
    mask, depth = fd.fdllm_tree_mask(parents)
    want = fd.fdllm_cache_tree_attention(q, cache, table, n, k, v, mask)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    m2, _ = fd.fdllm_tree_mask(parents, stream=other)
    got = fd.fdllm_cache_tree_attention(q, cache, table, n, k, v, m2, stream=other)
    other.synchronize()
    assert torch.equal(got, want)
    ws = torch.empty(fd.fdllm_cache_attention_workspace_bytes(2, M, 2, 2, 128), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fdllm_tree_mask(parents, out_mask=mask, out_depth=depth)
        fd.fdllm_cache_tree_attention(q, cache, table, n, k, v, mask, out=out, workspace=ws)
    for turn in range(3):
        parents.copy_(trees(2, M, turn + 5))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fd.fdllm_cache_tree_attention(q, cache, table, n, k, v, fd.fdllm_tree_mask(parents)[0]))


def test_refusals(fd):
    cache, table = ref.make_cache(fd, [40], 2, 64, 32, seed=3)
    q, k = gaussian((1, 2, 4, 64), 5, torch.bfloat16), gaussian((1, 2, 2, 64), 5, torch.bfloat16)
    mask, _ = fd.fdllm_tree_mask(ints([[-1, 0]]))
    call = lambda **kw: fd.fdllm_cache_tree_attention(**{**dict(
        q=q, cache=cache, block_table=table, cache_lens=ints([40]), k_new=k, v_new=k, mask=mask), **kw})
    call()
    for bad in (dict(mask=mask.long()), dict(mask=mask[:, :1]), dict(mask=mask.cpu()), dict(v_new=k[:, :1]),
                dict(k_new=k.half()), dict(q=q.float())):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    for bad in (dict(scale=math.inf), dict(workspace=torch.empty(128, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(fd.FdllmError):
            call(**bad)
    for bad in (ints([0, 1]), ints([[0]]).long(), ints([[0]]).cpu()):
        with pytest.raises((ValueError, TypeError)):
            fd.fdllm_tree_mask(bad)
    with pytest.raises(fd.FdllmError):
        fd.fdllm_tree_mask(torch.zeros(1, 1025, dtype=torch.int32, device="cuda"))
