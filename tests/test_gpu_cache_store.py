"""fdllm_cache_append and fdllm_cache_read: the held values are exactly those of the documented
fp32 quantisation (no tolerance), and slots outside a call keep what they held."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu


def rows(shape, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * (1 + 4 * (torch.rand(shape[-1], generator=g) < 0.1))
    return (x + 0.3).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("D,page,heads,n,start", [
    (128, 64, 3, 1, [0, 1, 63]), (128, 32, 2, 65, [0, 31, 7]), (64, 128, 1, 200, [5, 0, 128]),
    (64, 32, 2, 2, [30, 31, 32]), (128, 256, 1, 33, [255, 3, 8]), (64, 64, 2, 64, [0, 64, 32]),
])
def test_written_rows_read_back_as_their_held_values(fd, dtype, D, page, heads, n, start):
    B = 3
    per = -(-(max(start) + n) // page)
    cache = fd.KvCache.empty(B * per + 2, heads, page, D)
    for t in (cache.k_codes, cache.v_codes):
        t.random_(0, 256)
    cache.k_affine.normal_()
    cache.v_affine.normal_()
    table = torch.randperm(B * per + 2)[:B * per].view(B, per).int().cuda()
    at = torch.tensor(start, dtype=torch.int32).cuda()
    before = fd.fdllm_cache_read(cache, table, None, per * page, torch.float32)
    # strided rows: keys and values of one packed projection
    kv = rows((B, n, 2 * heads + 1, D), n, dtype)
    k, v = kv[:, :, :heads], kv[:, :, heads:2 * heads]
    fd.fdllm_cache_append(cache, table, at, k, v)
    after = fd.fdllm_cache_read(cache, table, None, per * page, torch.float32)
    got = fd.fdllm_cache_read(cache, table, at, n, dtype)
    for x, old, new, back in zip((k, v), before, after, got):
        held = ref.values(x).float()
        for b, s in enumerate(start):
            assert torch.equal(new[b, s:s + n].cpu(), held[b])
            assert torch.equal(new[b, :s], old[b, :s])
            assert torch.equal(new[b, s + n:], old[b, s + n:])
        assert torch.equal(back.cpu(), held.to(dtype))


def test_counts_cut_the_rows_and_pad_the_reading(fd):
    cache = fd.KvCache.empty(8, 2, 32, 64)
    table = torch.arange(8, dtype=torch.int32).view(2, 4).cuda()
    k, v = rows((2, 40, 2, 64), 1, torch.bfloat16), rows((2, 40, 2, 64), 2, torch.bfloat16)
    fd.fdllm_cache_append(cache, table, None, k, v)
    count = torch.tensor([0, 37], dtype=torch.int32).cuda()
    k2, v2 = k + 1, v - 1
    fd.fdllm_cache_append(cache, table, None, k2, v2, count=count)
    rk, rv = fd.fdllm_cache_read(cache, table, None, 40, torch.float32)
    assert torch.equal(rk[0].cpu(), ref.values(k[0]).float())
    assert torch.equal(rk[1, :37].cpu(), ref.values(k2[1, :37]).float())
    assert torch.equal(rv[1, 37:].cpu(), ref.values(v[1, 37:]).float())
    rk, rv = fd.fdllm_cache_read(cache, table, None, 40, torch.bfloat16, count=count)
    assert bool((rk[0] == 0).all()) and bool((rk[1, 37:] == 0).all())
    assert torch.equal(rv[1, :37].cpu(), ref.values(v2[1, :37]).bfloat16())


def test_special_rows(fd):
    """Constant rows, ties between codes, non-finite rows, the largest and smallest numbers."""
    D = 64
    x = torch.zeros(1, 10, 1, D)
    x[0, 0] = 2.5
    x[0, 1] = torch.arange(D).float() * 0.5            # halves of a step
    x[0, 2] = torch.randn(D)
    x[0, 2, 0, 5] = math.nan
    x[0, 3] = torch.randn(D)
    x[0, 3, 0, 7] = math.inf
    x[0, 4] = torch.randn(D)
    x[0, 4, 0, 9] = -math.inf
    x[0, 5] = torch.linspace(-3e38, 3e38, D)           # range overflows fp32
    x[0, 6] = torch.linspace(0, 1e38, D)
    x[0, 7] = torch.linspace(0, 1e-44, D)              # subnormal steps
    x[0, 8] = torch.linspace(-1, 1, D) * 1e-30
    x[0, 9, 0, 3] = -0.0
    k = x.cuda()
    cache = fd.KvCache.empty(1, 1, 32, D)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    fd.fdllm_cache_append(cache, table, None, k, k)
    rk, rv = fd.fdllm_cache_read(cache, table, None, 10, torch.float32)
    want = ref.values(x).float()
    assert bool(torch.isnan(want[0, 2:6]).all()) and bool(torch.isfinite(want[0, 6:]).all())
    for got in (rk, rv):
        assert torch.equal(torch.isnan(got).cpu(), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got).cpu(), torch.nan_to_num(want))


def test_slots_that_do_not_exist(fd):
    cache = fd.KvCache.empty(2, 1, 32, 64)
    k = rows((3, 40, 1, 64), 3, torch.float32)
    # sequence 0: second page out of range; 1: starts behind the table; 2: negative start
    table = torch.tensor([[0, 9], [1, -1], [1, 1]], dtype=torch.int32).cuda()
    fd.fdllm_cache_append(cache, table[:1], None, k[:1], k[:1])
    rk, _ = fd.fdllm_cache_read(cache, table[:1], None, 70, torch.float32)
    assert torch.equal(rk[0, :32].cpu(), ref.values(k[0, :32]).float())
    assert bool(torch.isnan(rk[0, 32:]).all())
    saved = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_affine, cache.v_affine)]
    start = torch.tensor([64, -3], dtype=torch.int32).cuda()
    fd.fdllm_cache_append(cache, table[1:], start, k[1:], k[1:])
    for a, b in zip(saved, (cache.k_codes, cache.v_codes, cache.k_affine, cache.v_affine)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    rk, rv = fd.fdllm_cache_read(cache, table[1:], start, 40, torch.float32)
    assert bool(torch.isnan(rk[0]).all()) and bool(torch.isnan(rv[1, :3]).all())


def test_pages_behind_32_bits(fd):
    """A pool whose codes span more than 2^32 bytes: its last pages are written and read."""
    pages, heads, page, D = 70000, 16, 64, 128
    cache = fd.KvCache.empty(pages, heads, page, D)
    assert cache.k_codes.numel() > 2 ** 32
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32).cuda()
    k, v = rows((1, 150, heads, D), 4, torch.bfloat16), rows((1, 150, heads, D), 5, torch.bfloat16)
    fd.fdllm_cache_append(cache, table, None, k, v)
    rk, rv = fd.fdllm_cache_read(cache, table, None, 150, torch.bfloat16)
    assert torch.equal(rk.cpu(), ref.values(k).bfloat16())
    assert torch.equal(rv.cpu(), ref.values(v).bfloat16())
    lens = torch.tensor([150], dtype=torch.int32).cuda()
    q = rows((1, 3, heads, D), 6, torch.bfloat16)
    out, lse = fd.fdllm_cache_attention(q, cache, table, lens, return_lse=True)
    small, where = fd.KvCache.empty(3, heads, page, D), torch.arange(3, dtype=torch.int32).view(1, 3).cuda()
    fd.fdllm_cache_append(small, where, None, k, v)
    out2, lse2 = fd.fdllm_cache_attention(q, small, where, lens, return_lse=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_refusals(fd):
    cache = fd.KvCache.empty(4, 2, 32, 64)
    table = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    k = torch.zeros(1, 3, 2, 64, device="cuda")
    with pytest.raises(ValueError):
        fd.KvCache(cache.k_codes, cache.v_codes[:2], cache.k_affine, cache.v_affine)
    for page, D in ((48, 64), (16, 64), (512, 64), (32, 96)):
        odd = fd.KvCache.empty(2, 1, page, D)
        with pytest.raises(fd.FdllmError):
            fd.fdllm_cache_read(odd, table, None, 3)
    with pytest.raises(ValueError):
        fd.fdllm_cache_append(cache, table, None, k, k[:, :2])
    with pytest.raises(TypeError):
        fd.fdllm_cache_append(cache, table, None, k.double(), k.double())
    with pytest.raises(fd.FdllmError) as e:  # rows that are not 16-byte aligned
        flat = torch.zeros(1 + k.numel(), device="cuda")
        fd.fdllm_cache_append(cache, table, None, flat[1:].view_as(k), k)
    assert e.value.status == 2
    with pytest.raises(TypeError):
        fd.fdllm_cache_append(cache, table, torch.zeros(1, device="cuda"), k, k)
    with pytest.raises(ValueError):
        fd.fdllm_cache_read(cache, table.cpu(), None, 3)
