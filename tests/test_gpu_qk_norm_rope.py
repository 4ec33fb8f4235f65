"""fdllm_qk_norm_rope against a 64-bit evaluation of its formulas.

Tolerance: half an ulp of the output type, plus 16 fp32 roundings of |u| + |v| (the pair's
normed values: norm, weight, products, sum, cosine and sine), plus the angle's 2^-31 half turns
and the 64-bit reference's own pos * 2^-53 radians."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu

FREQ = lambda pairs, base=10000.0: base ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))


def check(got, x, weight, positions, sections, inv_freq, eps, interleaved):
    want = ref.rope(x, weight, positions, sections, inv_freq, eps, interleaved)
    pairs = len(inv_freq)
    y = ref.rope(x, weight, positions * 0, sections, inv_freq, eps, interleaved)
    size = y.abs()
    if pairs:
        i = torch.arange(pairs) * 2 if interleaved else torch.arange(pairs)
        j = i + 1 if interleaved else i + pairs
        both = size[..., i] + size[..., j]
        size[..., i], size[..., j] = both, both
    far = float(positions.abs().max()) if positions.numel() else 0.0
    tol = ref.EPS[x.dtype] * want.abs() + size * (16 * 2.0 ** -24 + far * 2.0 ** -52) + \
        (2.0 ** -25 if x.dtype == torch.float16 else 1e-38)
    err = (got.cpu().double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,Hq,Hk,D,axes,interleaved", [
    (1, 32, 8, 128, 1, False), (1, 1, 1, 64, 1, True), (33, 5, 3, 128, 3, False),
    (7, 3, 1, 256, 2, True), (5, 2, 2, 96, 1, False), (3, 4, 2, 6, 1, True), (2, 1, 0, 512, 4, False),
])
def test_matches_the_formula(fd, dtype, T, Hq, Hk, D, axes, interleaved):
    g = torch.Generator().manual_seed(T * 1000 + D + axes)
    qkv = (torch.randn(T, Hq + 2 * Hk + 1, D, generator=g) * 3).to(dtype).cuda()
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk] if Hk else None
    wq = torch.randn(D, generator=g).to(dtype).cuda()
    wk = torch.randn(D, generator=g).to(dtype).cuda()
    pairs = D // 2
    sections = [pairs // axes] * (axes - 1)
    sections.append(pairs - sum(sections))
    pos = torch.randint(-5000, 5000, (axes, T), generator=g, dtype=torch.int32).cuda()
    freq = FREQ(pairs)
    oq, ok = fd.fdllm_qk_norm_rope(q, k, pos, freq, q_weight=wq, k_weight=wk, eps=1e-6,
                                   sections=sections, interleaved=interleaved)
    check(oq, q, wq, pos, sections, freq, 1e-6, interleaved)
    if Hk:
        check(ok, k, wk, pos, sections, freq, 1e-6, interleaved)


def test_many_tokens_take_the_four_token_form(fd):
    g = torch.Generator().manual_seed(2)
    q = torch.randn(4099, 3, 64, generator=g).bfloat16().cuda()
    w = torch.randn(64, generator=g).bfloat16().cuda()
    pos = torch.arange(4099, dtype=torch.int32).cuda()
    oq, _ = fd.fdllm_qk_norm_rope(q, None, pos, FREQ(32), q_weight=w)
    check(oq, q, w, pos[None], [32], FREQ(32), 1e-6, False)


@pytest.mark.parametrize("pairs,interleaved", [(0, False), (16, False), (16, True), (31, False)])
def test_partial_rotation_and_no_norm(fd, pairs, interleaved):
    g = torch.Generator().manual_seed(pairs)
    q = torch.randn(4, 2, 128, generator=g).cuda()
    k = torch.randn(4, 1, 128, generator=g).cuda()
    pos = torch.tensor([0, 1, 77, 4000], dtype=torch.int32).cuda()
    w = torch.randn(128, generator=g).cuda()
    oq, ok = fd.fdllm_qk_norm_rope(q, k, pos, FREQ(pairs), k_weight=w, interleaved=interleaved)
    check(oq, q, None, pos[None], [pairs], FREQ(pairs), 1e-6, interleaved)
    check(ok, k, w, pos[None], [pairs], FREQ(pairs), 1e-6, interleaved)


def test_far_positions_keep_their_angle(fd):
    q = torch.randn(4, 1, 128, generator=torch.Generator().manual_seed(5)).cuda()
    pos = torch.tensor([2 ** 31 - 1, -2 ** 31 + 1, 1234567, 10 ** 9], dtype=torch.int32).cuda()
    oq, _ = fd.fdllm_qk_norm_rope(q, None, pos, FREQ(64))
    check(oq, q, None, pos[None], [64], FREQ(64), 1e-6, False)


def test_in_place_odd_base_and_zero_rows(fd):
    g = torch.Generator().manual_seed(8)
    flat = torch.randn(3 * 2 * 128 + 1, generator=g).bfloat16().cuda()
    q = flat[1:].view(3, 2, 128)  # a base of 2 bytes: the element-wise form
    q[1] = 0
    before = q.clone()
    pos = torch.tensor([3, 4, 5], dtype=torch.int32).cuda()
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    oq, _ = fd.fdllm_qk_norm_rope(q, None, pos, FREQ(64), q_weight=w, out_q=q)
    assert oq.data_ptr() == q.data_ptr() and bool((q[1] == 0).all())
    check(q, before, w, pos[None], [64], FREQ(64), 1e-6, False)
    aligned = before.clone()
    fd.fdllm_qk_norm_rope(aligned, None, pos, FREQ(64), q_weight=w, out_q=aligned)
    check(aligned, before, w, pos[None], [64], FREQ(64), 1e-6, False)


def test_no_tokens_and_another_stream(fd):
    empty = torch.empty(0, 2, 64, device="cuda")
    oq, ok = fd.fdllm_qk_norm_rope(empty, empty, torch.empty(0, dtype=torch.int32, device="cuda"),
                                   FREQ(32))
    assert oq.shape == (0, 2, 64) and ok.shape == (0, 2, 64)
    q = torch.randn(64, 8, 128, device="cuda")
    pos = torch.arange(64, dtype=torch.int32, device="cuda")
    want, _ = fd.fdllm_qk_norm_rope(q, None, pos, FREQ(64))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got, _ = fd.fdllm_qk_norm_rope(q, None, pos, FREQ(64), stream=other)
    other.synchronize()
    assert torch.equal(got, want)


def test_refusals(fd):
    q = torch.zeros(2, 2, 64, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    call = lambda **kw: fd.fdllm_qk_norm_rope(**{**dict(q=q, k=None, positions=pos,
                                                        inv_freq=FREQ(32)), **kw})
    call()
    for bad in (dict(inv_freq=FREQ(33)), dict(eps=-1.0), dict(eps=math.nan),
                dict(inv_freq=torch.full((32,), math.inf, dtype=torch.float64)),
                dict(sections=[31])):
        with pytest.raises(fd.FdllmError):
            call(**bad)
    for bad in (dict(inv_freq=FREQ(32).float()), dict(q=q[..., ::2]), dict(positions=pos[:1]),
                dict(q=q.cpu()), dict(k=torch.zeros(3, 2, 64, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    with pytest.raises(TypeError):
        call(positions=pos.long())
