"""fdllm_distill_loss, fdllm_distill_grad and fdllm_distill_step against their formulas in 64 bits; the
tolerances are those of draft_ref.py."""
import math

import pytest
import torch

import draft_ref as ref

pytestmark = pytest.mark.gpu

BF, HF, FP = torch.bfloat16, torch.float16, torch.float32


def inputs(B, L, V, K, dtype, seed, rest, masked=0.6, top_dtype=None, temperature=1.0):
    g = torch.Generator().manual_seed(seed)
    x = 1.5 * torch.randn(B, L, V, generator=g)
    index = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(B * L)]).view(B, L, K)
    top = 3 + 4 * torch.rand(B, L, K, generator=g)
    x.scatter_(2, index, top + 0.7 * torch.randn(B, L, K, generator=g))
    top = top.to(top_dtype or FP)
    lse = None
    if rest:
        held = 0.5 + 0.45 * torch.rand(B, L, generator=g)
        lse = (torch.logsumexp(top.float() / temperature, -1) - held.log()).contiguous().cuda()
    mask = (torch.rand(B, L, generator=g) < masked).to(torch.uint8) * 255
    weights = torch.randn(B, L, generator=g)
    return dict(logits=x.to(dtype).cuda(), mask=mask.cuda(), top_index=index.int().cuda(),
                top_logits=top.cuda(), teacher_lse=lse, temperature=temperature), weights.cuda()


def check(fd, kw, weights):
    """All three calls, and autograd, against the reference."""
    want = ref.distill(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], kw["teacher_lse"],
                       kw["temperature"], weights)
    stats = torch.empty((*kw["mask"].shape, 4), device="cuda")
    loss = fd.fdllm_distill_loss(out_stats=stats, **kw)
    grad = fd.fdllm_distill_grad(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], stats,
                                 weights, kw["teacher_lse"], kw["temperature"])
    step = fd.fdllm_distill_step(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], weights,
                                 kw["teacher_lse"], kw["temperature"])
    x = kw["logits"].detach().requires_grad_()
    auto = fd.fdllm_distill_loss(**{**kw, "logits": x})
    auto.backward(weights)
    for got, exact, tol in ((loss, *want[:2]), (step[0], *want[:2]), (auto.detach(), *want[:2]),
                            (grad, *want[2:]), (step[1], *want[2:]), (x.grad, *want[2:])):
        got = got.cpu().double()
        nan = torch.isnan(exact)
        assert torch.equal(torch.isnan(got), nan)
        err = (got - exact).abs()[~nan]
        assert bool((err <= tol[~nan]).all()), float((err / tol[~nan].clamp_min(1e-40)).max())
    assert fd.fdllm_cache_status() == 0
    out = kw["mask"] == 0
    assert bool((loss[out] == 0).all()) and bool((grad[out] == 0).all()) and bool((step[1][out] == 0).all())
    return step


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("B,L,V,K", [(1, 1, 1, 1), (1, 2, 2, 1), (2, 3, 7, 3), (2, 2, 8, 8), (1, 5, 513, 17),
                                     (3, 2, 4099, 64), (2, 2, 8192, 1000), (1, 2, 50021, 5)])
def test_shapes(fd, rest, dtype, B, L, V, K):
    kw, weights = inputs(B, L, V, K, dtype, B + L + V + K, rest, masked=0.8)
    check(fd, kw, weights)


@pytest.mark.parametrize("seed", range(12))
def test_random(fd, seed):
    r = torch.Generator().manual_seed(seed)
    pick = lambda low, high: int(torch.randint(low, high + 1, (1,), generator=r))
    V = pick(3, 3000)
    K = pick(1, min(V, 300))
    kw, weights = inputs(pick(1, 4), pick(1, 9), V, K, (BF, HF, FP)[pick(0, 2)], seed, bool(pick(0, 1)),
                         top_dtype=(BF, HF, FP)[pick(0, 2)], temperature=(0.3, 1.0, 2.5)[pick(0, 2)])
    gone = torch.rand(kw["top_index"].shape, generator=r) < 0.2  # absent entries
    kw["top_index"][gone.cuda()] = torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1])[pick(0, 3)]
    check(fd, kw, weights)


def test_full_vocabulary(fd):
    for dtype, rest in ((BF, True), (FP, False)):
        kw, weights = inputs(1, 3, 126464, 64, dtype, 5, rest, masked=1.1)
        check(fd, kw, weights)


def test_largest_vocabulary(fd):
    kw, weights = inputs(1, 2, 1 << 20, 1024, BF, 6, True, masked=1.1)
    check(fd, kw, weights)


@pytest.mark.parametrize("rest", [False, True])
def test_tokens_listed_more_than_once(fd, rest):
    kw, weights = inputs(2, 4, 600, 48, FP, 7, rest)
    kw["top_index"][:, :, 10:30] = kw["top_index"][:, :, :20]
    kw["top_index"][0, 0] = 5
    if rest:
        kw["teacher_lse"] += 1.0
    a = check(fd, kw, weights)
    b = fd.fdllm_distill_step(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], weights,
                              kw["teacher_lse"])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_masked_position_and_no_listed_token(fd):
    kw, weights = inputs(2, 3, 100, 4, BF, 8, False)
    kw["mask"][:] = 0
    kw["logits"][:] = math.nan
    check(fd, kw, weights)
    kw, weights = inputs(2, 3, 100, 4, BF, 8, False, masked=1.1)
    kw["top_index"][:] = -1
    loss, grad = check(fd, kw, weights)
    assert bool((loss == 0).all()) and bool((grad == 0).all())
    kw["teacher_lse"] = torch.zeros(2, 3, device="cuda")  # the rest has all of the mass: r = 1
    check(fd, kw, weights)


def test_every_token_listed(fd):
    """No other token: the rest's term is 0, whatever rounding leaves of R."""
    kw, weights = inputs(2, 3, 64, 64, FP, 9, True, masked=1.1)
    kw["teacher_lse"] = torch.logsumexp(kw["top_logits"], -1)
    check(fd, kw, weights)
    kw["teacher_lse"] += 0.3
    check(fd, kw, weights)


@pytest.mark.parametrize("dtype", [BF, HF, FP])
def test_a_student_sure_of_listed_tokens(fd, dtype):
    """The rest has e^-200 of the student's mass: its logarithm and its gradient are there all the
    same."""
    kw, weights = inputs(2, 3, 700, 5, dtype, 10, True, masked=1.1)
    kw["logits"].scatter_(2, kw["top_index"].long(), 230.0)
    kw["logits"][0, 0, 3] = -math.inf
    loss, grad = check(fd, kw, weights)
    assert bool((loss > 5).all())


@pytest.mark.parametrize("dtype", [BF, HF, FP])
def test_values_of_any_size(fd, dtype):
    low = torch.finfo(dtype).min
    kw, weights = inputs(4, 2, 300, 6, dtype, 11, False, masked=1.1)
    kw["logits"][0] = -math.inf
    kw["logits"][0].scatter_(1, kw["top_index"][0].long(), 1.0)  # all other tokens masked out
    kw["logits"][1] = low
    kw["logits"][2, :, ::2] = low
    kw["logits"][3] = 6e4 if dtype == HF else 1e38
    check(fd, kw, weights)
    kw["teacher_lse"] = torch.logsumexp(kw["top_logits"], -1) + 0.5
    check(fd, kw, weights)


def test_a_listed_token_that_the_student_rules_out(fd):
    kw, weights = inputs(1, 2, 50, 3, FP, 12, False, masked=1.1)
    kw["logits"][0, 0, kw["top_index"][0, 0, 1].long()] = -math.inf
    stats = torch.empty(1, 2, 4, device="cuda")
    loss = fd.fdllm_distill_loss(out_stats=stats, **kw)
    assert loss[0, 0].item() == math.inf and math.isfinite(loss[0, 1].item())
    grad = fd.fdllm_distill_step(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], weights)[1]
    want = ref.distill(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], None, 1.0, weights)
    assert bool(((grad.cpu().double() - want[2]).abs() <= want[3]).all())


@pytest.mark.parametrize("dtype", [BF, HF, FP])
def test_non_finite_rows(fd, dtype):
    kw, weights = inputs(2, 4, 130, 6, dtype, 13, False, masked=1.1, top_dtype=FP)
    kw["logits"][0, 0, 129] = math.nan
    kw["logits"][0, 1, 0] = math.inf
    kw["logits"][0, 2] = -math.inf
    kw["logits"][0, 3, kw["top_index"][0, 3, 2].long()] = math.nan
    kw["top_logits"][1, 0, 1] = math.nan
    kw["top_logits"][1, 1, 1] = -math.inf  # no mass: nothing
    kw["top_logits"][1, 2, 1] = math.inf
    loss, grad = check(fd, kw, weights)
    assert torch.isnan(loss).tolist() == [[True] * 4, [True, False, True, False]]


def test_in_place(fd):
    for dtype, V in ((BF, 4099), (HF, 126464), (FP, 126464), (FP, 301)):
        kw, weights = inputs(2, 6, V, 33, dtype, 14, True)
        want = fd.fdllm_distill_step(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], weights,
                                     kw["teacher_lse"])
        x = kw["logits"].clone()
        loss, grad = fd.fdllm_distill_step(x, kw["mask"], kw["top_index"], kw["top_logits"], weights,
                                           kw["teacher_lse"], out_grad=x)
        assert grad.data_ptr() == x.data_ptr()
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])


def test_gradient_by_differences(fd):
    """The loss of fp32 logits moved along a direction: its slope is the gradient's product with it.
    A step h leaves h^2 times a third derivative (below 1 here) and two losses' errors over 2 h."""
    for rest in (False, True):
        kw, _ = inputs(1, 4, 90, 7, FP, 15, rest, masked=1.1)
        one = torch.ones(1, 4, device="cuda")
        grad = fd.fdllm_distill_step(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], one,
                                     kw["teacher_lse"])[1]
        way = torch.nn.functional.normalize(
            torch.randn(1, 4, 90, generator=torch.Generator().manual_seed(1)), dim=-1).cuda()
        h = 2.0 ** -6
        up, down = (fd.fdllm_distill_loss(**{**kw, "logits": kw["logits"] + s * h * way}) for s in (1, -1))
        slope = (up - down).double() / (2 * h)
        tol = ref.distill(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], kw["teacher_lse"])[1]
        err = (slope - (grad.double() * way.double()).sum(-1)).abs().cpu()
        # (the moved logits' rounding, 2^-24 of up to 8, counts in both losses)
        assert bool((err <= h * h + (2 * tol + 2 * 8 * 2.0 ** -24) / (2 * h) * 1.5).all())


def test_autograd_inside_a_graph_of_operations(fd):
    kw, weights = inputs(2, 3, 200, 5, FP, 16, True)
    w = torch.randn(200, 200, generator=torch.Generator().manual_seed(2)).cuda().requires_grad_()
    x = kw["logits"]
    count = (kw["mask"] != 0).sum()
    total = fd.fdllm_distill_loss(**{**kw, "logits": x @ w}).sum() / count
    total.backward()
    y = (x @ w.detach())
    each = (torch.ones(2, 3, device="cuda") / count)
    dy = fd.fdllm_distill_step(y, kw["mask"], kw["top_index"], kw["top_logits"], each, kw["teacher_lse"])[1]
    assert torch.equal(w.grad, (x.flatten(0, 1).t() @ dy.flatten(0, 1)))
    z = y.clone().requires_grad_()
    with pytest.raises(RuntimeError):
        torch.autograd.grad(fd.fdllm_distill_loss(**{**kw, "logits": z}).sum(), z, create_graph=True)
    with torch.no_grad():
        assert fd.fdllm_distill_loss(**{**kw, "logits": x @ w}).requires_grad is False
    with pytest.raises(ValueError):
        fd.fdllm_distill_loss(**{**kw, "logits": x @ w}, stream=torch.cuda.Stream())
    with pytest.raises(ValueError):
        fd.fdllm_distill_loss(**{**kw, "logits": x @ w, "top_logits": kw["top_logits"].requires_grad_()})


def test_autograd_is_not_captured(fd):
    """Neither pass: capture ends with an error of the call, and eager work goes on."""
    kw, weights = inputs(2, 3, 200, 5, BF, 20, False)
    x = kw["logits"].requires_grad_()
    eager = fd.fdllm_distill_loss(**kw)
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            fd.fdllm_distill_loss(**kw)
    grad, = torch.autograd.grad(eager, x, weights)
    step = fd.fdllm_distill_step(x, kw["mask"], kw["top_index"], kw["top_logits"], weights)
    assert torch.equal(grad, step[1])


def test_a_gradient_over_saved_logits_is_seen(fd):
    kw, weights = inputs(1, 3, 200, 5, FP, 21, False)
    x = (kw["logits"] * 1.0).requires_grad_()
    y = x * 2.0
    loss = fd.fdllm_distill_loss(**{**kw, "logits": y})
    fd.fdllm_distill_step(y, kw["mask"], kw["top_index"], kw["top_logits"], weights, out_grad=y)
    with pytest.raises(RuntimeError):
        loss.backward(weights)
    with torch.inference_mode():
        z = kw["logits"] * 1.0
        fd.fdllm_distill_step(z, kw["mask"], kw["top_index"], kw["top_logits"], weights, out_grad=z)


def test_a_gradient_over_another_view_of_saved_logits_is_seen(fd):
    kw, weights = inputs(1, 3, 200, 5, FP, 22, False)
    rest = (kw["mask"], kw["top_index"], kw["top_logits"])
    stats = torch.empty(1, 3, 4, device="cuda")
    for call in (lambda y: fd.fdllm_distill_step(y.detach(), *rest, weights, out_grad=y.detach()),
                 lambda y: fd.fdllm_distill_grad(y.detach(), *rest, stats, weights, out_grad=y.detach())):
        y = (kw["logits"] * 1.0).requires_grad_() * 2.0
        loss = fd.fdllm_distill_loss(**{**kw, "logits": y})
        fd.fdllm_distill_loss(out_stats=stats, **{**kw, "logits": y.detach()})
        call(y)
        with pytest.raises(RuntimeError):
            loss.backward(weights)


def test_every_form_may_be_captured_after_one_call(fd):
    """A first call of few short rows sets up what long rows, long lists and clusters need too."""
    calls = []
    for B, L, V, K in ((1, 1, 33, 2), (2, 3, 40009, 200), (1, 200, 20000, 7), (1, 1, 126464, 9)):
        kw, weights = inputs(B, L, V, K, HF, 51, True, masked=1.1)
        calls.append((kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], weights, kw["teacher_lse"]))
    for args in calls:
        graph = torch.cuda.CUDAGraph()
        if args is calls[0]:
            fd.fdllm_distill_step(*args)
            torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got = fd.fdllm_distill_step(*args)
        graph.replay()
        want = fd.fdllm_distill_step(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("temperature", [1e-3, 0.05, 30.0, 1e4])
@pytest.mark.parametrize("V", [700, 20003])
def test_temperatures_of_any_size(fd, temperature, V):
    for dtype, rest in ((BF, True), (FP, False)):
        kw, weights = inputs(2, 3, V, 9, dtype, 22, False, masked=1.1, temperature=temperature)
        if rest:
            kw["teacher_lse"] = torch.logsumexp(kw["top_logits"].double() / temperature, -1).float() + 0.7
        if temperature < 0.01:  # scores of several thousand: the tolerance's 64 covers the logits' part only
            kw["logits"] *= 0.01
            kw["top_logits"] *= 0.01
            if rest:
                kw["teacher_lse"] = torch.logsumexp(kw["top_logits"].double() / temperature, -1).float() + 0.7
        check(fd, kw, weights)


def test_another_stream_and_a_graph(fd):
    kw, weights = inputs(3, 5, 4099, 20, BF, 17, True)
    args = (kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], weights, kw["teacher_lse"])
    want = fd.fdllm_distill_step(*args)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = fd.fdllm_distill_step(*args, stream=other)
    again = fd.fdllm_distill_step(*args)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, again))
    outs = [torch.empty_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fdllm_distill_step(*args, out_loss=outs[0], out_grad=outs[1])
    for turn in range(3):
        kw["logits"].add_(torch.randn(kw["logits"].shape, generator=torch.Generator().manual_seed(turn)).cuda())
        kw["mask"].copy_((torch.rand(3, 5, generator=torch.Generator().manual_seed(turn)) < 0.5))
        graph.replay()
        want = fd.fdllm_distill_step(*args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("V", [1003, 1000])
def test_many_rows(fd, V):
    """More rows than the GPU holds at once; rows alike give results alike, whatever their place: the
    same bits where rows are whole 16-byte vectors.  (Of 1003 values of two bytes each row begins at
    another place of a vector, so sums are taken in another order: equal up to the tolerance.)"""
    kw, weights = inputs(1, 1, V, 9, BF, 18, True, masked=1.1)
    n = 3000
    big = {k: v.expand(n // 10, 10, *v.shape[2:]).contiguous() if isinstance(v, torch.Tensor) else v
           for k, v in kw.items()}
    big["mask"][::3, ::2] = 0
    w = weights.expand(n // 10, 10).contiguous()
    loss, grad = fd.fdllm_distill_step(big["logits"], big["mask"], big["top_index"], big["top_logits"], w,
                                       big["teacher_lse"])
    on = big["mask"] != 0
    assert bool((loss[~on] == 0).all()) and bool((grad[~on] == 0).all())
    if V % 8 == 0:
        assert bool((loss[on] == loss[on][0]).all()) and bool((grad[on] == grad[on][0]).all())
    want = ref.distill(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], kw["teacher_lse"], 1.0, weights)
    for got, exact, tol in ((loss[on], want[0][0], want[1][0]), (grad[on], want[2][0], want[3][0])):
        assert bool(((got.cpu().double() - exact).abs() <= tol).all())


@pytest.mark.parametrize("dtype,rest,B,V", [(BF, True, 36, 20011), (HF, False, 12, 32767), (FP, True, 41, 16001),
                                            (BF, False, 16, 70001), (FP, True, 25, 16411)])
def test_many_long_rows(fd, dtype, rest, B, V):
    """Several rows to a CTA, with one set of marks and with two, and the form of a CTA to each of many."""
    kw, weights = inputs(B, 13, V, 33, dtype, 21 + B, rest, masked=0.9)
    loss, grad = check(fd, kw, weights)
    into = kw["logits"].clone()
    again = fd.fdllm_distill_step(into, kw["mask"], kw["top_index"], kw["top_logits"], weights, kw["teacher_lse"],
                                  kw["temperature"], out_grad=into)
    assert torch.equal(again[0], loss) and torch.equal(into, grad)


@pytest.mark.parametrize("dtype,V,K", [(BF, 50021, 40), (FP, 49999, 1024), (HF, 131072, 7)])
def test_loss_of_many_long_rows(fd, dtype, V, K):
    """A CTA to each of more rows than the GPU holds; the same thirteen again and again."""
    kw, _ = inputs(1, 13, V, K, dtype, 31, True, masked=0.7, temperature=0.7)
    want, tol, _, _ = ref.distill(kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"], kw["teacher_lse"],
                                  0.7, torch.ones(1, 13, device="cuda"))
    big = {k: v.expand(100, *v.shape[1:]).contiguous() if isinstance(v, torch.Tensor) else v for k, v in kw.items()}
    stats = torch.full((100, 13, 4), 7.0, device="cuda")
    loss = fd.fdllm_distill_loss(out_stats=stats, **big)
    assert bool(((loss.cpu().double() - want).abs() <= tol).all())
    assert bool((stats[big["mask"] == 0] == 0).all())
    assert torch.equal(loss, fd.fdllm_distill_loss(**big))
    assert fd.fdllm_cache_status() == 0


def test_refusals(fd):
    kw, weights = inputs(2, 3, 64, 4, BF, 19, True)
    loss = lambda **more: fd.fdllm_distill_loss(**{**kw, **more})
    step = lambda **more: fd.fdllm_distill_step(**{**kw, "grad_loss": weights, **more})
    loss(), step()
    for call in (loss, step):
        for bad in (dict(temperature=0.0), dict(temperature=math.inf), dict(temperature=-1.0)):
            with pytest.raises(fd.FdllmError):
                call(**bad)
        for bad in (dict(mask=kw["mask"].bool()), dict(mask=kw["mask"][:1]), dict(logits=kw["logits"][0]),
                    dict(logits=kw["logits"][:, :, ::2]), dict(top_index=kw["top_index"].long()),
                    dict(top_index=kw["top_index"][:, :, :3]), dict(top_logits=kw["top_logits"].double()),
                    dict(teacher_lse=kw["teacher_lse"].cpu()), dict(logits=kw["logits"].cpu())):
            with pytest.raises((TypeError, ValueError)):
                call(**bad)
    with pytest.raises(TypeError):
        step(grad_loss=weights.bfloat16())
    with pytest.raises(ValueError):
        step(out_grad=torch.empty(2, 3, 65, dtype=BF, device="cuda"))


@pytest.mark.parametrize("dtype,B,L,V,K,masked", [(BF, 4, 80, 151937, 300, 0.7), (FP, 4, 60, 151937, 300, 0.7),
                                                  (BF, 1, 3, 126464, 64, 1.1), (HF, 1, 9, 131072, 1024, 0.9),
                                                  (FP, 2, 6, 126464, 33, 0.6), (BF, 2, 150, 50021, 200, 0.5),
                                                  (HF, 3, 5, 4099, 40, 0.8), (FP, 3, 70, 301, 9, 0.8)])
def test_gradient_in_place(fd, dtype, B, L, V, K, masked):
    """fdllm_distill_grad over the logits themselves: one CTA to a row and clusters of two to eight, with
    tokens listed in every share, several rows to each."""
    g = torch.Generator().manual_seed(34)
    logits = (1.5 * torch.randn(L, V, generator=g)).to(dtype).cuda().expand(B, L, V).contiguous()
    index = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(B * L)]).view(B, L, K).int()
    index[:, :, K // 2] = index[:, :, 0]  # (one twice)
    top = (3 + 4 * torch.rand(B, L, K, generator=g)).cuda()
    mask = (torch.rand(B, L, generator=g) < masked).to(torch.uint8).cuda()
    lse = torch.logsumexp(top, -1) + 1.0
    weights = torch.randn(B, L, generator=g).cuda()
    rest = mask, index.cuda(), top
    stats = torch.empty(B, L, 4, device="cuda")
    fd.fdllm_distill_loss(logits, *rest, lse, out_stats=stats)
    want = fd.fdllm_distill_grad(logits, *rest, stats, weights, lse)
    step = fd.fdllm_distill_step(logits, *rest, weights, lse)[1]
    assert bool((want[mask == 0] == 0).all()) and bool((want[mask != 0] != 0).any())
    assert torch.equal(step[mask == 0], want[mask == 0])
    for _ in range(3):
        x = logits.clone()
        got = fd.fdllm_distill_grad(x, *rest, stats, weights, lse, out_grad=x)
        assert got.data_ptr() == x.data_ptr() and torch.equal(x, want)
    assert fd.fdllm_cache_status() == 0


@pytest.mark.parametrize("V", [700, 20003])
@pytest.mark.parametrize("temperature", [1e-6, 1e-3, 0.05])
def test_a_teachers_gaps_at_low_temperatures(fd, temperature, V):
    """Logits near 8 that differ by a few temperatures: the teacher's probabilities are of the gaps, which
    fp32 holds, whatever logit / temperature is (8e6: a step of 0.5)."""
    for dtype in (FP, BF):
        kw, weights = inputs(2, 3, V, 9, FP, 32, False, masked=1.1, temperature=temperature)
        kw["logits"] = (8.0 + temperature * kw["logits"]).to(dtype)
        kw["top_logits"] = 8.0 + temperature * kw["top_logits"]
        check(fd, kw, weights)


@pytest.mark.parametrize("V", [700, 40009])
def test_a_teachers_sum_that_is_nan(fd, V):
    """Such a position's loss and gradient are NaN, whatever is listed: nothing, some tokens or all that
    the student allows."""
    kw, weights = inputs(1, 5, V, 9, FP, 33, True, masked=1.1)
    kw["teacher_lse"][0, :3] = math.nan
    kw["top_index"][0, 0] = -1
    at = kw["top_index"][0, 2].long()
    kept = kw["logits"][0, 2, at]
    kw["logits"][0, 2] = -math.inf
    kw["logits"][0, 2, at] = kept
    stats = torch.empty(1, 5, 4, device="cuda")
    loss = fd.fdllm_distill_loss(out_stats=stats, **kw)
    args = kw["logits"], kw["mask"], kw["top_index"], kw["top_logits"]
    grad = fd.fdllm_distill_grad(*args, stats, weights, kw["teacher_lse"])
    step = fd.fdllm_distill_step(*args, weights, kw["teacher_lse"])
    for x in (loss, step[0]):
        assert torch.isnan(x).tolist() == [[True] * 3 + [False] * 2]
    for x in (grad, step[1]):
        assert bool(torch.isnan(x[0, :3]).all()) and not bool(torch.isnan(x[0, 3:]).any())
