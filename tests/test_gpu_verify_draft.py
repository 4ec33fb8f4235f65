"""fdllm_verify_draft against a 64-bit walk: tokens, nodes and counts are equal wherever no test and
no draw lies within 1e-5 of its border (fp32 probabilities are that exact), and inputs that do are
few (their number is checked)."""
import math

import pytest
import torch

import draft_ref as ref

pytestmark = pytest.mark.gpu

BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
BORDER = 1e-5


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def logits(shape, g, dtype, std=1.5):
    x = std * torch.randn(shape, generator=g)
    x[..., :: max(1, shape[-1] // 7)] += 5.0
    return x.to(dtype)


def inputs(B, M, V, dtype, kind, seed, temperature=1.0):
    """A chain drawn from the draft's logits, a tree or a chain of chosen tokens, greedy or not."""
    g = torch.Generator().manual_seed(seed)
    target = logits((B, M, V), g, dtype)
    kw = dict(uniform=torch.rand(B, M, generator=g),
              noise=torch.empty(B, V).exponential_(generator=g).clamp_min(1e-8),
              temperature=0.0 if kind == "greedy" else temperature)
    near = target.float() + 0.5 * torch.randn(target.shape, generator=g)
    tokens = torch.randint(0, V, (B, M), generator=g)
    if kind == "draft":
        kw["draft"] = near[:, :M - 1].to(dtype)
        race = torch.empty(B, M - 1, V).exponential_(generator=g).clamp_min(1e-8)
        tokens[:, 1:] = (kw["draft"].float() / temperature - race.log()).argmax(-1)
    else:
        parents = torch.arange(M) - 1 - (torch.rand(B, M, generator=g) ** 2 * 6).long()
        parents = parents.clamp_min(0).int()
        best = near.topk(min(4, V), -1)[1]
        for b in range(B):
            fork = {}
            for j in range(1, M):
                up = int(parents[b, j])
                tokens[b, j] = best[b, up, fork.get(up, 0) % best.shape[-1]]
                fork[up] = fork.get(up, 0) + 1
        if kind != "chosen":
            kw["parents"] = parents
    return target, tokens.int(), kw


def cuda(x):
    return x.cuda() if isinstance(x, torch.Tensor) else x


def run(fd, target, tokens, **kw):
    got = [x.cpu() for x in fd.fdllm_verify_draft(
        target.cuda(), tokens.cuda(), **{k: cuda(v) for k, v in kw.items()})]
    assert fd.fdllm_cache_status() == 0
    return got


def check(fd, target, tokens, most_near=0, **kw):
    got = run(fd, target, tokens, **kw)
    *want, margin = ref.verify(target, tokens, **kw)
    sure = torch.tensor([m > BORDER for m in margin])
    assert int((~sure).sum()) <= most_near
    for a, b in zip(got, want):
        assert torch.equal(a[sure], b[sure])
    return got


@pytest.mark.parametrize("kind", ["draft", "tree", "chosen", "greedy"])
@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("B,M,V", [(1, 1, 1), (3, 2, 1), (2, 1, 50), (5, 2, 7), (3, 5, 1000),
                                   (2, 17, 4099), (4, 33, 8192), (3, 3, 50021), (2, 2, 126464)])
def test_shapes(fd, kind, dtype, B, M, V):
    target, tokens, kw = inputs(B, M, V, dtype, kind, seed=B + M + V)
    check(fd, target, tokens, **kw)


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("kind", ["draft", "greedy"])
@pytest.mark.parametrize("more", [-9, -8, -1, 0, 1, 7, 8, 9])
def test_rows_of_about_whole_chunks(fd, dtype, kind, more):
    """Rows that end a few values before or behind a chunk of 64 KB, at every place of a vector."""
    V = (1 if dtype == FP else 2) * 16384 + more
    target, tokens, kw = inputs(3, 3, V, dtype, kind, seed=more + 30)
    target[:, :, -1] = 11.0  # the last values count
    check(fd, target, tokens, **kw)
    lens = torch.tensor([3, 1, 2], dtype=torch.int32)
    check(fd, target, tokens, lens=lens, **kw)


@pytest.mark.parametrize("kind", ["draft", "tree", "chosen", "greedy"])
@pytest.mark.parametrize("B,M,V,dtype", [(16, 9, 50021, FP), (5, 40, 70003, BF), (40, 5, 81920, HF),
                                         (1, 120, 126464, BF), (70, 12, 17000, BF)])
def test_rows_that_the_walk_cannot_reach(fd, kind, B, M, V, dtype):
    """Large calls: NaN in the rows of nodes that are not on the way changes nothing."""
    target, tokens, kw = inputs(B, M, V, dtype, kind, seed=B + M)
    lens = (M - torch.arange(B) % 3 * (M // 3)).int()
    got = check(fd, target, tokens, most_near=1, lens=lens, **kw)
    on_path = torch.zeros(B, M, dtype=torch.bool)
    for b in range(B):
        on_path[b, got[1][b][got[1][b] >= 0].long()] = True
    target[~on_path] = math.nan
    if "draft" in kw:
        kw["draft"][~on_path[:, :-1]] = math.nan
    again = run(fd, target, tokens, lens=lens, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("kind", ["tree", "greedy"])
@pytest.mark.parametrize("B,M,V,dtype", [(3, 40, 60001, BF), (1, 1024, 17003, HF), (20, 24, 17003, FP),
                                         (41, 128, 4999, HF), (160, 20, 8199, HF), (7, 4, 126464, FP)])
def test_trees_read_along_the_way(fd, kind, B, M, V, dtype):
    """Large calls with trees of every depth: rows of any alignment, more sequences than SMs; chains and
    stars; a row that is no number in the middle of a path."""
    target, tokens, kw = inputs(B, M, V, dtype, kind, seed=B + M + 1)
    lens = (M + 1 - torch.arange(B) % 4 * (M // 3)).int()
    check(fd, target, tokens, most_near=1, lens=lens, **kw)
    # every node of a chain is taken, however deep; the first child's subtree or another's
    chain = torch.arange(-1, M - 1).expand(B, M).int().contiguous()
    if kind == "greedy":
        tokens[:, 1:] = target[:, :-1].float().argmax(-1)
    else:
        kw["uniform"][:] = 0.0
        tokens[:, 1:] = (7 * torch.arange(M - 1) + torch.arange(B)[:, None]) % V
    kw["parents"] = chain
    got = check(fd, target, tokens, **kw)
    assert got[2].tolist() == [M - 1] * B and torch.equal(got[0][:, :-1], tokens[:, 1:])
    at = M // 2
    target[0, at, V // 2] = math.nan
    got = check(fd, target, tokens, **kw)
    assert got[2].tolist() == [-1] + [M - 1] * (B - 1)
    kw["parents"] = chain.clone()
    kw["parents"][:, at:] = 0  # one deep path, and leaves: the NaN is a leaf's
    if kind == "tree":
        kw["uniform"][:, at:] = 1.0 - 2.0 ** -24
    got = check(fd, target, tokens, **kw)
    assert int(got[2].min()) >= at - 1
    kw["parents"][:] = 0
    check(fd, target, tokens, lens=lens, **kw)


def test_trees_read_along_the_way_replayed_and_apart(fd):
    target, tokens, kw = inputs(6, 33, 40003, BF, "tree", seed=44)
    want = check(fd, target, tokens, **kw)
    wide = torch.zeros(7, 35, 40006, dtype=BF, device="cuda").transpose(0, 1)[:33].transpose(0, 1)[1:, :, 3:]
    wide.copy_(target)
    kw, tokens = {k: cuda(v) for k, v in kw.items()}, tokens.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for got in (fd.fdllm_verify_draft(wide, tokens, **kw), fd.fdllm_verify_draft(wide, tokens, stream=side, **kw)):
        torch.cuda.synchronize()
        assert all(torch.equal(a.cpu(), b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [fd.fdllm_verify_draft(wide, tokens, **kw) for _ in range(2)]
    for turn in range(3):
        kw["uniform"].copy_(torch.rand(6, 33, generator=torch.Generator().manual_seed(turn)))
        graph.replay()
        again = fd.fdllm_verify_draft(wide, tokens, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(again, *outs))


@pytest.mark.parametrize("seed", range(16))
def test_many_sequences(fd, seed):
    kind = ("draft", "tree", "chosen", "greedy")[seed % 4]
    B, M, V = 70 + seed, 2 + seed, 300 + 7 * seed
    target, tokens, kw = inputs(B, M, V, (BF, HF, FP)[seed % 3], kind, seed, (0.5, 1.0, 1.7)[seed // 4 % 3])
    lens = (torch.arange(B) * 7 % (M + 3)).int() - 1  # below 1 and above M among them
    got = check(fd, target, tokens, most_near=2, lens=lens, **kw)
    if kind == "draft":  # both ends happen
        assert int((got[2] == 0).sum()) and int((got[2] > 0).sum())


def test_rows_behind_the_nodes_are_not_read(fd):
    for kind in ("draft", "tree", "greedy"):
        target, tokens, kw = inputs(4, 9, 515, BF, kind, seed=3)
        lens = torch.tensor([1, 4, 9, 6], dtype=torch.int32)
        want = run(fd, target, tokens, lens=lens, **kw)
        for b, n in enumerate(lens.tolist()):
            target[b, n:] = math.nan
            tokens[b, n:] = -5
            if "draft" in kw:
                kw["draft"][b, n - 1:] = math.nan
        got = check(fd, target, tokens, lens=lens, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_long_chain_and_wide_star(fd):
    target, tokens, kw = inputs(2, 1024, 65, HF, "draft", seed=5)
    kw["draft"] = target[:, :-1].clone()  # the target itself: every token is taken
    kw["uniform"][:] = 1.0 - 2.0 ** -14
    got = run(fd, target, tokens, **kw)
    assert got[2].tolist() == [1023, 1023]
    assert torch.equal(got[0][:, :-1], tokens[:, 1:])
    # a root with 1023 children: half of their tokens repeat, and all but the last are turned down
    target, tokens, kw = inputs(2, 1024, 2048, FP, "tree", seed=6)
    kw["parents"][:] = 0
    tokens[:, 1:] = (torch.arange(1023) % 512).int()
    target[:, 0, :512] = -30.0
    kw["uniform"][:] = 0.5
    got = check(fd, target, tokens, **kw)
    assert got[2].tolist() == [0, 0] and bool((got[0][:, 0] >= 512).all())
    kw["parents"][:, 1000:] = -1
    kw["parents"][0, 700:900] = 5000
    check(fd, target, tokens, **kw)


def test_unreachable_nodes_and_foreign_tokens(fd):
    target, tokens, kw = inputs(3, 6, 100, FP, "tree", seed=8)
    for b, bad in enumerate((-1, 100, 2 ** 31 - 1)):
        tokens[b, 1:4] = bad
    kw["parents"][:, 1:] = ints([0, 0, 0, -7, 9]).cpu()
    got = check(fd, target, tokens, **kw)
    assert got[2].tolist() == [0, 0, 0]
    target, tokens, kw = inputs(3, 4, 100, FP, "draft", seed=9)
    tokens[:, 1] = -1
    kw["uniform"][:, 1] = 0.0
    check(fd, target, tokens, **kw)
    assert run(fd, target, tokens, temperature=0.0)[2].tolist() == [0, 0, 0]


@pytest.mark.parametrize("dtype", [BF, HF, FP])
def test_non_finite_rows(fd, dtype):
    """Only those on the way count."""
    target, tokens, kw = inputs(6, 4, 40, dtype, "greedy", seed=10)
    best = target.float().argmax(-1)
    tokens[:, 1:] = best[:, :3]
    target[0, 0, 39] = math.nan
    target[1, 2, 0] = math.inf
    target[2, 1] = -math.inf
    target[3, 3, 5] = -math.inf  # a masked token: nothing
    tokens[4, 1] = (best[4, 0] + 1) % 40  # turned down: what is behind does not matter
    target[4, 1:] = math.nan
    target[5, 3, 7] = math.nan
    got = check(fd, target, tokens, temperature=0.0)
    assert got[2].tolist() == [-1, -1, -1, 3, 0, -1]
    assert bool((got[0][[0, 1, 2, 5]] == -1).all()) and bool((got[1][[0, 1, 2, 5]] == -1).all())
    target, tokens, kw = inputs(3, 3, 40, dtype, "draft", seed=11)
    kw["uniform"][:] = torch.tensor([0.0, 0.0, 1.0 - 2.0 ** -24])
    kw["draft"][0, 0, 3] = math.nan
    kw["draft"][1, 1] = -math.inf
    got = check(fd, target, tokens, **kw)
    assert got[2][0] == -1 and got[2][1] == -1 and got[2][2] >= 0


@pytest.mark.parametrize("dtype", [BF, HF, FP])
def test_values_of_any_size(fd, dtype):
    """Rows shifted far from zero, of the type's lowest value, with masked tokens."""
    low = torch.finfo(dtype).min
    for shift, std in ((0.0, 60.0), (3e4 if dtype == HF else 1e30, 0.0), (low, 0.0)):
        target, tokens, kw = inputs(3, 4, 77, dtype, "chosen", seed=12)
        if std == 0.0:
            target[:] = shift  # all tokens alike
            target[:, :, ::2] = -math.inf if shift != low else low
        else:
            target *= std / 1.5
        check(fd, target, tokens, **kw)
    target, tokens, kw = inputs(3, 4, 77, dtype, "draft", seed=13)
    kw["draft"][:, :, 5:] = -math.inf
    tokens[:, 1:] = torch.tensor([2, 50, 3])  # the second was drawn with probability 0: taken
    check(fd, target, tokens, **kw)


def test_same_rows_are_always_taken(fd):
    target, tokens, kw = inputs(20, 8, 900, BF, "draft", seed=14)
    kw["draft"] = target[:, :-1].clone()
    kw["uniform"][:] = 1.0 - 2.0 ** -14
    got = run(fd, target, tokens, **kw)
    assert got[2].tolist() == [7] * 20


def test_no_weight_left_gives_way_to_the_target(fd):
    """One token has all of the target's mass: the draft had it too and was turned down by nothing
    but a rounding, or the tree tried it."""
    target = torch.full((2, 2, 30), -math.inf)
    target[:, :, 7] = 1.0
    tokens = torch.full((2, 2), 7, dtype=torch.int32)
    uniform = torch.full((2, 2), 1.0)  # (not below 1: turned down all the same)
    noise = torch.ones(2, 30)
    for kw in (dict(draft=target[:, :1].clone()), dict()):
        got = run(fd, target, tokens, uniform=uniform, noise=noise, **kw)
        assert got[2].tolist() == [0, 0] and got[0][:, 0].tolist() == [7, 7]


def test_noise_that_is_no_number(fd):
    target = torch.zeros(4, 1, 20)
    noise = torch.full((4, 20), 3.0)
    noise[0, 5] = 1.0
    noise[1] = math.nan
    noise[1, 9] = 7.0
    noise[2, 4:] = -1.0
    noise[3, :] = math.inf
    noise[3, 11] = 2.0
    tokens = torch.zeros(4, 1, dtype=torch.int32)
    got = run(fd, target, tokens, uniform=torch.zeros(4, 1), noise=noise)
    assert got[0][:, 0].tolist() == [5, 9, 0, 11]


@pytest.mark.parametrize("kind", ["draft", "tree"])
def test_what_comes_out_is_the_targets_distribution(fd, kind):
    """The first token over many sequences with the same logits: counts within 5 standard
    deviations of the target's probabilities, however far the draft's are."""
    n, V = 40000, 6
    g = torch.Generator().manual_seed(15)
    row, other = torch.randn(V, generator=g), torch.randn(V, generator=g) * 2
    target = row.expand(n, 3, V).contiguous()
    kw = dict(uniform=torch.rand(n, 3, generator=g),
              noise=torch.empty(n, V).exponential_(generator=g).clamp_min(1e-10), temperature=0.8)
    if kind == "draft":
        q = torch.softmax(other / 1.3, 0)
        tokens = torch.multinomial(q.expand(n, V), 3, True, generator=g).int()
        kw.update(draft=other.expand(n, 2, V).contiguous(), draft_temperature=1.3)
    else:
        tokens = torch.tensor([0, 2, 4], dtype=torch.int32).expand(n, 3).contiguous()
        kw["parents"] = torch.tensor([-1, 0, 0], dtype=torch.int32).expand(n, 3).contiguous()
    got = run(fd, target, tokens, **kw)
    p = torch.softmax(row.double() / 0.8, 0)
    counts = torch.bincount(got[0][:, 0].long(), minlength=V).double()
    assert bool(((counts - n * p).abs() <= 5 * torch.sqrt(n * p * (1 - p))).all())


def test_ties_go_to_the_lowest_token(fd):
    for dtype in (BF, HF, FP):
        for V in (1000, 4097):
            target = torch.zeros(1, 1, V, dtype=dtype)
            target[0, 0, 13::50] = 2.0
            tokens = torch.zeros(1, 1, dtype=torch.int32)
            assert run(fd, target, tokens, temperature=0.0)[0].tolist() == [[13]]
            got = run(fd, target, tokens, uniform=torch.zeros(1, 1), noise=torch.ones(1, V))
            assert got[0].tolist() == [[13]]


def test_deterministic_on_another_stream_in_a_graph_and_side_by_side(fd):
    target, tokens, kw = inputs(7, 6, 5003, BF, "draft", seed=16)
    target, tokens, kw = cuda(target), cuda(tokens), {k: cuda(v) for k, v in kw.items()}
    want = fd.fdllm_verify_draft(target, tokens, **kw)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = fd.fdllm_verify_draft(target, tokens, stream=other, **kw)
    again = fd.fdllm_verify_draft(target, tokens, **kw)  # at the same time
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)
    outs = [torch.empty_like(x) for x in want]
    ws = torch.full((fd.fdllm_verify_draft_workspace_bytes(7, 6, 5003),), 255, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fdllm_verify_draft(target, tokens, out_tokens=outs[0], out_nodes=outs[1], out_n=outs[2],
                              workspace=ws, **kw)
    for turn in range(3):
        kw["uniform"].copy_(torch.rand(7, 6, generator=torch.Generator().manual_seed(turn)))
        graph.replay()
        graph.replay()
        want = fd.fdllm_verify_draft(target, tokens, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("V", [512, 515, 50021])
def test_rows_of_larger_tensors(fd, dtype, V):
    """Rows that lie apart, at any alignment, in any order of batch and rows, or repeat."""
    target, tokens, kw = inputs(3, 4, V, dtype, "draft", seed=18 + V)
    want = check(fd, target, tokens, **kw)
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(3, 9, V + 5, generator=g).to(dtype).cuda()
    wide[:, 2:6, 3:V + 3] = target.cuda()
    turned = torch.randn(5, 3, V + 1, generator=g).to(dtype).cuda().transpose(0, 1)
    turned[:, 1:4, 1:] = kw["draft"].cuda()
    more = {k: cuda(v) for k, v in kw.items() if k != "draft"}
    got = fd.fdllm_verify_draft(wide[:, 2:6, 3:V + 3], tokens.cuda(), draft=turned[:, 1:4, 1:], **more)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(got, want))
    one = target[:1, :1].cuda().expand(3, 4, V)
    want = run(fd, one.contiguous().cpu(), tokens, **{k: v for k, v in kw.items() if k != "draft"})
    got = fd.fdllm_verify_draft(one, tokens.cuda(), **more)
    assert all(torch.equal(a.cpu(), b) for a, b in zip(got, want))


def test_refusals(fd):
    target, tokens, kw = inputs(2, 3, 64, BF, "draft", seed=17)
    target, tokens, kw = cuda(target), cuda(tokens), {k: cuda(v) for k, v in kw.items()}
    call = lambda **more: fd.fdllm_verify_draft(**{**dict(target=target, tokens=tokens), **kw, **more})
    call()
    parents = ints([[-1, 0, 0]] * 2)
    for bad in (dict(parents=parents), dict(temperature=0.0), dict(temperature=-1.0), dict(noise=None),
                dict(temperature=math.nan), dict(uniform=None), dict(draft_temperature=0.0),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(fd.FdllmError):
            call(**bad)
    for bad in (dict(draft=kw["draft"].float()), dict(draft=target), dict(tokens=tokens.long()),
                dict(tokens=tokens[:, :2]), dict(uniform=kw["uniform"].cpu()),
                dict(target=torch.cat((target, target), -1)[:, :, ::2]),
                dict(target=target.double()), dict(target=target[0]), dict(lens=ints([1]))):
        with pytest.raises((TypeError, ValueError)):
            call(**bad)


@pytest.mark.parametrize("kind,M,V", [("draft", 4, 515), ("draft", 5, 50021), ("tree", 40, 50021)])
def test_a_wait_that_ran_out_is_told_by_every_sequence(fd, kind, M, V):
    """Short rows, long ones, and a tree that is read along the way: after a wait that ran out nothing
    is reported as taken until the status was asked for; then all is as before, whatever the workspace
    holds."""
    target, tokens, kw = inputs(5, M, V, BF, kind, seed=41)
    target, tokens, kw = cuda(target), cuda(tokens), {k: cuda(v) for k, v in kw.items()}
    size = fd.fdllm_verify_draft_workspace_bytes(5, M, V)
    call = lambda fill: fd.fdllm_verify_draft(
        target, tokens, workspace=torch.full((size,), fill, dtype=torch.uint8, device="cuda"), **kw)
    want = call(0)
    assert bool((want[2] >= 0).all())
    assert fd.fdllm_cache_status() == 0
    assert fd.fdllm_cache_check_wait(1) == 0
    out, nodes, n = call(0)
    assert n.tolist() == [-2] * 5 and bool((out == -1).all()) and bool((nodes == -1).all())
    assert fd.fdllm_cache_status() != 0
    assert fd.fdllm_cache_status() == 0
    for fill in (0, 1, 255):
        assert all(torch.equal(a, b) for a, b in zip(call(fill), want))
