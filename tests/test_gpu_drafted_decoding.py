"""The drafted-decoding example: its operators together, each against its 64-bit reference on what
the pass handed it, and the pass against a plain forward in 64 bits."""
import importlib.util
import os

import pytest
import torch

import cache_ref
import draft_ref

pytestmark = pytest.mark.gpu

TREE = [-1, 0, 0, 0, 1, 1, 2, 4, 7]


@pytest.fixture(scope="module")
def example(fd):
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "drafted_decoding.py")
    spec = importlib.util.spec_from_file_location("drafted_decoding", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(example, model, prefix, lens, tokens, parents):
    """`forward_nodes` in fp64 on the CPU over the values that the cache holds."""
    B, M = tokens.shape
    norm = lambda y: y / torch.sqrt((y * y).mean(-1, keepdim=True) + example.EPS)
    x = model.embed.cpu().double()[tokens.cpu().long()]
    sees, depth = draft_ref.tree_mask(parents.cpu())
    at = (lens.cpu().long()[:, None] + depth).flatten()
    group = model.heads // model.kv_heads
    for layer, cache in zip(model.layers, prefix.caches):
        w = {name: t.cpu().double() for name, t in layer.items()}
        qkv = (norm(x) @ w["qkv"].t()).view(B * M, -1, model.head_dim)
        turn = lambda y, weight: cache_ref.rope(y, weight, at, None, model.inv_freq, example.EPS, False)
        q = turn(qkv[:, :model.heads], w["q_norm"]).view(B, M, model.heads, -1)
        k = turn(qkv[:, model.heads:-model.kv_heads], w["k_norm"]).view(B, M, model.kv_heads, -1)
        v = qkv[:, -model.kv_heads:].reshape(B, M, model.kv_heads, -1)
        kd, vd = cache_ref.unpack_cache(cache)
        out = torch.zeros_like(q)
        for b in range(B):
            ck, cv = (cache_ref.sequence(t, prefix.table.cpu()[b], cache.page_size, int(lens[b])) for t in (kd, vd))
            for i in range(M):
                on = sees[b, i]
                for h in range(model.heads):
                    kh = torch.cat((ck[h // group], k[b, on, h // group]))
                    vh = torch.cat((cv[h // group], v[b, on, h // group]))
                    out[b, i, h] = torch.softmax(kh @ q[b, i, h] * model.head_dim ** -0.5, 0) @ vh
        x = x + out.flatten(2) @ w["out"].t()
        y = norm(x) @ w["up"].t()
        x = x + (y * torch.sigmoid(y)) @ w["down"].t()
    return norm(x) @ model.vocab_w.cpu().double().t()


@pytest.mark.parametrize("tree", [None, TREE])
def test_passes(example, fd, tree):
    """Two layers round their streams and products to bfloat16 some ten times each, at 2^-9 of
    values of order one: the logits' root mean square error stays below 2^-5 of their own."""
    model, drafter = example.Model(seed=3), example.Drafter(1024, seed=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    B, P, nodes = 3, 37, 9
    prompt = torch.randint(0, 1023, (B, P), generator=torch.Generator().manual_seed(6)).int().cuda()
    prefix = example.PrefixCache(model, B, P + 60)
    chain = torch.arange(-1, P - 2, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    logits, state = example.forward_nodes(model, prefix, prompt[:, :-1], chain)
    prefix.append(state)
    root, taken = prompt[:, -1], 0
    for _ in range(4):
        head = drafter.head.clone()
        held = [[t.clone() for t in cache_ref.unpack_cache(c)] for c in prefix.caches]
        s = example.step(model, drafter, prefix, root, nodes, tree, g)
        # (what was appended lies behind these lengths)
        want = plain(example, model, prefix, s["lens"], s["nodes"], s["parents"])
        error = float(((s["logits"].cpu().double() - want) ** 2).mean().sqrt() / (want ** 2).mean().sqrt())
        assert error <= 2.0 ** -5, error
        # the tokens, from the pass's own logits
        drawn = None if s["drawn"] is None else s["drawn"].cpu()
        *found, margin = draft_ref.verify(s["logits"].cpu(), s["nodes"].cpu(),
                                          None if tree is None else s["parents"].cpu(), None, drawn, 1.0, 1.0,
                                          s["uniform"].cpu(), s["noise"].cpu())
        assert min(margin) > 1e-5
        for a, b in zip((s["tokens"], s["path"], s["n"]), found):
            assert torch.equal(a.cpu(), b)
        # the cache: the path's rows behind what was there, nothing else
        for cache, layer, was in zip(prefix.caches, s["state"], held):
            now = cache_ref.unpack_cache(cache)
            for b in range(B):
                n, m = int(s["lens"][b]), int(s["n"][b]) + 1
                path = s["path"][b, :m].long()
                for x, y, kind in zip(now, was, ("k", "v")):
                    row = lambda t, end: cache_ref.sequence(t, prefix.table.cpu()[b], cache.page_size, end)
                    assert torch.equal(row(x, n), row(y, n))
                    assert torch.equal(row(x, n + m)[:, n:], cache_ref.values(layer[kind][b, path]).transpose(0, 1))
        assert prefix.lens.tolist() == [int(a) + int(b) + 1 for a, b in zip(s["lens"], s["n"])]
        # the drafter's step: the formula's gradient of its logits, through its projection
        x = example.rms(drafter.embed[s["nodes"].long()])
        rows = x @ head.bfloat16().t()
        mask = torch.zeros(B, nodes, dtype=torch.uint8)
        for b in range(B):
            mask[b, s["path"][b, :int(s["n"][b]) + 1].long().cpu()] = 1
        values, index = s["logits"].float().topk(32, -1)
        count = int(mask.sum())
        weights = torch.full((B, nodes), 1.0 / count)
        lse = torch.logsumexp(s["logits"].float(), -1)
        loss, loss_tol, grad, grad_tol = draft_ref.distill(rows, mask, index, values, lse, 1.0, weights)
        assert abs(float(s["loss"]) - float(loss.sum()) / count) <= float(loss_tol.sum()) / count + 1e-5
        moved = (head - drafter.head).cpu().double()
        x64 = x.cpu().double().flatten(0, 1)
        exact = drafter.rate * grad.flatten(0, 1).t() @ x64
        # (a product in bf16 with fp32 sums: its result rounded, and the gradient's own tolerance)
        tol = drafter.rate * grad_tol.flatten(0, 1).t() @ x64.abs() + 2.0 ** -8 * exact.abs() + \
            32 * 2.0 ** -24 * (drafter.rate * grad.abs().flatten(0, 1).t() @ x64.abs() + head.abs().cpu().double())
        assert bool(((moved - exact).abs() <= tol).all())
        taken += int(s["n"].sum())
        root = s["tokens"].gather(1, s["n"].long()[:, None])[:, 0]
    assert fd.fdllm_cache_status() == 0


@pytest.mark.parametrize("tree", [None, TREE])
def test_decoding(example, tree):
    prompt = torch.randint(0, 1023, (3, 21), generator=torch.Generator().manual_seed(8)).int().cuda()
    runs = []
    for _ in range(2):
        done, losses, prefix = example.decode(example.Model(seed=7), example.Drafter(1024, seed=8), prompt, 20, tree=tree)
        assert all(0 <= t < 1024 for d in done for t in d) and losses
        assert prefix.lens.tolist() == [20 + len(d) for d in done]
        runs.append((done, losses))
    assert runs[0] == runs[1]


def test_a_pass_in_a_graph(example, fd):
    """Mask, attention and verification captured together and replayed on new tokens."""
    model = example.Model(layers=1, seed=9)
    B, M = 2, len(TREE)
    prompt = torch.randint(0, 1023, (B, 30), generator=torch.Generator().manual_seed(10)).int().cuda()
    prefix = example.PrefixCache(model, B, 64)
    chain = torch.arange(-1, 29, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    prefix.append(example.forward_nodes(model, prefix, prompt, chain)[1])
    tokens = torch.randint(0, 1023, (B, M), generator=torch.Generator().manual_seed(11)).int().cuda()
    parents = torch.tensor(TREE, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()
    uniform = torch.rand(B, M, generator=torch.Generator().manual_seed(12)).cuda()
    noise = torch.empty(B, 1024).exponential_(generator=torch.Generator().manual_seed(13)).cuda()

    def once():
        logits, _ = example.forward_nodes(model, prefix, tokens, parents)
        return (logits,) + fd.fdllm_verify_draft(logits, tokens, parents=parents, uniform=uniform, noise=noise)

    once()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = once()
    for turn in range(3):
        tokens.copy_(torch.randint(0, 1023, (B, M), generator=torch.Generator().manual_seed(20 + turn)).int())
        graph.replay()
        want = once()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("tree", [None, TREE])
def test_slow_sequences_are_decoded_to_their_end(example, tree):
    """Every sequence has its tokens, and none much more: those that are done wait for the others."""
    prompt = torch.randint(0, 1023, (8, 21), generator=torch.Generator().manual_seed(14)).int().cuda()
    model, drafter = example.Model(seed=15), example.Drafter(1024, seed=16)
    done, _, prefix = example.decode(model, drafter, prompt, 120, tree=tree)
    nodes = 6 if tree is None else len(TREE)
    assert all(120 <= len(d) < 120 + nodes for d in done)
    assert prefix.lens.tolist() == [20 + len(d) for d in done]
